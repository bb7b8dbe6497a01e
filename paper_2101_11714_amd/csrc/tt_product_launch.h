// Which kernel computes a product, and its launches.  The kernels of each type are compiled in a file of their own (tt_product_*.hip).
#pragma once

#include "tt_product_few.h"
#include "tt_product_stream.h"
#include "tt_rows_args.h"

namespace tt {

// C = A B^T, of M x N with sums over K, by tiles and parts of k.
struct Size {
    int64_t M, N, K;
};

struct Plan {
    int64_t tiles_m, tiles_n;
    int parts;
    int64_t k_part;
};

constexpr int64_t MOST_TILES = 512;                          // workgroups that parts are made for

// Kinds of tiles, and what a step of 128 bytes of k takes, in us, as measured on 256 compute units.
// 16 bits.  256 x 256, one on a compute unit: 1.87 (8,192 x 16,384 x 4,096: 1,127 TFLOP/s).  128 x 128: 0.70 alone on its compute unit and 1.17 beside another
// one (2,048 x 2,048 x 4,096, one tile each: 48 us, by the others in four parts 41 and the parts' sums 15; 8,192 x 4,096 x 4,096: 293, by the others 221).
// 32 bits.  128 x 64 takes 1.13 of a compute unit, 64 x 64 0.60 and 32 x 64 0.32, alone or beside others (2,048^3 149, 148 and 152 us; 512^3 14.7, 14.7 and 10.1,
// 1,001 x 777 x 1,283 41, 37 and 32, 1,024 x 4,096 x 4,096 280, 280 and 291; 256 x 1,024 x 1,024 24 us as 64 tiles of 64 x 64, in four parts 15).
struct TileKind {
    int64_t m, n, room;          // room: how many tiles run together
    double step, alone;
};
constexpr TileKind KINDS[2][3] = {{{128, 64, 256, 1.13, 1.13}, {64, 64, 256, 0.60, 0.60}, {32, 64, 256, 0.32, 0.32}}, {{256, 256, 256, 1.87, 1.87}, {128, 128, 512, 1.17, 0.70}, {}}};

// Which kind and how many parts of each of n products that run together: whatever should be done first.  Parts cost a launch, and their sums
// a write and a read.
inline int plan_of(const Size *d, int n, int32_t type, Plan *p, double &best)
{
    const int64_t step = 128 / element_bytes(type);
    const bool f32 = type == TT_F32;
    int best_kind = 0;
    best = 0;
    for (int kind = 0; kind < (f32 ? 3 : 2); ++kind) {
        const TileKind &t = KINDS[!f32][kind];
        const int64_t most = f32 ? 2 * MOST_TILES : t.room;
        int64_t tiles[2] = {}, steps[2] = {};
        for (int i = 0; i < n; ++i) {
            tiles[i] = ceil_div(d[i].M, t.m) * ceil_div(d[i].N, t.n);
            steps[i] = tiles[i] ? ceil_div(d[i].K, step) : 0;
        }
        auto can = [&](int i, int64_t parts) { return parts == 1 || (i < n && parts * tiles[i] <= most && 4 * parts <= steps[i]); };
        int64_t parts[2];
        for (parts[0] = 1; can(0, parts[0]); parts[0] *= 2)
            for (parts[1] = 1; can(1, parts[1]); parts[1] *= 2) {
                int64_t wgs = 0, work = 0, longest = 0, shortest = 0;
                double us = 0;
                bool joins = false;
                for (int i = 0; i < n; ++i) {
                    if (!tiles[i]) continue;
                    const int64_t each = ceil_div(steps[i], parts[i]);
                    if (wgs == 0 || each < shortest) shortest = each;
                    if (each > longest) longest = each;
                    wgs += tiles[i] * parts[i];
                    work += tiles[i] * parts[i] * each;
                    if (parts[i] > 1) us += (double)parts[i] * (double)d[i].M * (double)d[i].N * 8.0 / 5.0e6;
                    joins |= parts[i] > 1;
                }
                if (joins) us += f32 ? 6.0 : 3.0;
                if (n == 2 && kind == 2) us *= 1.15;         // (gradients' operands: 354 x 4,096 x 4,480 294 us, by larger tiles 270)
                if (wgs <= 256) {
                    us += t.alone * (double)longest;
                } else if (n == 1 || shortest == longest) {
                    const int64_t whole = wgs / t.room, rest = wgs % t.room;
                    us += (double)longest * (t.step * (double)(whole + (rest > 256 || (rest && t.room == 256))) + (rest && rest <= 256 && t.room > 256 ? t.alone : 0.0));
                } else {
                    const double all = (double)work / (double)t.room + 0.5 * (double)shortest;
                    us += t.step * (all > (double)longest ? all : (double)longest);
                }
                if (best == 0 || us < best) {
                    best = us;
                    best_kind = kind;
                    for (int i = 0; i < n; ++i) {
                        const int64_t each = ceil_div(steps[i], parts[i]);
                        p[i].tiles_m = tiles[i] ? ceil_div(d[i].M, t.m) : 0;
                        p[i].tiles_n = ceil_div(d[i].N, t.n);
                        p[i].k_part = (each > 0 ? each : 1) * step;
                        p[i].parts = steps[i] > 0 ? (int)ceil_div(d[i].K, p[i].k_part) : 1;
                    }
                }
            }
    }
    return best_kind;
}

// Whether the kernel of few rows takes a product of up to 64, as one of 16, 32 or 64: it needs no parts and no copies, but every workgroup goes through all of k,
// which takes (1.6 to 7.3) ns for a value of 16 bits, and twice as long for one of 32.  bf16: 17 x 4,096 x 4,096 12 us instead of 15 by tiles, 48 x 1,024 x
// 4,096 8.6 instead of 12, but 64 x 8,192 x 1,024 39 instead of 17 and 8 x 16,384 x 256 26 instead of 16; fp32: 32 x 4,096 x 4,096 27 and 31, 64 x 8,192 x 1,024
// 77 and 20.
constexpr int64_t PF_CLASS[3] = {16, 32, 64};

inline bool few(int rows_class, int64_t N, int64_t K, int32_t type, bool whole)
{
    const int64_t M = PF_CLASS[rows_class];
    const bool two = M > 16 && N >= 256 * 32;                // two blocks of columns a workgroup
    const double ns = M == 16 ? 1.6 : M == 32 ? (two ? 4.3 : 2.8) : (two ? 7.3 : 4.6), wgs = (double)ceil_div(N, two ? 32 : 16) / 256.0;
    const double us = 3.0 + (double)K * ns * 1e-3 * (type == TT_F32 ? 2.0 : 1.0) * (wgs > 1.0 ? wgs : 1.0);
    Plan p;
    double tiles;
    const Size d{M, N, K};
    plan_of(&d, 1, type, &p, tiles);
    return us <= tiles + 6.0 + (whole ? 0.0 : 8.0);
}

inline bool few_rows(int64_t M, int64_t N, int64_t K, int32_t type, bool whole) { return M <= PF_MOST && few(M <= 16 ? 0 : M <= 32 ? 1 : 2, N, K, type, whole); }

// What the parts' sums of a product take: nothing where it has one part, whose sums go through the epilogue.
inline size_t parts_bytes(const Size &d, const Plan &p) { return p.parts > 1 ? (size_t)p.parts * (size_t)d.M * (size_t)(8 * ceil_div(d.N, 8)) * sizeof(float) : 0; }

// What they take at most for M rows, or for fewer, whatever the product's way: with more rows there are fewer parts, but no more than
// 256 wide tiles' or MOST_TILES narrow ones' worth of rows, or twice as many of 64 columns.
inline size_t product_bytes(int64_t M, int64_t N, int64_t K, int32_t type)
{
    if (M <= 0 || N <= 0) return 0;
    const int64_t most = ceil_div(K, 128 / element_bytes(type)) / 4, wide = ceil_div(N, 256);
    if (wide >= 256 || most < 2) return 0;
    const int64_t rows = M * (most < 2 * MOST_TILES ? most : 2 * MOST_TILES), tiled = MOST_TILES * 256 / wide;
    return (size_t)(rows < tiled ? rows : tiled) * (size_t)(8 * ceil_div(N, 8)) * sizeof(float);
}

// rows of whole 16-byte chunks, at strides that a buffer's offsets can bear
inline bool whole_chunks(const tt_rows_t &r, int64_t columns)
{
    return r.type == TT_F32 || (columns % 8 == 0 && r.ld % 8 == 0 && (uintptr_t)r.data % 16 == 0 && r.ld <= PS_MOST_STRIDE);
}

// bytes of a copy in whole chunks
inline size_t packed_bytes(int64_t rows, int64_t columns, int32_t type) { return (size_t)rows * (size_t)(8 * ceil_div(columns, 8)) * (size_t)element_bytes(type); }

// An operand: rows, dense along their columns; packed: where its copy in whole chunks goes where it needs one, null: it is not to be copied (few rows
// bear any alignment).
struct Operand {
    const void *data;
    int64_t ld, rows, columns;
    void *packed;
};

// what copies the operands that are to be copied, by so many workgroups; the operands then are the copies
inline PackArgs pack_args(Operand &a, Operand &b, int64_t &workgroups)
{
    PackArgs q{};
    workgroups = 0;
    auto add = [&](int i, Operand &o) {
        if (!o.packed || o.rows == 0 || o.columns == 0) return;
        q.from[i] = o.data;
        q.to[i] = o.packed;
        q.ld[i] = o.ld;
        q.columns[i] = o.columns;
        q.row[i] = (int)ceil_div(o.columns, 8);
        q.chunks[i] = o.rows * q.row[i];
        workgroups += ceil_div(q.chunks[i], WG * PACK_U);
        o.data = o.packed;
        o.ld = 8 * q.row[i];
        o.packed = nullptr;
    };
    add(0, a);
    add(1, b);
    return q;
}

// A product: A and B (null: there is none), and what is done with its sums; parts: room for the parts' ones.
struct Product {
    Operand a, b;
    Size d;
    EpilogueArgs e;
    float *parts;
    bool few;                    // by the kernel of few rows, else
    int kind;                    // by tiles of this kind (a gradient's two products: the same), as planned
    Plan plan;
};

// x W^T by the kernels of type T (out_type: T or 32 bits), and the gradients dz W and dz^T x with what is left to do for the bias (w_type: of the second).
template <typename T>
int product_of(int32_t out_type, const Product &x, hipStream_t st);
template <typename T>
int gradients_of(int32_t w_type, const Product &dx, const Product &dw, const BiasSum &b, hipStream_t st);
#define TT_PRODUCTS(prefix, T)                                             \
    prefix template int tt::product_of<T>(int32_t, const tt::Product &, hipStream_t); \
    prefix template int tt::gradients_of<T>(int32_t, const tt::Product &, const tt::Product &, const tt::BiasSum &, hipStream_t);
TT_PRODUCTS(extern, float)
TT_PRODUCTS(extern, bf16_t)
TT_PRODUCTS(extern, f16_t)

}  // namespace tt
