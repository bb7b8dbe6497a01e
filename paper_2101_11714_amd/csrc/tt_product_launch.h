// Which kernel computes a product, and its launches.  The kernels of each type are compiled in a file of their own (tt_product_*.hip).
#pragma once

#include "tt_product_few.h"
#include "tt_product_stream.h"
#include "tt_rows_args.h"

namespace tt {

// which operands' rows are dense in k: x W^T, dz W, dz^T x
enum Layout { DENSE_DENSE, DENSE_STRIDED, STRIDED_STRIDED };

// How a product is computed.
enum Way { FEW, TILES, TALL_TILES, STREAM, STREAM_WIDE };        // (tiles: 32 bits; streams: 16)

struct Plan {
    Way way;
    int64_t tiles_m, tiles_n;
    int parts;
    int64_t k_part;
};

constexpr int64_t MOST_TILES = 512;                          // workgroups that parts are made for

// Tiles of 256 or of 128, and how many parts of k: whatever should be done first, by what was measured on 256 compute units.  A step of a wide tile,
// one on a compute unit, takes 1.87 us (8,192 x 16,384 x 4,096: 1,127 TFLOP/s); one of a narrow tile 0.70 us alone on its compute unit and 1.17 beside
// another one (2,048 x 2,048 x 4,096, one tile each: 48 us, by wide tiles in four parts 41 and the parts' sums 15; 8,192 x 4,096 x 4,096: 293, by
// wide ones 221).  Parts cost a launch, and their sums a write and a read.
inline void stream_plan(Plan &p, int64_t M, int64_t N, int64_t K)
{
    const int64_t steps = ceil_div(K, PS_K);
    double best = 0;
    for (const bool wide : {true, false}) {
        const int64_t tile = wide ? 256 : 128, tiles_m = ceil_div(M, tile), tiles_n = ceil_div(N, tile), tiles = tiles_m * tiles_n, room = wide ? 256 : MOST_TILES;
        for (int64_t parts = 1; parts == 1 || (parts * tiles <= room && 4 * parts <= steps); parts *= 2) {
            const int64_t each = ceil_div(steps, parts), all = tiles * parts, whole = all / room, rest = all % room;
            double us = wide ? 1.87 * (double)(whole + (rest > 0)) : 1.17 * (double)(whole + (rest > 256)) + (rest > 0 && rest <= 256 ? 0.70 : 0.0);
            us = us * (double)each + 5.0;
            if (parts > 1) us += 3.0 + (double)parts * (double)M * (double)N * 8.0 / 5.0e6;
            if (best == 0 || us < best) {
                best = us;
                p.way = wide ? STREAM_WIDE : STREAM;
                p.tiles_m = tiles_m;
                p.tiles_n = tiles_n;
                p.k_part = each * PS_K;
            }
        }
    }
    p.parts = K > 0 ? (int)ceil_div(K, p.k_part) : 1;
}

// The same for 32 bits, by tiles of 64 x 64 or of 128 x 64: a step takes 0.60 us of a compute unit or 1.13 (2,048^3 by the one 158, by the other 152 us,
// one or two workgroups alike; 4,096^3 1,128 and 1,075), a launch for the parts' sums 6.  1,001 x 1,283 x 777: 37 us by both, as one part or as three;
// 256 x 1,024 x 1,024: 24 us as 64 workgroups, in four parts 14.
inline void tiles_plan(Plan &p, int64_t M, int64_t N, int64_t K)
{
    const int64_t steps = ceil_div(K, PB_K<float>);
    double best = 0;
    for (const bool tall : {true, false}) {
        const int64_t tiles_m = ceil_div(M, tall ? 128 : 64), tiles_n = ceil_div(N, 64), tiles = tiles_m * tiles_n;
        for (int64_t parts = 1; parts == 1 || (parts * tiles <= 2 * MOST_TILES && 4 * parts <= steps); ++parts) {
            const int64_t each = ceil_div(steps, parts);
            if (parts > 1 && ceil_div(steps, each) < parts) continue;
            double us = (double)ceil_div(tiles * parts, 256) * (double)each * (tall ? 1.13 : 0.60);
            if (parts > 1) us += 6.0 + (double)parts * (double)M * (double)N * 8.0 / 5.0e6;
            if (best == 0 || us < best) {
                best = us;
                p.way = tall ? TALL_TILES : TILES;
                p.tiles_m = tiles_m;
                p.tiles_n = tiles_n;
                p.k_part = each * PB_K<float>;
            }
        }
    }
    p.parts = K > 0 ? (int)ceil_div(K, p.k_part) : 1;
}

inline Plan plan_of(int64_t M, int64_t N, int64_t K, int32_t type, bool dense)
{
    Plan p{};
    p.parts = 1;
    p.k_part = K;
    if (dense && M <= PF_MOST) p.way = FEW;
    else if (type != TT_F32) stream_plan(p, M, N, K);
    else tiles_plan(p, M, N, K);
    return p;
}

// What the parts' sums of a product of M rows, or of fewer, take at most, whatever its way: with more rows there are fewer parts, but no more than
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

// C = A B^T, of M x N with sums over K, by the kernels of type T; out_type: T or 32 bits.
template <typename T>
int product_of(Layout layout, int32_t out_type, const Operand &a, const Operand &b, int64_t M, int64_t N, int64_t K, const EpilogueArgs &e, void *workspace, hipStream_t st);
extern template int product_of<float>(Layout, int32_t, const Operand &, const Operand &, int64_t, int64_t, int64_t, const EpilogueArgs &, void *, hipStream_t);
extern template int product_of<bf16_t>(Layout, int32_t, const Operand &, const Operand &, int64_t, int64_t, int64_t, const EpilogueArgs &, void *, hipStream_t);
extern template int product_of<f16_t>(Layout, int32_t, const Operand &, const Operand &, int64_t, int64_t, int64_t, const EpilogueArgs &, void *, hipStream_t);

template <typename... A>
int product(int32_t type, A... args)
{
    return type == TT_F32 ? product_of<float>(args...) : type == TT_BF16 ? product_of<bf16_t>(args...) : product_of<f16_t>(args...);
}

}  // namespace tt
