// Matrix products on the matrix cores, C[m][n] = sum over k of A(m, k) B(n, k), in 32-bit sums, for operands of 32 or 16 bits whose
// rows are dense in k (x, a weight) or in m or n (the gradients' operands), with an epilogue on the sums.
#pragma once

#include <type_traits>

#include "tt_rows_io.h"

namespace tt {

typedef float mfma_acc_t __attribute__((ext_vector_type(4)));

// ---- what is done with the sums -----------------------------------------------------------------------------------------

enum { ACT_NONE = 0, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU, ACT_COUNT };

constexpr float GELU_TANH_SCALE = 0.7978845608028654f, GELU_TANH_CUBE = 0.044715f;      // sqrt(2 / pi)

// By the device's exponential of 2 and reciprocal, which are off by a unit in the last place: the product z log2(e) is rounded, so that exp(-z) is off by
// |z| 2^-24 of itself and the result by a third of 2^-24 for that (a library's exponential and a true quotient: gradients through an activation,
// 8,192 x 4,096, 52 instead of 38 us).  Where the exponential passes 2^128, below z = -88.7, its reciprocal is 0, and SiLU, which is above -3e-37 there, too.  (1 + tanh(u)) / 2 is this function of 2 u.
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z)); }

// its slope p (1 - p), without the difference (which is off by 2^-24 as such: 35 times that in the other functions' slopes), and p itself
__device__ __forceinline__ float logistic_slope(float z, float &p)
{
    const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + e);
    p = z < 0.f ? e * r : r;
    return e * r * r;
}

// The normal distribution up to z, and exp(-z^2 / 2): for -|z| that is exp(-z^2 / 2) u P(u), u = 1 / (1 + |z| / 4), with a polynomial of degree 9 whose
// largest error relative to u P(u) = exp(z^2 / 2) erfc(|z| / sqrt 2) / 2 is 0.75 times 2^-24 with its coefficients in 32 bits (fitted by least squares that were
// weighted until the errors' peaks were alike).  Computed in 32 bits it is off by up to 3.4 times 2^-24 as such, most of it from the polynomial's sum, and in the
// tail by up to (z^2 + 8) 2^-24 of itself, since the exponential's argument is rounded; no branches, which the library's error function has.
__device__ __forceinline__ float normal_to(float z, float &e)
{
    constexpr float P[10] = {0.0997355655f, 0.0997364372f, 0.0934662372f, 0.0816042423f, 0.0589695089f, 0.0637153611f, -0.0317454860f, 0.0956253558f, -0.0808927864f, 0.0197855458f};
    const float u = __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, fabsf(z), 1.f));
    float p = P[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) p = __builtin_fmaf(p, u, P[i]);
    e = __builtin_amdgcn_exp2f(-0.7213475204444817f * z * z);
    const float q = e * (u * p);
    return z > 0.f ? 1.f - q : q;
}

__device__ __forceinline__ float act_of(float z, int act)
{
    float e;
    switch (act) {
    case ACT_RELU: return z > 0.f || z != z ? z : 0.f;
    case ACT_GELU: return z * normal_to(z, e);
    case ACT_GELU_TANH: return z * logistic(2.f * GELU_TANH_SCALE * (z + GELU_TANH_CUBE * z * z * z));
    case ACT_SILU: return z * logistic(z);
    default: return z;
    }
}

// of several values, the choice made once
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int act)
{
    auto all = [&](auto kind) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = act_of(v[j], decltype(kind)::value);
    };
    switch (act) {
    case ACT_RELU: return all(std::integral_constant<int, ACT_RELU>{});
    case ACT_GELU: return all(std::integral_constant<int, ACT_GELU>{});
    case ACT_GELU_TANH: return all(std::integral_constant<int, ACT_GELU_TANH>{});
    case ACT_SILU: return all(std::integral_constant<int, ACT_SILU>{});
    }
}

// the activation's slope
__device__ __forceinline__ float act_slope(float z, int act)
{
    switch (act) {
    case ACT_RELU: return z > 0.f ? 1.f : z != z ? z : 0.f;
    case ACT_GELU: {
        float e;
        const float p = normal_to(z, e);
        return p + z * e * 0.3989422804014327f;
    }
    case ACT_GELU_TANH: {
        float p;
        const float q = logistic_slope(2.f * GELU_TANH_SCALE * (z + GELU_TANH_CUBE * z * z * z), p);
        return q == 0.f ? p : p + 2.f * GELU_TANH_SCALE * z * q * (1.f + 3.f * GELU_TANH_CUBE * z * z);           // (z z can pass what 32 bits hold)
    }
    case ACT_SILU: {
        float p;
        const float q = logistic_slope(z, p);
        return p + z * q;
    }
    default: return 1.f;
    }
}

// y = act(sum + bias) + add, and the value before the activation.  add may be the output itself.
struct EpilogueArgs {
    const void *bias;            // null: none
    int bias_type;               // TT_F32, ...
    int act;
    const void *add;             // of the output's type; null: none
    void *pre;                   // of the operands' type; null: not kept
    void *out;
    int64_t ld_add, ld_pre, ld_out;
};

__device__ __forceinline__ void load_bias(const EpilogueArgs &e, int64_t n, int have, float (&b)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        b[j] = 0.f;
        if (!e.bias || j >= have) continue;
        b[j] = e.bias_type == TT_F32 ? ((const float *)e.bias)[n + j] : e.bias_type == TT_BF16 ? (float)((const bf16_t *)e.bias)[n + j] : (float)((const f16_t *)e.bias)[n + j];
    }
}

// Eight neighbouring sums of row m from column n on, of which `have` exist (at least one).  T: the operands' type, O: the output's.
template <typename T, typename O>
__device__ __forceinline__ void finish8(const EpilogueArgs &e, int64_t m, int64_t n, int have, const float (&b)[8], float (&v)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += b[j];
    if (e.pre) put8((T *)e.pre + m * e.ld_pre + n, have, v);
    activate(v, e.act);
    if (e.add) {
        const O *p = (const O *)e.add + m * e.ld_add + n;
        if (have >= 8) {
            float r[8];
            widen8(fetch8<true>(p, 8, 8), r);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += r[j];
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < have) v[j] += (float)p[j];
        }
    }
    put8((O *)e.out + m * e.ld_out + n, have, v);
}

// ---- tiles of operands in LDS -------------------------------------------------------------------------------------------
//
// A step takes 128 bytes of k, PB_K<T> values.  A matrix instruction 16 x 16 takes of each operand 16 bytes of k per lane from one
// of 16 rows (8 values of 16 bits: one instruction of k = 32; 4 of 32 bits: four of k = 4 whose k are not neighbours, the same
// ones in both operands), so that 64 bytes are a "half".
//   dense in k:   the tile is [rows][bytes of the step], read by 16 bytes per lane;
//   strided in k: it is [values of the step][rows], as it lies in memory; 16-bit values are read transposed by the LDS (4 rows of k x 16
//                 columns to 16 lanes), 32-bit values one by one.
// In both, 16-byte chunks are permuted along a row by an exclusive or with bits of its number, so that the lanes that read at
// the same time find different banks.
// The second operand is the instruction's first, whose rows go to a lane's four registers in fours: a lane has four neighbouring
// columns of one row of C.

template <typename T>
constexpr int PB_K = 128 / (int)sizeof(T);

constexpr int BLOCK = 16;

template <typename T, bool KDENSE, int ROWS>
struct OperandTile {
    static constexpr int CH = 16 / sizeof(T);                // values of a chunk
    static constexpr int LINE = KDENSE ? 8 : ROWS / CH;      // chunks of a line
    static constexpr int LINES = KDENSE ? ROWS : 8 * CH;
    static constexpr int CHUNKS = LINE * LINES, BYTES = CHUNKS * 16;
    static_assert((LINE & (LINE - 1)) == 0, "a permutation of the line's chunks");

    // (transposed reads: 32 lanes read four lines each of two groups, eight lines apart)
    static __device__ __forceinline__ int swizzle(int line)
    {
        const int x = KDENSE ? line & 7 : sizeof(T) == 4 ? (line >> 2 & 3) << 2 : (line & 3) << 1 | (line & 8);
        return x & (LINE - 1);
    }
    // byte offset of a chunk
    static __device__ __forceinline__ int at(int line, int chunk) { return (line * LINE + (chunk ^ swizzle(line))) * 16; }

    // this lane's 16 bytes of block b of the wave's rows from `row0` on, half h of the step
    static __device__ __forceinline__ uint4 fragment(const char *lds, int row0, int b, int h, int lane)
    {
        const int r = lane & 15, q = lane >> 4, first = row0 + 16 * b;
        if constexpr (KDENSE) {
            return *reinterpret_cast<const uint4 *>(lds + at(first + r, 4 * h + q));
        } else if constexpr (sizeof(T) == 2) {
            typedef short Four __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) Four *Shared;
            const int col = first + 4 * (r & 3), k = 32 * h + 8 * q + (r >> 2);
            struct { Four lo, hi; } x;
            x.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared)(lds + at(k, col >> 3) + (col & 4) * 2));
            x.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Shared)(lds + at(k + 4, col >> 3) + (col & 4) * 2));
            return __builtin_bit_cast(uint4, x);
        } else {
            const int col = first + r;
            uint4 x;
            uint32_t *w = reinterpret_cast<uint32_t *>(&x);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = *reinterpret_cast<const uint32_t *>(lds + at(16 * h + 4 * q + j, col >> 2) + (col & 3) * 4);
            return x;
        }
    }
};

// acc[i][j] += (16 rows of B, block j) x (16 rows of A, block i): lane l has row l & 15 of A and rows 4 (l >> 4) .. + 3 of the block of B.  32 bits: four
// instructions for a block, each of which has all blocks behind it before the next one needs its sums.
template <typename T, int BM, int BN>
__device__ __forceinline__ void block_products(const uint4 (&b)[BN], const uint4 (&a)[BM], mfma_acc_t (&acc)[BM][BN])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < BM; ++i)
#pragma unroll
                for (int j = 0; j < BN; ++j) {
                    const uint32_t x = c == 0 ? b[j].x : c == 1 ? b[j].y : c == 2 ? b[j].z : b[j].w, y = c == 0 ? a[i].x : c == 1 ? a[i].y : c == 2 ? a[i].z : a[i].w;
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x), __uint_as_float(y), acc[i][j], 0, 0, 0);
                }
    } else {
        typedef T Eight __attribute__((ext_vector_type(8)));
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j) {
                const Eight x = __builtin_bit_cast(Eight, b[j]), y = __builtin_bit_cast(Eight, a[i]);
                if constexpr (__is_same(T, bf16_t)) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, acc[i][j], 0, 0, 0);
                else acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, acc[i][j], 0, 0, 0);
            }
    }
}

// ---- loads that bear any alignment and any edge ---------------------------------------------------------------------------

// 16 bytes from a place of 4-byte alignment or (HALVES: 16-bit values) of 2: there the words around them, of which each has one of the values, are loaded
// and shifted.  (The device loads 16 bytes from any address, but from odd ones at a third of the rate: few rows, 14 x 3,065 x 512, 20 us instead of 10.)
template <typename T, bool HALVES>
struct Chunk {
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
    typedef Words Aligned __attribute__((aligned(4)));
    Words w;
    uint32_t next, shift;        // HALVES: the word behind them, 16 at odd places

    __device__ __forceinline__ void load(const T *p)
    {
        if (HALVES) {
            const uintptr_t at = (uintptr_t)p;
            const char *from = (const char *)(at & ~(uintptr_t)3);
            shift = (uint32_t)(at & 2) * 8;
            w = *reinterpret_cast<const Aligned *>(from);
            next = *reinterpret_cast<const uint32_t *>(from + 12 + (at & 2) * 2);
        } else {
            w = *reinterpret_cast<const Aligned *>(p);
        }
    }
    __device__ __forceinline__ uint4 get() const
    {
        if (!HALVES) return {w.x, w.y, w.z, w.w};
        return {__builtin_amdgcn_alignbit(w.y, w.x, shift), __builtin_amdgcn_alignbit(w.z, w.y, shift), __builtin_amdgcn_alignbit(w.w, w.z, shift), __builtin_amdgcn_alignbit(next, w.w, shift)};
    }

    // From value c on of a line of N values (one at least): the line's last 16 bytes where fewer are left; lines of less than 16 bytes value by value.
    __device__ __forceinline__ void load(const T *line, int64_t c, int64_t N)
    {
        constexpr int CH = 16 / sizeof(T);
        if (N >= CH) return load(line + (c < N - CH ? c : N - CH));
        struct { T v[CH]; } x;
#pragma unroll
        for (int j = 0; j < CH; ++j) x.v[j] = line[j < N ? j : N - 1];
        w = __builtin_bit_cast(Words, x);
        next = shift = 0;
    }
    // what load() brought, moved into place, with zeros behind the line's end
    __device__ __forceinline__ uint4 get(int64_t c, int64_t N) const { return settled(get(), c, N); }

    static __device__ __forceinline__ uint4 settled(uint4 w, int64_t c, int64_t N)
    {
        constexpr int CH = 16 / sizeof(T), PER = 4 / sizeof(T);
        const int n = N - c >= CH ? CH : N > c ? (int)(N - c) : 0;           // values that exist
        const int d = N >= CH ? (CH - n) * (int)sizeof(T) : 0;               // bytes to move down by
        auto pick = [](bool yes, uint32_t x, uint32_t y) { return yes ? x : y; };
        w = {pick(d & 8, w.z, w.x), pick(d & 8, w.w, w.y), pick(d & 8, 0u, w.z), pick(d & 8, 0u, w.w)};
        w = {pick(d & 4, w.y, w.x), pick(d & 4, w.z, w.y), pick(d & 4, w.w, w.z), pick(d & 4, 0u, w.w)};
        if (sizeof(T) == 2)
            w = {pick(d & 2, w.x >> 16 | w.y << 16, w.x), pick(d & 2, w.y >> 16 | w.z << 16, w.y), pick(d & 2, w.z >> 16 | w.w << 16, w.z), pick(d & 2, w.w >> 16, w.w)};
        if (N < CH || n == 0) {
            auto word = [&](uint32_t x, int k) {
                const int left = n - k * PER;                // values of this word
                return left >= PER ? x : left == 1 && PER == 2 ? x & 0xffffu : 0u;
            };
            w = {word(w.x, 0), word(w.y, 1), word(w.z, 2), word(w.w, 3)};
        }
        return w;
    }
};

// Operands of 16 bits whose rows are not whole chunks, copied into rows that are, with zeros behind their ends: two of them in one launch.  (Loaded through
// registers as they lie, with shifts and edges: 4,096 x 4,096 x 4,096 from rows of 4,099 values 223 us; copied and then by chunks 123.)
struct PackArgs {
    const void *from[2];
    void *to[2];
    int64_t ld[2], columns[2], chunks[2];                    // chunks: of the operand (0: none)
    int row[2];                                              // chunks of a row
};
constexpr int PACK_U = 4;

template <typename T>
__device__ __forceinline__ void pack_rows(const PackArgs &p, int64_t id)
{
    const int64_t first_wgs = (p.chunks[0] + 256 * PACK_U - 1) / (256 * PACK_U);
    const int which = id >= first_wgs;
    const int64_t base = (id - (which ? first_wgs : 0)) * 256 * PACK_U, left = p.chunks[which] - base;
    if (left <= 0) return;
    const int64_t row0 = base / p.row[which], columns = p.columns[which];
    const uint32_t per = (uint32_t)p.row[which], rest = (uint32_t)(base - row0 * per) + threadIdx.x;
    Chunk<T, true> x[PACK_U];
    int64_t c[PACK_U];
#pragma unroll
    for (int u = 0; u < PACK_U; ++u) {
        const uint32_t at = rest + ((int64_t)threadIdx.x + u * 256 < left ? u * 256 : 0), row = at / per;
        c[u] = 8 * (int64_t)(at - row * per);
        if ((int64_t)threadIdx.x < left) x[u].load((const T *)p.from[which] + (row0 + row) * p.ld[which], c[u], columns);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < PACK_U; ++u)
        if ((int64_t)threadIdx.x + u * 256 < left) reinterpret_cast<uint4 *>(p.to[which])[base + threadIdx.x + u * 256] = x[u].get(c[u], columns);
}

template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackArgs p)
{
    pack_rows<T>(p, workgroup());
}

struct ProductArgs {
    const void *a, *b;
    int64_t lda, ldb;            // between rows of a tile that is dense in k, between values of k otherwise
    int64_t M, N, K;
    int tiles_m, tiles_n, parts;
    int64_t k_part;              // values of k of one part (a multiple of the step's)
    float *part;                 // sums of parts, [parts][M][ld_part]; null: one part, whose sums go through the epilogue
    int64_t ld_part;
};

// tile number -> place: eight rows of tiles at a time, so that the tiles that run together share operands
__device__ __forceinline__ void tile_place(int tile, int tiles_m, int tiles_n, int &tm, int &tn)
{
    constexpr int BAND = 8;
    const int band = tile / (BAND * tiles_n), rest = tile - band * BAND * tiles_n, rows = min(BAND, tiles_m - band * BAND);
    tn = rest / rows;
    tm = band * BAND + rest - tn * rows;
}

// A workgroup's tile and part of k: the workgroups of one XCD, which have every eighth number, take neighbouring tiles of one part, whose operands its L2
// then holds.
__device__ __forceinline__ void tile_of(int id, const ProductArgs &p, int &tm, int &tn, int &part)
{
    const int tiles = p.tiles_m * p.tiles_n, all = tiles * p.parts, each = all / 8, more = all % 8, xcd = id % 8, nth = id / 8;
    const int at = xcd * each + min(xcd, more) + nth;
    part = at / tiles;
    tile_place(at - part * tiles, p.tiles_m, p.tiles_n, tm, tn);
}

// A wave's sums on their way out, 16 * BM rows of 64: SOME blocks of 16 rows at a time through LDS of the wave's own (4 KB a block), from where a
// lane takes eight neighbouring columns, eight lanes a row's 64, through the epilogue, or as they are where they are a part's.  What is added to them
// is loaded for U rows together, before they are read: row by row a gradient that is added to one of 32 bits (2,637 x 163 from 320 rows) took 27 us instead of 14.
// FULL: with bias, activation and the value before it; else only what is added.
constexpr int LEAVE_BLOCK = BLOCK * 64 * 4;

template <typename T, typename O, int BM, int SOME, bool FULL>
__device__ __forceinline__ void leave_tile(const ProductArgs &p, const EpilogueArgs &e, int part, int64_t m0, int64_t n0, int lane, char *lds, mfma_acc_t (&acc)[BM][4])
{
    constexpr int U = SOME == 1 || (FULL && BM > 4) ? 2 : 4;
    const int c = lane & 7;
    const int64_t n = n0 + 8 * c;
    const int have = p.N - n < 8 ? (int)(p.N - n) : 8;
    float bias[8] = {};
    if (FULL && !p.part) load_bias(e, n, have, bias);
#pragma unroll
    for (int i0 = 0; i0 < BM; i0 += SOME) {
#pragma unroll
        for (int i = 0; i < SOME; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = lane & 15, chunk = (4 * j + (lane >> 4)) ^ row;
                *reinterpret_cast<mfma_acc_t *>(lds + i * LEAVE_BLOCK + row * 256 + chunk * 16) = acc[i0 + i][j];
            }
        if (have <= 0) continue;
#pragma unroll 1
        for (int r0 = lane >> 3; r0 < 16 * SOME; r0 += 8 * U) {
            const int64_t m1 = m0 + 16 * i0 + r0;
            if (m1 >= p.M) break;
            Vec8<O> add[U];
            if (!p.part && e.add && have == 8)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t m = m1 + 8 * u < p.M ? m1 + 8 * u : m1;
                    add[u] = fetch8<true>((const O *)e.add + m * e.ld_add + n, 8, 8);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = r0 + 8 * u, row = r & 15;
                const int64_t m = m1 + 8 * u;
                if (m >= p.M) break;
                float v[8];
                *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(lds + r * 256 + ((2 * c) ^ row) * 16);
                *reinterpret_cast<float4 *>(v + 4) = *reinterpret_cast<const float4 *>(lds + r * 256 + ((2 * c + 1) ^ row) * 16);
                if (p.part) {
                    put8<true>(p.part + ((int64_t)part * p.M + m) * p.ld_part + n, 8, v);
                } else if (have < 8) {
                    finish8<T, O>(e, m, n, have, bias, v);
                } else {
                    if (FULL) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += bias[j];
                        if (e.pre) put8<true>((T *)e.pre + m * e.ld_pre + n, 8, v);
                        activate(v, e.act);
                    }
                    if (e.add) {
                        float x[8];
                        widen8(add[u], x);
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += x[j];
                    }
                    put8<true>((O *)e.out + m * e.ld_out + n, 8, v);
                }
            }
        }
    }
}

// The parts' sums added in their order, and the epilogue: eight columns, the at-th of them.
template <typename T, typename O>
__device__ __forceinline__ void join_parts(const ProductArgs &p, const EpilogueArgs &e, int64_t at)
{
    const int64_t nv = p.ld_part / 8, m = at / nv, n = 8 * (at - m * nv);
    if (m >= p.M) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias[8];
    const int have = p.N - n < 8 ? (int)(p.N - n) : 8;
    load_bias(e, n, have, bias);
    constexpr int U = 8;                                     // parts whose loads are on their way together
    for (int s0 = 0; s0 < p.parts; s0 += U) {
        Vec8<float> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = fetch8<true>(p.part + ((int64_t)(s0 + u < p.parts ? s0 + u : s0) * p.M + m) * p.ld_part + n, 8, 8);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float y[8];
            widen8(x[u], y);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += s0 + u < p.parts ? y[j] : 0.f;
        }
    }
    finish8<T, O>(e, m, n, have, bias, v);
}

template <typename T, typename O>
__global__ __launch_bounds__(256) void join_parts_kernel(ProductArgs p, EpilogueArgs e)
{
    join_parts<T, O>(p, e, workgroup() * 256 + threadIdx.x);
}

// What a thread loads of an operand's tile of 32-bit values through registers: PIECES chunks of 16 bytes.
// MIDDLE: all values of the step exist, from any address.  Else value by value, of lines that end the last one again, and with zeros for k behind the end.
// Rows of a tile behind the operand's last one give sums that nobody stores: the last one, or in the middle what follows a line (its next one), stands for them.
template <typename T, bool KDENSE, int ROWS, int THREADS>
struct Staged {
    static_assert(sizeof(T) == 4, "");
    typedef OperandTile<T, KDENSE, ROWS> Tile;
    static constexpr int PIECES = Tile::CHUNKS / THREADS, CH = Tile::CH;
    static_assert(Tile::CHUNKS % THREADS == 0, "every thread has as many");
    typedef uint32_t Set __attribute__((ext_vector_type(4)));            // (PIECES of them: a step's values on their way)
    typedef Set Aligned __attribute__((aligned(4)));
    const uint32_t *line[PIECES];                            // where the thread's chunks begin at k = 0
    int64_t ld, rows, row0;
    int64_t safe;                // values of k up to which a chunk may pass its line's end

    static __device__ __forceinline__ int line_of(int i) { return (i * THREADS + threadIdx.x) / Tile::LINE; }
    static __device__ __forceinline__ int chunk_of(int i) { return (i * THREADS + threadIdx.x) % Tile::LINE; }
    __device__ __forceinline__ int64_t column(int i) const { const int64_t c = row0 + chunk_of(i) * CH; return c < rows ? c : rows - 1; }
    __device__ __forceinline__ Staged(const void *data, int64_t stride, int64_t first, int64_t n, int64_t lines)
        : ld(stride), rows(n), row0(first), safe(KDENSE || first + ROWS <= n ? lines : stride > 0 ? lines - CH : 0)
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int64_t row = first + line_of(i);
            if (KDENSE) line[i] = (const uint32_t *)data + (row < n ? row : n - 1) * ld + chunk_of(i) * CH;
            else line[i] = (const uint32_t *)data + line_of(i) * ld + column(i);
        }
    }
    // the step's values from k on, of which those below `end` exist
    template <bool MIDDLE>
    __device__ __forceinline__ void fetch(Set (&set)[PIECES], int64_t k, int64_t end) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (MIDDLE) {
                set[i] = *reinterpret_cast<const Aligned *>(line[i] + (KDENSE ? k : k * ld));
                continue;
            }
            const int64_t c = column(i), l = k + line_of(i);
            const uint32_t *p = KDENSE ? line[i] - chunk_of(i) * CH : line[i] - c + ((l < end ? l : end - 1) - line_of(i)) * ld;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int64_t at = KDENSE ? k + chunk_of(i) * CH + j : c + j, last = KDENSE ? end - 1 : rows - 1;
                set[i][j] = p[at < last ? at : last];
            }
        }
    }
    // (k, end: as they were fetched)
    template <bool MIDDLE>
    __device__ __forceinline__ void put(const Set (&set)[PIECES], char *lds, int64_t k, int64_t end) const
    {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            Set x = set[i];
            if (!MIDDLE)
#pragma unroll
                for (int j = 0; j < CH; ++j) x[j] = k + (KDENSE ? chunk_of(i) * CH + j : line_of(i)) < end ? x[j] : 0u;
            *reinterpret_cast<Set *>(lds + Tile::at(line_of(i), chunk_of(i))) = x;
        }
    }
};

// A tile of TM x 64 per workgroup of four waves below each other (32 x 64: of two times two, of which two take each half of a step), operands through registers into LDS, so that every alignment and edge is right.  Three
// steps' tiles of each operand in LDS: what a half of a step multiplies has been read from LDS in the half before, over the step's end, too; the step after
// the next one is written, from what two steps ago was asked for.  (Two steps' tiles, read when they are multiplied, one step ahead: 256 x 1,024 x 1,024
// 16.5 instead of 14.4 us, a step alone on its compute unit 0.98 instead of 0.60.)
template <int TM>
struct TileShape {
    static constexpr int THREADS = 256, EACH = TM > 64 ? 2 : TM > 32 ? 3 : 4, STAGE = (TM + 64) * 128, LDS = 3 * STAGE;            // EACH: waves of a SIMD
};

template <typename T, typename O, bool AK, bool BK, int TM>
__device__ __forceinline__ void product_tile(const ProductArgs &p, const EpilogueArgs &e, int id, char *lds)
{
    constexpr int TN = 64, KB = PB_K<T>, KS = TM == 32 ? 2 : 1, BM = TM * KS / 4 / BLOCK, BN = TN / BLOCK, SOME = BM;
    typedef Staged<T, AK, TM, 256> SA;
    typedef Staged<T, BK, TN, 256> SB;
    constexpr int STAGE = TileShape<TM>::STAGE;
    static_assert(STAGE == SA::Tile::BYTES + SB::Tile::BYTES && 4 * SOME * LEAVE_BLOCK <= 3 * STAGE, "room for the tiles and for the sums");
    int tm, tn, part;
    tile_of(id, p, tm, tn, part);
    const int64_t m0 = (int64_t)tm * TM, n0 = (int64_t)tn * TN, k0 = part * p.k_part;
    const int64_t k_end = k0 + p.k_part < p.K ? k0 + p.k_part : p.K;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = KS == 2 ? wave >> 1 : 0, wm = (KS == 2 ? wave & 1 : wave) * (BM * BLOCK);
    const SA a(p.a, p.lda, m0, p.M, p.K);
    const SB b(p.b, p.ldb, n0, p.N, p.K);

    mfma_acc_t acc[BM][BN];
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j) acc[i][j] = mfma_acc_t{0.f, 0.f, 0.f, 0.f};
    const int64_t safe = a.safe < b.safe ? a.safe : b.safe, inside = k_end < safe ? k_end : safe;
    typename SA::Set sa[2][SA::PIECES];
    typename SB::Set sb[2][SB::PIECES];
    auto fetch = [&](auto middle, int set, int64_t k) {
        if (decltype(middle)::value || k + KB <= inside) {
            a.template fetch<true>(sa[set], k, k_end);
            b.template fetch<true>(sb[set], k, k_end);
        } else if (k < k_end) {
            a.template fetch<false>(sa[set], k, k_end);
            b.template fetch<false>(sb[set], k, k_end);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto put = [&](auto middle, int set, int stage, int64_t k) {
        if (!decltype(middle)::value && k >= k_end) return;
        a.template put<decltype(middle)::value>(sa[set], lds + stage * STAGE, k, k_end);
        b.template put<decltype(middle)::value>(sb[set], lds + stage * STAGE + SA::Tile::BYTES, k, k_end);
    };
    uint4 fa[2][BM], fb[2][BN];
    auto read = [&](int stage, int h, int to) {
        const char *now = lds + stage * STAGE;
#pragma unroll
        for (int i = 0; i < BM; ++i) fa[to][i] = SA::Tile::fragment(now, wm, i, h, lane);
#pragma unroll
        for (int j = 0; j < BN; ++j) fb[to][j] = SB::Tile::fragment(now + SA::Tile::BYTES, 0, j, h, lane);
    };
    auto first = [&](auto middle) {
        fetch(middle, 0, k0);
        fetch(middle, 1, k0 + KB);
        put(middle, 0, 0, k0);
        fetch(middle, 0, k0 + 2 * KB);
        put(middle, 1, 1, k0 + KB);
        fetch(middle, 1, k0 + 3 * KB);
    };
    int stage = 0;
    auto after = [](int s, int n) { return s + n >= 3 ? s + n - 3 : s + n; };
    auto step = [&](auto middle, int set, int64_t k) {
        if (KS == 1) read(stage, 1, 1);
        put(middle, set, after(stage, 2), k + 2 * KB);
        fetch(middle, set, k + 4 * KB);
        stage = after(stage, 1);
        if (KS == 2) read(stage, half, set ^ 1);
        block_products<T>(fb[KS == 1 ? 0 : set], fa[KS == 1 ? 0 : set], acc);
        if (KS == 1) {
            read(stage, 0, 0);
            block_products<T>(fb[1], fa[1], acc);
        }
        __syncthreads();
    };
    int64_t k = k0;
    if (k0 + 4 * KB <= inside) first(std::true_type{});
    else first(std::false_type{});
    __syncthreads();
    read(0, half, 0);
    for (; k + 6 * KB <= inside; k += 2 * KB) {
        step(std::true_type{}, 0, k);
        step(std::true_type{}, 1, k + KB);
    }
    for (; k < k_end; k += 2 * KB) {
        step(std::false_type{}, 0, k);
        if (k + KB < k_end) step(std::false_type{}, 1, k + KB);
    }
    if (KS == 2) {                                           // the second half's sums to the waves that have the first's
        mfma_acc_t *other = reinterpret_cast<mfma_acc_t *>(lds + (wave & 1) * LEAVE_BLOCK) + lane;
        if (half)
#pragma unroll
            for (int j = 0; j < BN; ++j) other[64 * j] = acc[0][j];
        __syncthreads();
        if (half) return;
#pragma unroll
        for (int j = 0; j < BN; ++j) acc[0][j] += other[64 * j];
    }
    leave_tile<T, O, BM, SOME, AK && BK>(p, e, part, m0 + wm, n0, lane, lds + wave * SOME * LEAVE_BLOCK, acc);
}

template <typename T, typename O, int TM>
__global__ __launch_bounds__(256, TileShape<TM>::EACH) void product_kernel(ProductArgs p, EpilogueArgs e)
{
    __shared__ __attribute__((aligned(16))) char lds[TileShape<TM>::LDS];
    if (workgroup() < (int64_t)p.tiles_m * p.tiles_n * p.parts) product_tile<T, O, true, true, TM>(p, e, (int)workgroup(), lds);
}

// The gradients' products, dx = dz w and dw = dz^T x, in one launch, so that the one with longer sums goes first and the other one fills up behind it.
// (Both by turns, eight workgroups each: 8,192 x 4,096 x 4,096 559 instead of 451 us, since an L2 then holds neither's operands.)
struct PairArgs {
    ProductArgs p[2];
    EpilogueArgs e[2];
    int first;                   // of the two, which has the first workgroups
    int64_t wgs[2];              // of which it has so many
};

// which of the two, and its how manieth workgroup
__device__ __forceinline__ int which_of(const PairArgs &g, int64_t &id)
{
    int which = g.first;
    if (id >= g.wgs[which]) {
        id -= g.wgs[which];
        which ^= 1;
        if (id >= g.wgs[which]) return -1;
    }
    return which;
}

template <typename T, typename W, int TM>
__global__ __launch_bounds__(256, TM > 64 ? 2 : 3) /* (with four the smallest spills: 132 x 7,040 x 256 27 instead of 22 us) */ void pair_kernel(PairArgs g)
{
    __shared__ __attribute__((aligned(16))) char lds[TileShape<TM>::LDS];
    int64_t id = workgroup();
    const int which = which_of(g, id);
    if (which == 0) product_tile<T, T, true, false, TM>(g.p[0], g.e[0], (int)id, lds);
    else if (which == 1) product_tile<T, W, false, false, TM>(g.p[1], g.e[1], (int)id, lds);
}

// What is left to be done behind the pair: parts' sums of either, and the bias's gradient from bands of rows, in their order.
struct BiasSum {
    const float *part;           // null: there is none
    void *db;
    int type, add, bands, N, cols;
};

__device__ __forceinline__ void leave_bias(const BiasSum &b, int at, float y)
{
    if (b.type == TT_F32) ((float *)b.db)[at] = y + (b.add ? ((float *)b.db)[at] : 0.f);
    else if (b.type == TT_BF16) ((bf16_t *)b.db)[at] = (bf16_t)(y + (b.add ? (float)((bf16_t *)b.db)[at] : 0.f));
    else ((f16_t *)b.db)[at] = (f16_t)(y + (b.add ? (float)((f16_t *)b.db)[at] : 0.f));
}

// 32 columns of the bias, every eighth band a thread, or 256 times eight columns of a product
template <typename T, typename W>
__global__ __launch_bounds__(256) void finish_pair_kernel(PairArgs g, BiasSum b, int64_t wgs0, int64_t wgs1)
{
    __shared__ float sums[8][33];
    int64_t id = workgroup();
    if (id < wgs0) return join_parts<T, T>(g.p[0], g.e[0], id * 256 + threadIdx.x);
    if ((id -= wgs0) < wgs1) return join_parts<T, W>(g.p[1], g.e[1], id * 256 + threadIdx.x);
    if (!b.part || (id -= wgs1) >= (b.N + 31) / 32) return;
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5, at = (int)id * 32 + c;
    float s = 0.f;
    if (at < b.N)
#pragma unroll 8
        for (int i = q; i < b.bands; i += 8) s += b.part[(int64_t)i * b.cols + at];
    sums[q][c] = s;
    __syncthreads();
    if (q || at >= b.N) return;
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y += sums[i][c];
    leave_bias(b, at, y);
}

}  // namespace tt
