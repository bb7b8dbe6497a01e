// What the operators on rows of a language model's arrays share: vectors of eight columns in 32- and 16-bit types, and the
// counter-based generator behind dropout.
#pragma once

#include "tt_common.h"

namespace tt {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Eight neighbouring columns of a row, as they lie in memory.  Rows may start on any multiple of the element's size (odd
// dimensions and strides): the type's alignment is the element's, and the device loads and stores 16 bytes from any address.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Vec8 {
    T v[8];
};

// n: how many of the eight columns exist (8 or more: all).  WHOLE: all of them do, whatever n is; the kernels that move the most
// exist for rows of whole vectors and for others, since the test in front of every load keeps loads from being issued together.
template <bool WHOLE = false, typename T>
__device__ __forceinline__ Vec8<T> fetch8(const T *p, int n)
{
    Vec8<T> r;
    if (WHOLE || n >= 8) {
        r = *reinterpret_cast<const Vec8<T> *>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.v[j] = j < n ? p[j] : (T)0.f;
    }
    return r;
}

// one rounding, to the nearest even
template <bool WHOLE = false, typename T>
__device__ __forceinline__ void put8(T *p, int n, const float (&x)[8])
{
    Vec8<T> r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.v[j] = (T)x[j];
    if (WHOLE || n >= 8) {
        *reinterpret_cast<Vec8<T> *>(p) = r;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = r.v[j];
    }
}

// all zeros unless `keep`, before anything is computed from them (a register holds two 16-bit values)
template <typename T>
__device__ __forceinline__ void keep8(bool keep, Vec8<T> &r)
{
    struct Words { uint32_t w[2 * sizeof(T)]; };
    Words x = __builtin_bit_cast(Words, r);
#pragma unroll
    for (unsigned j = 0; j < 2 * sizeof(T); ++j) x.w[j] = keep ? x.w[j] : 0u;
    r = __builtin_bit_cast(Vec8<T>, x);
}

template <typename T>
__device__ __forceinline__ void widen8(const Vec8<T> &r, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)r.v[j];
}

// element offset of row r; a row's number and a row stride have 31 bits each
__device__ __forceinline__ int64_t row_at(int64_t r, int64_t ld) { return (int64_t)((uint64_t)(uint32_t)r * (uint64_t)(uint32_t)ld); }

// ---- sums over lanes ----------------------------------------------------------------------------------------------

template <int CTRL>
__device__ __forceinline__ int lane_move(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, false); }

// f over 1 << lg neighbouring lanes (lg <= 6), in every one of them: partners 1 and 2 lanes away, then the mirror image in 8 and in
// 16 lanes (whose quarters agree by then), then the other 16 and the other 32.  Register moves; an exchange through LDS takes
// several times as long.
template <typename V, typename F>
__device__ __forceinline__ V lanes_reduce(V x, int lg, F f)
{
    auto move = [](auto m, V v) { return __builtin_bit_cast(V, m(__builtin_bit_cast(int, v))); };
    if (lg > 0) x = f(x, move([](int v) { return lane_move<0xB1>(v); }, x));
    if (lg > 1) x = f(x, move([](int v) { return lane_move<0x4E>(v); }, x));
    if (lg > 2) x = f(x, move([](int v) { return lane_move<0x141>(v); }, x));
    if (lg > 3) x = f(x, move([](int v) { return lane_move<0x140>(v); }, x));
    if (lg > 4) {
        const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
        x = f(__builtin_bit_cast(V, (unsigned)p[0]), __builtin_bit_cast(V, (unsigned)p[1]));
    }
    if (lg > 5) {
        const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
        x = f(__builtin_bit_cast(V, (unsigned)p[0]), __builtin_bit_cast(V, (unsigned)p[1]));
    }
    return x;
}

// ---- dropout ------------------------------------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten rounds of two
// 32 x 32 -> 64 bit products on a counter of four words, keyed by two.  One block serves eight columns with 16 bits each.
// A column is kept iff its draw is at least q = round(65536 p), and then multiplied by 65536 / (65536 - q): p is rounded to
// a multiple of 2^-16, and for that p the expectation is exact.  32 bits a column would cost twice the products, which run at
// a quarter of the rate and already take as long as the memory traffic of a 16-bit array.

struct DropArgs {
    const int64_t *state;        // device: seed, step; null: no dropout
    uint32_t site;
    uint32_t most;               // 65536 q - 1: a column is dropped whose draw, as the high half of a word, is at most this
    float factor;                // 1 without dropout
};

struct DropKey {
    uint32_t k0, k1, step;
};

__device__ __forceinline__ DropKey drop_key(const DropArgs &d)
{
    DropKey k{0u, 0u, 0u};
    if (d.state) {
        const uint64_t seed = (uint64_t)d.state[0];
        k.k0 = (uint32_t)seed;
        k.k1 = (uint32_t)(seed >> 32);
        k.step = (uint32_t)d.state[1];
    }
    return k;
}

// The columns of one block that are dropped become 0, whatever they were; the factor of the others is the caller's.
__device__ __forceinline__ void drop8(const DropArgs &d, const DropKey &k, uint64_t block, float (&x)[8])
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = d.site, c3 = k.step, k0 = k.k0, k1 = k.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c1, k0, 0x96);   // (exclusive or of three)
        c1 = (uint32_t)b;
        c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c3, k1, 0x96);
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = (w[j] << 16) > d.most ? x[2 * j] : 0.f;
        x[2 * j + 1] = w[j] > d.most ? x[2 * j + 1] : 0.f;
    }
}

}  // namespace tt
