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

// n: how many of the eight columns exist (8 or more: all)
template <typename T>
__device__ __forceinline__ Vec8<T> fetch8(const T *p, int n)
{
    Vec8<T> r;
    if (n >= 8) {
        r = *reinterpret_cast<const Vec8<T> *>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.v[j] = j < n ? p[j] : (T)0.f;
    }
    return r;
}

// one rounding, to the nearest even
template <typename T>
__device__ __forceinline__ void put8(T *p, int n, const float (&x)[8])
{
    Vec8<T> r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.v[j] = (T)x[j];
    if (n >= 8) {
        *reinterpret_cast<Vec8<T> *>(p) = r;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = r.v[j];
    }
}

template <typename T>
__device__ __forceinline__ void widen8(const Vec8<T> &r, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)r.v[j];
}

// ---- dropout ------------------------------------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten rounds of two
// 32 x 32 -> 64 bit products on a counter of four words, keyed by two.  One block serves eight columns with 16 bits each.
// A column is kept iff its draw is at least q = round(65536 p), and then multiplied by 65536 / (65536 - q): p is rounded to
// a multiple of 2^-16, and for that p the expectation is exact.  32 bits a column would cost twice the products, which run at
// a quarter of the rate and already take as long as the memory traffic of a 16-bit array.

struct DropArgs {
    const int64_t *state;        // device: seed, step; null: no dropout
    uint32_t site, q;
    float factor;
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

// bit j: column 8 * (block within the row) + j is kept
__device__ __forceinline__ uint32_t drop_mask(const DropArgs &d, const DropKey &k, uint64_t block)
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = d.site, c3 = k.step, k0 = k.k0, k1 = k.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m |= ((w[j] & 0xffffu) >= d.q ? 1u : 0u) << (2 * j);
        m |= ((w[j] >> 16) >= d.q ? 1u : 0u) << (2 * j + 1);
    }
    return m;
}

// (chosen, not multiplied: a dropped value is 0 whatever it was)
__device__ __forceinline__ void drop8(const DropArgs &d, uint32_t mask, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (mask >> j) & 1u ? x[j] * d.factor : 0.f;
}

}  // namespace tt
