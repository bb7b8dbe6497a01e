// What the operators on rows of a language model's arrays share: vectors of eight columns in 32- and 16-bit types, and the
// counter-based generator behind dropout.
#pragma once

#include "tt_common.h"

namespace tt {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Eight neighbouring columns of a row, as they lie in memory, as 32-bit words (not as values: the compiler would join stores of single
// values at a row's end with the whole vectors' and split those).  Rows may start on any multiple of the element's size (odd
// dimensions and strides): the device loads and stores 16 bytes from any address.
template <typename T>
struct Vec8 {
    static constexpr int W = 2 * sizeof(T), PER = 4 / sizeof(T);             // words, values of a word
    typedef uint32_t Words __attribute__((ext_vector_type(W)));
    typedef Words Anywhere __attribute__((aligned(sizeof(T))));
    Words w;
};

// The columns of a vector of which n exist (8 or more: all) in rows of N.  No branch stands around a load, since what is loaded under
// a condition is waited for there: where fewer than eight are left the row's last eight are loaded, and settle8 moves the right
// ones into place when they are needed (rows of less than eight columns: one by one, the last one again for those behind it).
// WHOLE: N is a multiple of 8, and all of this away.
template <bool WHOLE = false, typename T>
__device__ __forceinline__ Vec8<T> fetch8(const T *p, int n, int N)
{
    Vec8<T> r;
    if (WHOLE || N >= 8) {
        r.w = *reinterpret_cast<const typename Vec8<T>::Anywhere *>(p - (WHOLE || n >= 8 ? 0 : 8 - n));
    } else {
        struct Values { T v[8]; } x;
#pragma unroll
        for (int j = 0; j < 8; ++j) x.v[j] = p[min(j, n - 1)];
        r.w = __builtin_bit_cast(typename Vec8<T>::Words, x);
    }
    return r;
}

// zeros behind the last column
template <bool WHOLE = false, typename T>
__device__ __forceinline__ void settle8(Vec8<T> &r, int n, int N)
{
    if (WHOLE || n >= 8) return;
    constexpr int W = Vec8<T>::W, PER = Vec8<T>::PER;
    if (N >= 8) {                                            // down by 8 - n places (the same for all rows)
        const int d = 8 - n;
#pragma unroll
        for (int by = 4; by >= 1; by >>= 1) {
            const bool move = d & by;
#pragma unroll
            for (int k = 0; k < W; ++k) {
                uint32_t x;
                if (by >= PER) x = k + by / PER < W ? r.w[k + by / PER < W ? k + by / PER : 0] : 0u;
                else x = r.w[k] >> 16 | (k + 1 < W ? r.w[k + 1 < W ? k + 1 : 0] << 16 : 0u);
                r.w[k] = move ? x : r.w[k];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= n) r.w[j / PER] &= PER == 1 ? 0u : j & 1 ? 0x0000ffffu : 0xffff0000u;
    }
}

template <typename T>
__device__ __forceinline__ Vec8<T> narrow8(const float (&x)[8])
{
    typedef float Two __attribute__((ext_vector_type(2)));
    typedef T Narrow __attribute__((ext_vector_type(2)));
    Vec8<T> r;
#pragma unroll
    for (int k = 0; k < Vec8<T>::W; ++k) {
        if constexpr (sizeof(T) == 4) r.w[k] = __float_as_uint(x[k]);
        else r.w[k] = __builtin_bit_cast(uint32_t, __builtin_convertvector((Two{x[2 * k], x[2 * k + 1]}), Narrow));
    }
    return r;
}

// one rounding, to the nearest even
template <bool WHOLE = false, typename T>
__device__ __forceinline__ void put8(T *p, int n, const float (&x)[8])
{
    const Vec8<T> r = narrow8<T>(x);
    if (WHOLE || n >= 8) {
        *reinterpret_cast<typename Vec8<T>::Anywhere *>(p) = r.w;
    } else {
        struct Values { T v[8]; };
        const Values y = __builtin_bit_cast(Values, r.w);
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) p[j] = y.v[j];
    }
}

// all zeros unless `keep`, before anything is computed from them
template <typename T>
__device__ __forceinline__ void keep8(bool keep, Vec8<T> &r)
{
#pragma unroll
    for (int k = 0; k < Vec8<T>::W; ++k) r.w[k] = keep ? r.w[k] : 0u;
}

template <typename T>
__device__ __forceinline__ void widen8(const Vec8<T> &r, float (&x)[8])
{
    struct Values { T v[8]; };
    const Values y = __builtin_bit_cast(Values, r.w);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (float)y.v[j];
}

// element offset of row r; a row's number and a row stride have 31 bits each
__device__ __forceinline__ int64_t row_at(int64_t r, int64_t ld) { return (int64_t)((uint64_t)(uint32_t)r * (uint64_t)(uint32_t)ld); }

// the number of a workgroup in a grid that may go on along y, which then has 1 << GRID_LG of them along x
constexpr int GRID_LG = 21;
__device__ __forceinline__ int64_t workgroup() { return ((int64_t)blockIdx.y << GRID_LG) + blockIdx.x; }

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

struct DropWords {
    uint32_t w[4];
};

// the words of one block
__device__ __forceinline__ DropWords drop_words(const DropArgs &d, const DropKey &k, uint64_t block)
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
    return {{c0, c1, c2, c3}};
}

// The columns of the words' block that are dropped become 0, whatever they were; the factor of the others is the caller's.
__device__ __forceinline__ void drop8(const DropArgs &d, const DropWords &words, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = (words.w[j] << 16) > d.most ? x[2 * j] : 0.f;
        x[2 * j + 1] = words.w[j] > d.most ? x[2 * j + 1] : 0.f;
    }
}

__device__ __forceinline__ void drop8(const DropArgs &d, const DropKey &k, uint64_t block, float (&x)[8]) { drop8(d, drop_words(d, k, block), x); }

}  // namespace tt
