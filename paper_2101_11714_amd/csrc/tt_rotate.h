// Norm of every head and rotation by position, forward and backward.
//
// A unit is 16 columns of a head: eight pairs that are turned (eight columns of each half, or eight pairs of neighbours), or 16 columns behind
// those.  A head is the 1 << lg neighbouring lanes that have a unit each; a lane keeps its columns in registers from the load to the store, so
// that a head is read once.  Such a group of lanes takes some heads of one row in turn, queries or keys, with the cosines and sines of its pairs and
// its part of the weight in registers: nothing goes through LDS, and nothing waits for other groups.
#pragma once

#include <type_traits>

#include "tt_rows_io.h"

namespace tt {

struct Heads {
    void *data;
    int64_t ld, ld_head;
};

struct RotateArgs {
    Heads q, k;                  // inputs (backward: the inputs of the forward pass)
    Heads gq, gk;                // backward: the outputs' gradients
    Heads oq, ok;                // outputs
    const void *wq, *wk;
    int wq_type, wk_type;
    int q_heads, k_heads;
    const void *positions;
    int64_t ld_positions;
    const float *freqs;
    int positions64, pairs, ends[4], neighbours;
    int64_t rows;
    int D, units, turned;        // units of a head, of which so many are turned
    int lg;                      // lanes of a head
    int each, q_slices, k_slices;// heads that a group takes, and groups for a row's queries and for its keys
    float eps;
    // backward
    int q_workgroups;            // the first ones, which take the queries
    void *gwq, *gwk;             // the weights' gradients, null: not wanted
    int gwq_type, gwk_type, add;
    float *part;                 // [workgroups][D] sums of theirs; null: one workgroup has them all
};

// 1 / (2 pi) as the sum of two numbers of 64 bits.
constexpr double TURN_HI = 0x1.45f306dc9c883p-3, TURN_LO = -0x1.6b01ec5417056p-57;

// cos and sin of the angle position * freq.  A position has up to 53 bits and the angle may be 2^52 radians and more, so that freq / (2 pi) is held as the
// sum of two numbers, and whole turns are taken off in the product, before it is rounded: the fraction of a turn is off by 2^-50.  (A rounded product of
// numbers of 64 bits has lost a tenth of a turn at 2^50 turns.  What this takes hardly shows: rotate_prefill 67.8 instead of 67.5 us,
// rotate_video 27.2 as before.)  From the nearest quarter the fraction is an eighth at most, pi / 4 as an angle, where the Taylor series up to x^9 and x^10 are exact to 3e-9.
__device__ __forceinline__ float2 turn_of(double position, float freq)
{
    const double f = freq, hi = f * TURN_HI, lo = fma(f, TURN_LO, fma(f, TURN_HI, -hi));
    const double t = fma(position, lo, fma(position, hi, -rint(position * hi)));
    const double q = rint(4.0 * t);
    const float x = (float)((t - 0.25 * q) * 6.283185307179586), z = x * x;
    const float s = x * (1.f + z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880)))));
    const float c = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
    const int quarter = (int)q & 3;
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    return make_float2(quarter == 1 || quarter == 2 ? -a : a, quarter >= 2 ? -b : b);
}

// Where a unit's two vectors of eight begin, and how many columns of each there are.
struct Unit {
    int at[2], n[2];
};

__device__ __forceinline__ Unit unit_of(const RotateArgs &a, int u)
{
    Unit r;
    if (u < a.turned) {
        if (a.neighbours) {
            r.at[0] = 16 * u;
            r.at[1] = 16 * u + 8;
            r.n[0] = 2 * a.pairs - r.at[0];
            r.n[1] = 2 * a.pairs - r.at[1];
        } else {
            r.at[0] = 8 * u;
            r.at[1] = a.pairs + 8 * u;
            r.n[0] = r.n[1] = a.pairs - 8 * u;
        }
    } else {
        r.at[0] = 2 * a.pairs + 16 * (u - a.turned);
        r.at[1] = r.at[0] + 8;
        r.n[0] = a.D - r.at[0];
        r.n[1] = a.D - r.at[1];
    }
    if (r.n[0] <= 0) r.at[0] = 0;
    if (r.n[1] <= 0) r.at[1] = 0;
    return r;
}

// the lane's cosines and sines in row `row`
__device__ __forceinline__ void turns_of(const RotateArgs &a, int64_t row, int u, float2 (&t)[8])
{
    double pos[4];
    for (int x = 0; x < 4; ++x) pos[x] = 0.0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        if (x && a.ends[x] == a.ends[x - 1]) continue;       // (no pair: an axis that may not be there)
        const int64_t at = x * a.ld_positions + row;
        pos[x] = a.positions64 ? (double)((const int64_t *)a.positions)[at] : (double)((const int32_t *)a.positions)[at];
    }
    float freq[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) freq[j] = a.freqs[min(8 * u + j, a.pairs - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int p = min(8 * u + j, a.pairs - 1);
        const double at = p < a.ends[0] ? pos[0] : p < a.ends[1] ? pos[1] : p < a.ends[2] ? pos[2] : pos[3];
        t[j] = turn_of(at, freq[j]);
        if (j & 1) __builtin_amdgcn_sched_barrier(0);        // (eight at once would take the registers that heads are on their way to)
    }
}

// Eight columns of a head from column `at` on.  WHOLE: a unit's vectors have eight columns or none (which load the head's first).
template <typename T, bool WHOLE>
__device__ __forceinline__ Vec8<T> fetch_unit(const T *head, int at, int D) { return fetch8<WHOLE>(head + at, D - at, D); }

// the first n of them, and zeros behind
template <bool WHOLE, typename T>
__device__ __forceinline__ void widen_unit(Vec8<T> r, int at, int n, int D, float (&x)[8])
{
    settle8<WHOLE>(r, D - at, D);
    widen8(r, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (WHOLE ? n > 0 : j < n) ? x[j] : 0.f;
}

template <bool WHOLE, typename T>
__device__ __forceinline__ void store_unit(T *head, int at, int n, const float (&x)[8])
{
    if (n > 0) put8<WHOLE>(head + at, n, x);
}

// the lane's part of a weight (null: ones)
template <bool WHOLE>
__device__ __forceinline__ void load_weight(const void *w, int type, const Unit &u, int D, float (&x)[2][8])
{
    auto load = [&](auto *p) {
        typedef std::remove_cv_t<std::remove_pointer_t<decltype(p)>> W;
        const Vec8<W> r0 = fetch_unit<W, WHOLE>(p, u.at[0], D), r1 = fetch_unit<W, WHOLE>(p, u.at[1], D);
        widen_unit<WHOLE>(r0, u.at[0], u.n[0], D, x[0]);
        widen_unit<WHOLE>(r1, u.at[1], u.n[1], D, x[1]);
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) x[0][j] = x[1][j] = 1.f;
    if (!w) return;
    if (type == TT_F32) load((const float *)w);
    else if (type == TT_BF16) load((const bf16_t *)w);
    else load((const f16_t *)w);
}

// the unit's pairs turned; BACK: the other way round
template <bool BACK, bool NEIGHBOURS>
__device__ __forceinline__ void turn_unit(const float2 (&t)[8], float (&x)[2][8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float &p = NEIGHBOURS ? x[j >> 2][2 * j & 7] : x[0][j], &q = NEIGHBOURS ? x[j >> 2][(2 * j & 7) + 1] : x[1][j];
        const float v = p, w = q, s = BACK ? -t[j].y : t[j].y;
        p = v * t[j].x - w * s;
        q = w * t[j].x + v * s;
    }
}

template <typename T>
__device__ __forceinline__ T *head_at(const Heads &h, int64_t row, int head) { return (T *)h.data + row * h.ld + head * h.ld_head; }

// a weight's gradient, null: not wanted
__device__ __forceinline__ void put_weight(void *w, int type, int at, float y, int add)
{
    if (!w) return;
    if (type == TT_F32) ((float *)w)[at] = y + (add ? ((float *)w)[at] : 0.f);
    else if (type == TT_BF16) ((bf16_t *)w)[at] = (bf16_t)(y + (add ? (float)((bf16_t *)w)[at] : 0.f));
    else ((f16_t *)w)[at] = (f16_t)(y + (add ? (float)((f16_t *)w)[at] : 0.f));
}

// A group's place: its row and the heads [from, to) of queries or keys.
struct Slice {
    int64_t row;
    int from, to;
};

__device__ __forceinline__ Slice slice_of(int64_t item, int slices, int each, int heads)
{
    Slice s;
    s.row = item / slices;
    s.from = (int)(item - s.row * slices) * each;
    s.to = min(s.from + each, heads);
    return s;
}

template <typename T, bool NORM, bool WHOLE, bool NEIGHBOURS>
__global__ __launch_bounds__(WG) void rotate_kernel(RotateArgs a)
{
    constexpr int U = sizeof(T) == 4 || !WHOLE ? 2 : 4;      // heads whose loads are on their way together
    const int g = 1 << a.lg, u = threadIdx.x & (g - 1), slices = a.q_slices + a.k_slices;
    const int64_t item = workgroup() * (WG >> a.lg) + (threadIdx.x >> a.lg);
    if (item >= a.rows * slices) return;                     // (whole groups)
    const bool in = u < a.units;
    Unit unit = unit_of(a, in ? u : 0);
    if (!in) unit.n[0] = unit.n[1] = 0;
    Slice s = slice_of(item, slices, a.each, 1 << 30);
    const bool key = s.from >= a.q_slices * a.each;
    if (key) s.from -= a.q_slices * a.each;
    s.to = min(s.from + a.each, key ? a.k_heads : a.q_heads);
    const Heads src = key ? a.k : a.q, dst = key ? a.ok : a.oq;
    float w[2][8];
    float2 turns[8];
    Vec8<T> raw[U][2];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const T *p = head_at<T>(src, s.row, min(h0 + i, s.to - 1));
            raw[i][0] = fetch_unit<T, WHOLE>(p, unit.at[0], a.D);
            raw[i][1] = fetch_unit<T, WHOLE>(p, unit.at[1], a.D);
        }
    };
    fetch(s.from);
    if (NORM) load_weight<WHOLE>(key ? a.wk : a.wq, key ? a.wk_type : a.wq_type, unit, a.D, w);
    const bool turned = u < a.turned;
    if (turned) turns_of(a, s.row, u, turns);
    for (int h0 = s.from; h0 < s.to; h0 += U) {
        if (h0 > s.from) fetch(h0);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (h0 + i >= s.to) break;
            float x[2][8];
            widen_unit<WHOLE>(raw[i][0], unit.at[0], unit.n[0], a.D, x[0]);
            widen_unit<WHOLE>(raw[i][1], unit.at[1], unit.n[1], a.D, x[1]);
            if (NORM) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += x[0][j] * x[0][j] + x[1][j] * x[1][j];
                sum = lanes_reduce(sum, a.lg, [](float p, float q) { return p + q; });
                const float rho = 1.f / sqrtf(sum / (float)a.D + a.eps);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[c][j] *= rho * w[c][j];
            }
            if (turned) turn_unit<false, NEIGHBOURS>(turns, x);
            T *p = head_at<T>(dst, s.row, h0 + i);
            store_unit<WHOLE>(p, unit.at[0], unit.n[0], x[0]);
            store_unit<WHOLE>(p, unit.at[1], unit.n[1], x[1]);
        }
    }
}

// Queries and keys have workgroups of their own, each of which has the sums of one weight in its registers.
template <typename T, bool NORM, bool WHOLE, bool NEIGHBOURS>
__global__ __launch_bounds__(WG, NORM ? 2 : WHOLE ? 4 : 3) void rotate_bwd_kernel(RotateArgs a)
{
    extern __shared__ float sums[];
    const int g = 1 << a.lg, u = threadIdx.x & (g - 1), groups = WG >> a.lg;
    const bool in = u < a.units, turned = u < a.turned;
    Unit unit = unit_of(a, in ? u : 0);
    if (!in) unit.n[0] = unit.n[1] = 0;
    const bool which = (int)blockIdx.x >= a.q_workgroups;
    const int first = which ? blockIdx.x - a.q_workgroups : blockIdx.x, workgroups = which ? gridDim.x - a.q_workgroups : a.q_workgroups;
    const int slices = which ? a.k_slices : a.q_slices, heads = which ? a.k_heads : a.q_heads;
    const Heads src = which ? a.k : a.q, grad = which ? a.gk : a.gq, dst = which ? a.ok : a.oq;
    float w[2][8], dw[2][8] = {};
    if (NORM) load_weight<WHOLE>(which ? a.wk : a.wq, which ? a.wk_type : a.wq_type, unit, a.D, w);
    for (int64_t item = (int64_t)first * groups + (threadIdx.x >> a.lg); item < a.rows * slices; item += (int64_t)workgroups * groups) {
        const Slice s = slice_of(item, slices, a.each, heads);
        float2 turns[8];
        Vec8<T> rd[2], rx[2], nd[2], nx[2];
        auto fetch = [&](int h) {
            const T *p = head_at<T>(grad, s.row, h);
            nd[0] = fetch_unit<T, WHOLE>(p, unit.at[0], a.D);
            nd[1] = fetch_unit<T, WHOLE>(p, unit.at[1], a.D);
            if (NORM) {
                const T *x = head_at<T>(src, s.row, h);
                nx[0] = fetch_unit<T, WHOLE>(x, unit.at[0], a.D);
                nx[1] = fetch_unit<T, WHOLE>(x, unit.at[1], a.D);
            }
        };
        fetch(s.from);
        if (turned) turns_of(a, s.row, u, turns);
#pragma unroll 1
        for (int h = s.from; h < s.to; ++h) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                rd[c] = nd[c];
                if (NORM) rx[c] = nx[c];
            }
            fetch(min(h + 1, s.to - 1));                 // the next head, while this one is worked on
            float d[2][8];
            widen_unit<WHOLE>(rd[0], unit.at[0], unit.n[0], a.D, d[0]);
            widen_unit<WHOLE>(rd[1], unit.at[1], unit.n[1], a.D, d[1]);
            if (turned) turn_unit<true, NEIGHBOURS>(turns, d);
            if (NORM) {
                float x[2][8], sum = 0.f, dot = 0.f;
                widen_unit<WHOLE>(rx[0], unit.at[0], unit.n[0], a.D, x[0]);
                widen_unit<WHOLE>(rx[1], unit.at[1], unit.n[1], a.D, x[1]);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        sum += x[c][j] * x[c][j];
                        dot += d[c][j] * w[c][j] * x[c][j];
                    }
                sum = lanes_reduce(sum, a.lg, [](float p, float q) { return p + q; });
                dot = lanes_reduce(dot, a.lg, [](float p, float q) { return p + q; });
                const float rho = 1.f / sqrtf(sum / (float)a.D + a.eps), along = rho * rho * dot / (float)a.D;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        dw[c][j] += d[c][j] * x[c][j] * rho;
                        d[c][j] = rho * (d[c][j] * w[c][j] - x[c][j] * along);
                    }
            }
            T *p = head_at<T>(dst, s.row, h);
            store_unit<WHOLE>(p, unit.at[0], unit.n[0], d[0]);
            store_unit<WHOLE>(p, unit.at[1], unit.n[1], d[1]);
        }
    }
    if (!NORM || !(which ? a.gwk : a.gwq)) return;
    // the groups' sums: lanes of a wave, then waves through LDS, in their order
    const int cols = 16 * a.units, lanes = g < WAVE ? g : WAVE;
    for (int b = a.lg; b < 6; ++b)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) dw[c][j] += __shfl_xor(dw[c][j], 1 << b);
    __syncthreads();
    if ((int)(threadIdx.x & 63) < lanes && in)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[(threadIdx.x >> 6) * cols + 16 * u + 8 * c + j] = dw[c][j];
    __syncthreads();
    for (int i = threadIdx.x; i < cols; i += WG) {
        const Unit x = unit_of(a, i >> 4);
        const int c = i >> 3 & 1, j = i & 7, at = (c ? x.at[1] : x.at[0]) + j;
        if (j >= (c ? x.n[1] : x.n[0])) continue;
        const float y = (sums[i] + sums[cols + i]) + (sums[2 * cols + i] + sums[3 * cols + i]);
        if (a.part) a.part[(int64_t)blockIdx.x * a.D + at] = y;
        else put_weight(which ? a.gwk : a.gwq, which ? a.gwk_type : a.gwq_type, at, y, a.add);
    }
}

// the workgroups' sums added in their order, 32 columns a workgroup: blockIdx.y 0 the queries' weight, 1 the keys'
__global__ __launch_bounds__(1024) void rotate_weight_kernel(RotateArgs a, int workgroups)
{
    __shared__ float sums[32][33];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5, at = blockIdx.x * 32 + c;
    const bool which = blockIdx.y;
    const int first = which ? a.q_workgroups : 0, last = which ? workgroups : a.q_workgroups;
    float s = 0.f;
    if (at < a.D)
#pragma unroll 4
        for (int b = first + q; b < last; b += 32) s += a.part[(int64_t)b * a.D + at];
    sums[q][c] = s;
    __syncthreads();
    if (q || at >= a.D) return;
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) y += sums[i][c];
    put_weight(which ? a.gwk : a.gwq, which ? a.gwk_type : a.gwq_type, at, y, a.add);
}

}  // namespace tt
