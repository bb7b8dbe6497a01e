// Norm of every head and rotation by position, forward and backward.
//
// A unit is 16 columns of a head: eight pairs that are turned (eight columns of each half, or eight pairs of neighbours), or 16 columns behind
// those.  A head is the 1 << lg neighbouring lanes that have a unit each; a lane keeps its columns in registers from the load to the store, so
// that a head is read once.  A workgroup takes some rows at a time: it leaves the cosines and sines of their pairs in LDS, once for all heads,
// and goes through the rows' heads, queries' and keys' alike.
#pragma once

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
    int q_heads, heads;          // heads: of queries and keys together
    const void *positions;
    int64_t ld_positions;
    const float *freqs;
    int positions64, pairs, ends[4], neighbours;
    int64_t rows;
    int D, units, turned;        // units of a head, of which so many are turned
    int lg, chunk;               // lanes of a head, rows at a time
    float eps;
    float *part;                 // backward: [workgroups][2][D] sums of the weights' gradients, null: not wanted
};

// cos and sin of 2 pi t.  The fraction of a turn is taken in 64 bits; from the nearest quarter it is an eighth at most, pi / 4 as an angle, where
// the Taylor series up to x^9 and x^10 are exact to 3e-9.
__device__ __forceinline__ float2 turn_of(double t)
{
    t -= rint(t);
    const double q = rint(4.0 * t);
    const float x = (float)((t - 0.25 * q) * 6.283185307179586), z = x * x;
    const float s = x * (1.f + z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880)))));
    const float c = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 + z * (-1.f / 3628800)))));
    const int quarter = (int)q & 3;
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    return make_float2(quarter == 1 || quarter == 2 ? -a : a, quarter >= 2 ? -b : b);
}

// cosines and sines of `n` rows from `row` on into LDS, [rows][pairs]
__device__ __forceinline__ void leave_turns(const RotateArgs &a, int64_t row, int n, float2 *turns)
{
    for (int i = threadIdx.x; i < n * a.pairs; i += WG) {
        const int r = i / a.pairs, p = i - r * a.pairs;
        const int axis = p < a.ends[0] ? 0 : p < a.ends[1] ? 1 : p < a.ends[2] ? 2 : 3;
        const int64_t at = axis * a.ld_positions + row + r;
        const double pos = a.positions64 ? (double)((const int64_t *)a.positions)[at] : (double)((const int32_t *)a.positions)[at];
        turns[i] = turn_of(pos * ((double)a.freqs[p] * 0.15915494309189535));
    }
}

// Where a unit's two vectors of eight begin, and how many columns of each there are.
struct Unit {
    int at[2], n[2];
    int limit;                   // columns in the part of the head that the vectors lie in
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
    return r;
}

// Up to eight columns of a head from column `at` on, zeros behind the n-th: the vector that ends at the head's end, or begins at its start,
// is loaded where fewer than eight lie there.  D: the head's columns.
template <typename T>
__device__ __forceinline__ void load_unit(const T *head, int at, int n, int D, float (&x)[8])
{
    if (at + 8 <= D) {
        widen8(fetch8<true>(head + at, 8, 8), x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = (float)head[j < n ? at + j : 0];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < n ? x[j] : 0.f;
}

template <typename T>
__device__ __forceinline__ void store_unit(T *head, int at, int n, const float (&x)[8])
{
    if (n > 0) put8(head + at, n, x);
}

__device__ __forceinline__ void load_weight(const void *w, int type, const Unit &u, float (&x)[2][8])
{
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = j < u.n[h] ? u.at[h] + j : 0;
            x[h][j] = !w ? 1.f : type == TT_F32 ? ((const float *)w)[c] : type == TT_BF16 ? (float)((const bf16_t *)w)[c] : (float)((const f16_t *)w)[c];
        }
}

// the unit's pairs turned; BACK: the other way round
template <bool BACK>
__device__ __forceinline__ void turn_unit(const RotateArgs &a, const float2 *turns, int u, float (&x)[2][8])
{
    float y[2][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 t = turns[min(8 * u + j, a.pairs - 1)];
        const float s = BACK ? -t.y : t.y;
        const float v = a.neighbours ? x[j >> 2][2 * j & 7] : x[0][j], w = a.neighbours ? x[j >> 2][(2 * j & 7) + 1] : x[1][j];
        y[0][j] = v * t.x - w * s;
        y[1][j] = w * t.x + v * s;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[0][j] = a.neighbours ? y[j & 1][j >> 1] : y[0][j];
        x[1][j] = a.neighbours ? y[j & 1][4 + (j >> 1)] : y[1][j];
    }
}

template <typename T>
__device__ __forceinline__ T *head_at(const Heads &h, int64_t row, int head) { return (T *)h.data + row * h.ld + head * h.ld_head; }

template <typename T, bool NORM>
__global__ __launch_bounds__(WG) void rotate_kernel(RotateArgs a)
{
    extern __shared__ float2 turns[];
    const int g = 1 << a.lg, u = threadIdx.x & (g - 1), group = threadIdx.x >> a.lg, groups = WG >> a.lg;
    const bool in = u < a.units;
    const Unit unit = unit_of(a, in ? u : 0);
    const int64_t row0 = workgroup() * a.chunk;
    if (row0 >= a.rows) return;
    const int n = a.rows - row0 < a.chunk ? (int)(a.rows - row0) : a.chunk;
    leave_turns(a, row0, n, turns);
    __syncthreads();
    for (int i = group; i < n * a.heads; i += groups) {
        const int r = i / a.heads, head = i - r * a.heads;
        const bool key = head >= a.q_heads;
        const int h = key ? head - a.q_heads : head;
        const int64_t row = row0 + r;
        const T *src = head_at<T>(key ? a.k : a.q, row, h);
        float x[2][8];
        load_unit(src, unit.at[0], in ? unit.n[0] : 0, a.D, x[0]);
        load_unit(src, unit.at[1], in ? unit.n[1] : 0, a.D, x[1]);
        if (NORM) {
            float s = 0.f, w[2][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s += x[0][j] * x[0][j] + x[1][j] * x[1][j];
            s = lanes_reduce(s, a.lg, [](float p, float q) { return p + q; });
            const float rho = 1.f / sqrtf(s / (float)a.D + a.eps);
            load_weight(key ? a.wk : a.wq, key ? a.wk_type : a.wq_type, unit, w);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) x[c][j] *= rho * w[c][j];
        }
        if (!in) continue;
        if (u < a.turned) turn_unit<false>(a, turns + r * a.pairs, u, x);
        T *dst = head_at<T>(key ? a.ok : a.oq, row, h);
        store_unit(dst, unit.at[0], unit.n[0], x[0]);
        store_unit(dst, unit.at[1], unit.n[1], x[1]);
    }
}

template <typename T, bool NORM>
__global__ __launch_bounds__(WG) void rotate_bwd_kernel(RotateArgs a)
{
    extern __shared__ float2 turns[];
    const int g = 1 << a.lg, u = threadIdx.x & (g - 1), group = threadIdx.x >> a.lg, groups = WG >> a.lg;
    const bool in = u < a.units;
    const Unit unit = unit_of(a, in ? u : 0);
    float dw[2][2][8] = {};
    for (int64_t row0 = (int64_t)blockIdx.x * a.chunk; row0 < a.rows; row0 += (int64_t)gridDim.x * a.chunk) {
        const int n = a.rows - row0 < a.chunk ? (int)(a.rows - row0) : a.chunk;
        __syncthreads();
        leave_turns(a, row0, n, turns);
        __syncthreads();
        for (int i = group; i < n * a.heads; i += groups) {
            const int r = i / a.heads, head = i - r * a.heads;
            const bool key = head >= a.q_heads;
            const int h = key ? head - a.q_heads : head;
            const int64_t row = row0 + r;
            const T *grad = head_at<T>(key ? a.gk : a.gq, row, h);
            float d[2][8];
            load_unit(grad, unit.at[0], in ? unit.n[0] : 0, a.D, d[0]);
            load_unit(grad, unit.at[1], in ? unit.n[1] : 0, a.D, d[1]);
            if (in && u < a.turned) turn_unit<true>(a, turns + r * a.pairs, u, d);
            if (NORM) {
                float x[2][8], w[2][8], s = 0.f, dot = 0.f;
                const T *src = head_at<T>(key ? a.k : a.q, row, h);
                load_unit(src, unit.at[0], in ? unit.n[0] : 0, a.D, x[0]);
                load_unit(src, unit.at[1], in ? unit.n[1] : 0, a.D, x[1]);
                load_weight(key ? a.wk : a.wq, key ? a.wk_type : a.wq_type, unit, w);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        s += x[c][j] * x[c][j];
                        dot += d[c][j] * w[c][j] * x[c][j];
                    }
                s = lanes_reduce(s, a.lg, [](float p, float q) { return p + q; });
                dot = lanes_reduce(dot, a.lg, [](float p, float q) { return p + q; });
                const float rho = 1.f / sqrtf(s / (float)a.D + a.eps), along = rho * rho * dot / (float)a.D;
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float p = d[c][j] * x[c][j] * rho;
                        dw[0][c][j] += key ? 0.f : p;
                        dw[1][c][j] += key ? p : 0.f;
                        d[c][j] = rho * (d[c][j] * w[c][j] - x[c][j] * along);
                    }
            }
            if (!in) continue;
            T *dst = head_at<T>(key ? a.ok : a.oq, row, h);
            store_unit(dst, unit.at[0], unit.n[0], d[0]);
            store_unit(dst, unit.at[1], unit.n[1], d[1]);
        }
    }
    if (!NORM || !a.part) return;
    // the groups' sums: lanes of a wave, then waves through LDS, in their order
    float *sums = reinterpret_cast<float *>(turns);
    const int cols = 16 * a.units, lanes = g < WAVE ? g : WAVE;
    for (int b = a.lg; b < 6; ++b)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) dw[s][c][j] += __shfl_xor(dw[s][c][j], 1 << b);
    for (int s = 0; s < 2; ++s) {
        __syncthreads();
        if ((int)(threadIdx.x & 63) < lanes && in)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) sums[(threadIdx.x >> 6) * cols + 16 * u + 8 * c + j] = s ? dw[1][c][j] : dw[0][c][j];
        __syncthreads();
        for (int i = threadIdx.x; i < cols; i += WG) {
            const Unit x = unit_of(a, i >> 4);
            const int c = i >> 3 & 1, j = i & 7;
            if (j < (c ? x.n[1] : x.n[0])) a.part[((int64_t)blockIdx.x * 2 + s) * a.D + (c ? x.at[1] : x.at[0]) + j] = (sums[i] + sums[cols + i]) + (sums[2 * cols + i] + sums[3 * cols + i]);
        }
    }
}

// the workgroups' sums added in their order: blockIdx.y 0 the queries' weight, 1 the keys'
__global__ __launch_bounds__(WG) void rotate_weight_kernel(const float *part, int n_part, int D, void *gq, int gq_type, void *gk, int gk_type, int add)
{
    __shared__ float sums[8][32];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5, at = blockIdx.x * 32 + c, which = blockIdx.y;
    void *out = which ? gk : gq;
    if (!out) return;
    const int type = which ? gk_type : gq_type;
    float s = 0.f;
    if (at < D)
        for (int b = q; b < n_part; b += 8) s += part[((int64_t)b * 2 + which) * D + at];
    sums[q][c] = s;
    __syncthreads();
    if (q || at >= D) return;
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y += sums[i][c];
    if (type == TT_F32) ((float *)out)[at] = y + (add ? ((float *)out)[at] : 0.f);
    else if (type == TT_BF16) ((bf16_t *)out)[at] = (bf16_t)(y + (add ? (float)((bf16_t *)out)[at] : 0.f));
    else ((f16_t *)out)[at] = (f16_t)(y + (add ? (float)((f16_t *)out)[at] : 0.f));
}

}  // namespace tt
