// Residual addition and root-mean-square norm of rows, and its gradients.
//
// Forward:  h = residual + drop(x),  rstd = (mean_j h_j^2 + eps)^(-1/2),  y = h rstd w; in 8 bits (e4m3): with
//           s = max |y| / 448 over the row or over each group of columns, q = y / s.
// Backward: with g = dy w,  dh = rstd (g - h rstd^2 mean_j(g_j h_j)) + dsum;  dresidual = dh, dx = drop'(dh),
//           dw = sum over rows of dy h rstd.
// One pass over the rows: a row stays in the registers of its lanes between the sums and the products that need them.
// Bound by HBM where there are rows enough, by latency where there are few.  16,384 rows of 4,096 columns in 16 bits, residual added, into
// 8 bits with a scale per 128 columns: 82 us, 5.75 TB/s; 7 rows of 8,192: 4.6 us.  Gradients of 8,192 rows of 4,096 with a residual stream in
// 32 bits and dropout: 101 us, 5.3 TB/s; of 100,003 rows of 64 in 32 bits: 23 us, 4.4 TB/s.
#pragma once

#include "tt_rows_io.h"

namespace tt {

constexpr int RN_MOST = 32768;   // columns
constexpr float E4M3_MOST = 448.f;

struct NormArgs {
    const void *x, *residual, *weight;
    void *sum, *y;
    float *rstd, *scales;
    int64_t ld_x, ld_res, ld_sum, ld_y, ld_scales, rows;
    int N, nv, weight_type, group;                           // group: columns per scale, 0: the whole row
    float eps;
    DropArgs drop;
};

// N for fetch8 and settle8.  Rows that take two vectors of one thread have more than 8 columns: said here, so that the code for
// narrower ones is left out (with it odd widths spilled: gradients of 4,096 rows of 12,001 columns 356 -> 167 us, of 20,001
// 2,280 -> 609; forward, of 16,383, 133 -> 117)
template <int VPT>
__device__ __forceinline__ int row_columns(int N) { return VPT > 1 ? max(N, 8) : N; }

// the weights of a thread's vectors, of any type; ones where there are none
template <bool WHOLE, int VPT, typename W>
__device__ __forceinline__ void load_weights(const W *p, int g, int t, int nv, int N, float (&w)[VPT][8])
{
    Vec8<W> x[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = min(i * g + t, nv - 1);
        x[i] = fetch8<WHOLE>(p + 8 * v, N - 8 * v, row_columns<VPT>(N));
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        settle8<WHOLE>(x[i], N - 8 * min(i * g + t, nv - 1), row_columns<VPT>(N));
        widen8(x[i], w[i]);
    }
}

template <bool WHOLE, int VPT>
__device__ __forceinline__ void weights(const void *p, int type, int g, int t, int nv, int N, float (&w)[VPT][8])
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) w[i][j] = 1.f;
    } else if (type == TT_F32) {
        load_weights<WHOLE>((const float *)p, g, t, nv, N, w);
    } else if (type == TT_BF16) {
        load_weights<WHOLE>((const bf16_t *)p, g, t, nv, N, w);
    } else {
        load_weights<WHOLE>((const f16_t *)p, g, t, nv, N, w);
    }
}

// Magnitudes as whole numbers: in the order of their values, with NaN above all of them, so that the largest of some is NaN if one is
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// f over the 1 << lg threads of a row: up to a wave in registers, then by LDS, one place per wave, in the waves' order.
// `slot`: a place per wave that no other reduction in flight uses; every thread of the workgroup calls.
template <typename V, typename F>
__device__ __forceinline__ V row_reduce(V x, int lg, V *slot, F f)
{
    x = lanes_reduce(x, lg < 6 ? lg : 6, f);
    if (lg > 6) {
        const int w = threadIdx.x >> 6, per = 1 << (lg - 6), w0 = w & ~(per - 1);
        if ((threadIdx.x & 63) == 0) slot[w] = x;
        __syncthreads();
        x = slot[w0];
        for (int q = 1; q < per; ++q) x = f(x, slot[w0 + q]);
    }
    return x;
}

// Quotients y / s for e4m3, |y| <= 448 s, as dividing and rounding to 32 bits gives them.  A product with the correctly rounded
// reciprocal is off by a unit in the last place or so, which is enough to decide ties; one step with its remainder rounds it correctly wherever
// the product is within a unit (Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990), as it is beside
// the ties of e4m3: their five bits are too few for the cases that the step misses.  Four operations where a division takes a dozen: 7 rows
// of 8,192 columns in 16 bits 4.5 us (4.3 with the product alone, 4.8 with divisions), 16,384 of 4,096 81.5 (81.2, 82.2).
struct Quotient8 {
    float up, s, inv;
    __device__ __forceinline__ explicit Quotient8(float scale)
    {
        up = scale < 0x1p-64f ? 0x1p64f : 1.f;               // (remainders of small values would be no normal numbers)
        const float x = scale * up;
        inv = 1.f / x;
        s = x < __builtin_inff() ? x : 0.f;                  // (finite / inf = 0)
    }
    __device__ __forceinline__ float operator()(float y) const
    {
        const float x = y * up, q = x * inv;
        return fmaf(-fmaf(q, s, -x), inv, q);                // (of these signs, so that -0 stays -0)
    }
};

template <bool WHOLE>
__device__ __forceinline__ void put8_e4m3(uint8_t *p, int n, const float (&q)[8])
{
    struct __attribute__((packed, aligned(1))) Two { uint32_t v[2]; } r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k], q[4 * k + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k + 2], q[4 * k + 3], w, true);
        r.v[k] = (uint32_t)w;
    }
    if (WHOLE || n >= 8) {
        *reinterpret_cast<Two *>(p) = r;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = (uint8_t)(r.v[j >> 2] >> (8 * (j & 3)));
    }
}

constexpr int RN_THREADS = 1024, RN_WAVES = RN_THREADS / WAVE;

// T: x and y (Y8: y in 8 bits), H: the residual stream.  1 << lg threads a row, VPT vectors a thread.  No load stands in a branch
// (it would be waited for there): threads without a row or a vector load the last one.
template <typename T, typename H, bool Y8, int VPT, bool WHOLE, bool RESIDUAL>
__global__ __launch_bounds__(RN_THREADS) void norm_fwd_kernel(const NormArgs a, int lg)
{
    __shared__ float sums[RN_WAVES];
    __shared__ uint32_t mosts[RN_WAVES];
    const int g = 1 << lg, t = threadIdx.x & (g - 1);
    const int64_t row_ = workgroup() * (blockDim.x >> lg) + (threadIdx.x >> lg);
    const bool in = row_ < a.rows;
    const int64_t row = in ? row_ : a.rows - 1;
    float h[VPT][8], w[VPT][8];
    {
        Vec8<T> x[VPT];
        Vec8<H> res[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = min(i * g + t, a.nv - 1), n = a.N - 8 * v;
            x[i] = fetch8<WHOLE>((const T *)a.x + row_at(row, a.ld_x) + 8 * v, n, row_columns<VPT>(a.N));
            if constexpr (RESIDUAL) res[i] = fetch8<WHOLE>((const H *)a.residual + row_at(row, a.ld_res) + 8 * v, n, row_columns<VPT>(a.N));
        }
        const DropKey key = drop_key(a.drop);
        weights<WHOLE>(a.weight, a.weight_type, g, t, a.nv, a.N, w);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = min(i * g + t, a.nv - 1);
            settle8<WHOLE>(x[i], a.N - 8 * v, row_columns<VPT>(a.N));
            widen8(x[i], h[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] *= a.drop.factor;
            if (a.drop.state) drop8(a.drop, key, (uint64_t)row_at(row, a.nv) + (uint64_t)v, h[i]);
            if constexpr (RESIDUAL) {
                float r[8];
                settle8<WHOLE>(res[i], a.N - 8 * v, row_columns<VPT>(a.N));
                widen8(res[i], r);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] += r[j];
            }
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = i * g + t;
        float part = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) part = fmaf(h[i][j], h[i][j], part);     // (columns behind the last are 0)
        if (v < a.nv) {
            ss += part;
            if (a.sum && in) put8<WHOLE>((H *)a.sum + row_at(row, a.ld_sum) + 8 * v, a.N - 8 * v, h[i]);
        }
    }
    ss = row_reduce(ss, lg, sums, [](float p, float q) { return p + q; });
    const float rstd = 1.f / sqrtf(ss / (float)a.N + a.eps);
    if (a.rstd && in && t == 0) a.rstd[row] = rstd;
    uint32_t most[VPT];
    uint32_t row_most = 0u;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = i * g + t, n = a.N - 8 * v;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i][j] = h[i][j] * rstd * w[i][j];
        if constexpr (Y8) {
            uint32_t m = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = larger(m, WHOLE || j < n ? magnitude(h[i][j]) : 0u);
            most[i] = v < a.nv ? m : 0u;
            row_most = larger(row_most, most[i]);
        } else {
            if (in && v < a.nv) put8<WHOLE>((T *)a.y + row_at(row, a.ld_y) + 8 * v, n, h[i]);
        }
    }
    if constexpr (Y8) {
        int lg_group = 0;                                    // lanes of a group: neighbours, a power of two
        if (a.group) lg_group = __builtin_ctz(a.group) - 3;
        else row_most = row_reduce(row_most, lg, mosts, larger);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t, n = a.N - 8 * v;
            const uint32_t m = a.group ? lanes_reduce(most[i], lg_group, larger) : row_most;
            const float s = __uint_as_float(m) / E4M3_MOST;
            const bool none = s < 1.17549435e-38f;           // nothing but zeros, or too little for a scale of 32 bits
            const Quotient8 by(s);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = none ? 0.f : by(h[i][j]);
            if (in && v < a.nv) {
                put8_e4m3<WHOLE>((uint8_t *)a.y + row_at(row, a.ld_y) + 8 * v, n, h[i]);
                if (a.group ? (v & ((1 << lg_group) - 1)) == 0 : v == 0)
                    a.scales[row_at(row, a.ld_scales) + (a.group ? v >> lg_group : 0)] = none ? 0.f : s;
            }
        }
    }
}

struct NormGradArgs {
    const void *dy, *h, *weight, *dsum;                      // dsum: of h's type, or null
    const float *rstd;
    void *dx, *dres;                                         // either may be null
    float *part;                                             // [workgroup][nv * 8], or null: no gradient of the weight, or
    void *dw;                                                // here, from the only workgroup
    int dw_type, add;
    int64_t ld_dy, ld_h, ld_dsum, ld_dx, ld_dres, rows;
    int N, nv, weight_type;
    DropArgs drop;
};

template <typename W>
__device__ __forceinline__ void put_weight(W *p, float x, int add)
{
    *p = (W)(add ? (float)*p + x : x);
}

// Rows go to the groups of threads in turn; a thread's columns are the same for all of them, so the weight's gradient of
// its rows stays in registers, and each workgroup leaves one row of sums.  Loads as in norm_fwd_kernel.  AGAIN: the longest rows do not
// fit the registers beside it: they are read a second time, mostly from the L2.  AHEAD: the next row is loaded before this one's sum
// (65,536 rows of 256 columns 33 -> 29 us; with two vectors a thread nothing: 105.3 / 104.5 at 8,192 columns).
constexpr int RN_BWD_THREADS = 512;                          // (1,024 have too few registers)

template <typename T, typename H, int VPT, bool WHOLE, bool DSUM>
__global__ __launch_bounds__(RN_BWD_THREADS) void norm_bwd_kernel(const NormGradArgs a, int lg)
{
    __shared__ float slots[2][RN_BWD_THREADS / WAVE];
    constexpr int THREADS = RN_BWD_THREADS;
    constexpr bool AGAIN = VPT > 4, AHEAD = VPT == 1;
    extern __shared__ float lds[];                           // [waves, or groups of whole waves][nv * 8], if more than one
    const int g = 1 << lg, t = threadIdx.x & (g - 1), groups = THREADS >> lg, gi = threadIdx.x >> lg;
    const DropKey key = drop_key(a.drop);
    float w[VPT][8], dw[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = 0.f;
    weights<WHOLE>(a.weight, a.weight_type, g, t, a.nv, a.N, w);
    const float inv_n = 1.f / (float)a.N;
    struct Row {
        Vec8<T> dy[VPT];
        Vec8<H> h[VPT], ds[VPT];
        float rstd;
    };
    auto load = [&](Row &x, int64_t row, int i) {
        const int v = min(i * g + t, a.nv - 1), n = a.N - 8 * v;
        x.dy[i] = fetch8<WHOLE>((const T *)a.dy + row_at(row, a.ld_dy) + 8 * v, n, row_columns<VPT>(a.N));
        x.h[i] = fetch8<WHOLE>((const H *)a.h + row_at(row, a.ld_h) + 8 * v, n, row_columns<VPT>(a.N));
    };
    auto load_sum = [&](Row &x, int64_t row, int i) {
        const int v = min(i * g + t, a.nv - 1);
        if constexpr (DSUM) x.ds[i] = fetch8<WHOLE>((const H *)a.dsum + row_at(row, a.ld_dsum) + 8 * v, a.N - 8 * v, row_columns<VPT>(a.N));
    };
    auto load_row = [&](Row &x, int64_t r) {
        const int64_t row = r < a.rows ? r : a.rows - 1;
        x.rstd = a.rstd[row];
        if constexpr (!AGAIN) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                load(x, row, i);
                load_sum(x, row, i);
            }
        }
    };
    const int64_t step = (int64_t)gridDim.x * groups;
    Row ahead;
    if constexpr (AHEAD) load_row(ahead, (int64_t)blockIdx.x * groups + gi);
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < a.rows; r0 += step, turn ^= 1) {
        const bool in = r0 + gi < a.rows;
        const int64_t row = in ? r0 + gi : a.rows - 1;
        Row x;
        if constexpr (AHEAD) {
            x = ahead;
            load_row(ahead, r0 + step + gi);
        } else {
            load_row(x, row);
        }
        const float rstd = x.rstd;
        auto settle = [&](int i) {
            const int n = a.N - 8 * min(i * g + t, a.nv - 1);
            settle8<WHOLE>(x.dy[i], n, row_columns<VPT>(a.N));
            settle8<WHOLE>(x.h[i], n, row_columns<VPT>(a.N));
        };
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if constexpr (AGAIN) load(x, row, i);
            settle(i);
            float p[8], q[8], part = 0.f;
            widen8(x.dy[i], p);
            widen8(x.h[i], q);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float m = in ? p[j] * q[j] : 0.f;      // (columns behind the last are 0)
                part = fmaf(m, w[i][j], part);
                dw[i][j] = fmaf(m, rstd, dw[i][j]);
            }
            dot += i * g + t < a.nv ? part : 0.f;
        }
        dot = row_reduce(dot, lg, slots[turn], [](float p, float q) { return p + q; });
        const float c = dot * inv_n * rstd * rstd * rstd;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t, n = a.N - 8 * v;
            if constexpr (AGAIN) {
                load(x, row, i);
                load_sum(x, row, i);
                settle(i);
            }
            float p[8], q[8], d[8];
            widen8(x.dy[i], p);
            widen8(x.h[i], q);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = p[j] * w[i][j] * rstd - q[j] * c;
            if constexpr (DSUM) {
                float s[8];
                settle8<WHOLE>(x.ds[i], a.N - 8 * min(v, a.nv - 1), row_columns<VPT>(a.N));
                widen8(x.ds[i], s);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] += s[j];
            }
            if (!in || v >= a.nv) continue;
            if (a.dres) put8<WHOLE>((H *)a.dres + row_at(row, a.ld_dres) + 8 * v, n, d);
            if (a.dx) {
                if (a.drop.state) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] *= a.drop.factor;
                    drop8(a.drop, key, (uint64_t)row_at(row, a.nv) + (uint64_t)v, d);
                }
                put8<WHOLE>((T *)a.dx + row_at(row, a.ld_dx) + 8 * v, n, d);
            }
        }
    }
    if (!a.part && !a.dw) return;
    // groups of a wave by lane exchange, then waves (or groups of more than one wave) through LDS, in their order
    for (int b = lg; b < 6; ++b)
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) dw[i][j] += __shfl_xor(dw[i][j], 1 << b);
    const int parts = lg < 6 ? THREADS / WAVE : groups, at = lg < 6 ? threadIdx.x >> 6 : gi, cols = 8 * a.nv;
    auto leave = [&](int c, float y) {
        if (a.part) a.part[(int64_t)blockIdx.x * cols + c] = y;
        else if (c < a.N) {
            if (a.dw_type == TT_F32) put_weight((float *)a.dw + c, y, a.add);
            else if (a.dw_type == TT_BF16) put_weight((bf16_t *)a.dw + c, y, a.add);
            else put_weight((f16_t *)a.dw + c, y, a.add);
        }
    };
    if (lg >= 6 || (threadIdx.x & 63) < g) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t;
            if (v < a.nv) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (parts > 1) lds[at * cols + 8 * v + j] = dw[i][j];
                    else leave(8 * v + j, dw[i][j]);
                }
            }
        }
    }
    if (parts == 1) return;
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += THREADS) {
        float s = lds[c];
        for (int q = 1; q < parts; ++q) s += lds[q * cols + c];
        leave(c, s);
    }
}

// dw: the workgroups' rows of sums added up, 64 columns a workgroup; 64 threads take every 64th row each, their sums are
// added in their order.
template <typename W>
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float *part, int n_part, int N, int nv, W *dw, int add)
{
    __shared__ float4 sums[64][17];
    const int c = threadIdx.x & 15, r = threadIdx.x >> 4, col = blockIdx.x * 64 + 4 * c;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < 8 * nv) {
#pragma unroll 4
        for (int q = r; q < n_part; q += 64) {
            const float4 x = *reinterpret_cast<const float4 *>(part + (int64_t)q * (8 * nv) + col);
            s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
        }
    }
    sums[r][c] = s;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const int at = blockIdx.x * 64 + threadIdx.x;
    if (at >= N) return;
    float y = add ? (float)dw[at] : 0.f;
    for (int q = 0; q < 64; ++q) y += reinterpret_cast<const float *>(&sums[q][threadIdx.x >> 2])[threadIdx.x & 3];
    dw[at] = (W)y;
}

}  // namespace tt
