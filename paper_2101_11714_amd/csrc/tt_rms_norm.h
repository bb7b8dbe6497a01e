// Residual addition and root-mean-square norm of rows, and its gradients.
//
// Forward:  h = residual + drop(x),  rstd = (mean_j h_j^2 + eps)^(-1/2),  y = h rstd w; in 8 bits (e4m3): with
//           s = max |y| / 448 over the row or over each group of columns, q = y / s.
// Backward: with g = dy w,  dh = rstd (g - h rstd^2 mean_j(g_j h_j)) + dsum;  dresidual = dh, dx = drop'(dh),
//           dw = sum over rows of dy h rstd.
// One pass over the rows: a row stays in the registers of its lanes between the sums and the products that need them.
// Bound by HBM where there are rows enough, by latency where there are few.
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

// eight weights of any type; ones where there are none
__device__ __forceinline__ void weights8(const void *w, int type, int v, int n, float (&x)[8])
{
    if (!w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 1.f;
    } else if (type == TT_F32) {
        widen8(fetch8((const float *)w + 8 * v, n), x);
    } else if (type == TT_BF16) {
        widen8(fetch8((const bf16_t *)w + 8 * v, n), x);
    } else {
        widen8(fetch8((const f16_t *)w + 8 * v, n), x);
    }
}

// the larger of two magnitudes, and NaN if either is
__device__ __forceinline__ float most_or_nan(float a, float b) { return a != a || a > b ? a : b; }

// Sum over the 1 << lg threads of a row (up to a wave by lane exchange, then by LDS: one slot per wave, in the waves' order).
// `slot`: NWAVES floats that no other reduction in flight uses; every thread of the workgroup calls.
template <typename F>
__device__ __forceinline__ float row_reduce(float x, int lg, float *slot, F f)
{
    const int in_wave = lg < 6 ? lg : 6;
    for (int b = 0; b < in_wave; ++b) x = f(x, __shfl_xor(x, 1 << b));
    if (lg > 6) {
        const int w = threadIdx.x >> 6, per = 1 << (lg - 6), w0 = w & ~(per - 1);
        if ((threadIdx.x & 63) == 0) slot[w] = x;
        __syncthreads();
        x = slot[w0];
        for (int q = 1; q < per; ++q) x = f(x, slot[w0 + q]);
    }
    return x;
}

__device__ __forceinline__ void put8_e4m3(uint8_t *p, int n, const float (&q)[8])
{
    struct __attribute__((packed, aligned(1))) Two { uint32_t v[2]; } r;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k], q[4 * k + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * k + 2], q[4 * k + 3], w, true);
        r.v[k] = (uint32_t)w;
    }
    if (n >= 8) {
        *reinterpret_cast<Two *>(p) = r;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = (uint8_t)(r.v[j >> 2] >> (8 * (j & 3)));
    }
}

// T: x and y (Y8: y in 8 bits), H: the residual stream.  1 << lg threads a row, VPT vectors a thread.
template <typename T, typename H, bool Y8, int VPT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_fwd_kernel(const NormArgs a, int lg)
{
    __shared__ float slots[2][BLOCK / WAVE];
    const int g = 1 << lg, t = threadIdx.x & (g - 1);
    const int64_t row = (int64_t)blockIdx.x * (BLOCK >> lg) + (threadIdx.x >> lg);
    const bool in = row < a.rows;
    float h[VPT][8];
    {
        Vec8<T> x[VPT];
        Vec8<H> res[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t, n = a.N - 8 * v;
            if (in && v < a.nv) {
                x[i] = fetch8((const T *)a.x + row * a.ld_x + 8 * v, n);
                if (a.residual) res[i] = fetch8((const H *)a.residual + row * a.ld_res + 8 * v, n);
            }
        }
        const DropKey key = drop_key(a.drop);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t;
            if (in && v < a.nv) {
                widen8(x[i], h[i]);
                if (a.drop.state) drop8(a.drop, drop_mask(a.drop, key, (uint64_t)row * (uint64_t)a.nv + (uint64_t)v), h[i]);
                if (a.residual) {
                    float r[8];
                    widen8(res[i], r);
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[i][j] += r[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = 0.f;
            }
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = i * g + t;
        if (a.sum && in && v < a.nv) put8((H *)a.sum + row * a.ld_sum + 8 * v, a.N - 8 * v, h[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(h[i][j], h[i][j], ss);
    }
    ss = row_reduce(ss, lg, slots[0], [](float p, float q) { return p + q; });
    const float rstd = 1.f / sqrtf(ss / (float)a.N + a.eps);
    if (a.rstd && in && t == 0) a.rstd[row] = rstd;
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = i * g + t, n = a.N - 8 * v;
        if (v < a.nv) {
            float w[8];
            weights8(a.weight, a.weight_type, v, n, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = j < n ? h[i][j] * rstd * w[j] : 0.f;
        }
        if constexpr (Y8) {
            if (!a.group) {
#pragma unroll
                for (int j = 0; j < 8; ++j) most = most_or_nan(most, fabsf(h[i][j]));
            }
        } else {
            if (in && v < a.nv) put8((T *)a.y + row * a.ld_y + 8 * v, n, h[i]);
        }
    }
    if constexpr (Y8) {
        if (!a.group) most = row_reduce(most, lg, slots[1], most_or_nan);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t, n = a.N - 8 * v;
            float m = most;
            if (a.group) {                                   // a group's lanes are neighbours: a power of two up to 16 (or all of a shorter row's)
                m = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) m = most_or_nan(m, fabsf(h[i][j]));
                for (int b = 1; b < (a.group >> 3); b <<= 1) m = most_or_nan(m, __shfl_xor(m, b));
            }
            const float s = m / E4M3_MOST;
            if (in && v < a.nv) {
                const bool none = s < 1.17549435e-38f;       // nothing but zeros, or too little for a scale of 32 bits
                const float inv = none ? 0.f : 1.f / s;
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = h[i][j] * inv;
                put8_e4m3((uint8_t *)a.y + row * a.ld_y + 8 * v, n, q);
                if (a.group ? (8 * v) % a.group == 0 : v == 0)
                    a.scales[row * a.ld_scales + (a.group ? (8 * v) / a.group : 0)] = none ? 0.f : s;
            }
        }
    }
}

struct NormGradArgs {
    const void *dy, *h, *weight, *dsum;                      // dsum: of h's type, or null
    const float *rstd;
    void *dx, *dres;                                         // either may be null
    float *part;                                             // [workgroup][nv * 8], or null: no gradient of the weight
    int64_t ld_dy, ld_h, ld_dsum, ld_dx, ld_dres, rows;
    int N, nv, weight_type;
    DropArgs drop;
};

// Rows go to the groups of threads in turn; a thread's columns are the same for all of them, so the weight's gradient of
// its rows stays in registers, and each workgroup leaves one row of sums.
template <typename T, typename H, int VPT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_bwd_kernel(const NormGradArgs a, int lg)
{
    __shared__ float slots[2][BLOCK / WAVE];
    extern __shared__ float lds[];                           // [groups - 1][nv * 8]
    const int g = 1 << lg, t = threadIdx.x & (g - 1), groups = BLOCK >> lg, gi = threadIdx.x >> lg;
    const DropKey key = drop_key(a.drop);
    float w[VPT][8], dw[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = i * g + t;
        if (v < a.nv) weights8(a.weight, a.weight_type, v, a.N - 8 * v, w[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = 0.f;
    }
    const float inv_n = 1.f / (float)a.N;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < a.rows; r0 += (int64_t)gridDim.x * groups, turn ^= 1) {
        const int64_t row = r0 + gi;
        const bool in = row < a.rows;
        Vec8<T> dy[VPT];
        Vec8<H> h[VPT], ds[VPT];
        float rstd = 0.f;
        if (in) {
            rstd = a.rstd[row];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int v = i * g + t, n = a.N - 8 * v;
                if (v < a.nv) {
                    dy[i] = fetch8((const T *)a.dy + row * a.ld_dy + 8 * v, n);
                    h[i] = fetch8((const H *)a.h + row * a.ld_h + 8 * v, n);
                    if (a.dsum) ds[i] = fetch8((const H *)a.dsum + row * a.ld_dsum + 8 * v, n);
                }
            }
        }
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t;
            if (in && v < a.nv) {
                float p[8], q[8];
                widen8(dy[i], p);
                widen8(h[i], q);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (8 * v + j < a.N) {
                        const float m = p[j] * q[j];
                        dot = fmaf(m, w[i][j], dot);
                        dw[i][j] = fmaf(m, rstd, dw[i][j]);
                    }
            }
        }
        dot = row_reduce(dot, lg, slots[turn], [](float p, float q) { return p + q; });
        const float c = dot * inv_n * rstd * rstd * rstd;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int v = i * g + t, n = a.N - 8 * v;
            if (!in || v >= a.nv) continue;
            float p[8], q[8], d[8];
            widen8(dy[i], p);
            widen8(h[i], q);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = p[j] * w[i][j] * rstd - q[j] * c;
            if (a.dsum) {
                float s[8];
                widen8(ds[i], s);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] += s[j];
            }
            if (a.dres) put8((H *)a.dres + row * a.ld_dres + 8 * v, n, d);
            if (a.dx) {
                if (a.drop.state) drop8(a.drop, drop_mask(a.drop, key, (uint64_t)row * (uint64_t)a.nv + (uint64_t)v), d);
                put8((T *)a.dx + row * a.ld_dx + 8 * v, n, d);
            }
        }
    }
    if (!a.part) return;
    if (groups > 1) {
        __syncthreads();
        if (gi) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (i * g + t < a.nv)
#pragma unroll
                    for (int j = 0; j < 8; ++j) lds[(gi - 1) * (8 * a.nv) + j * a.nv + i * g + t] = dw[i][j];
        }
        __syncthreads();
        if (gi) return;
        for (int q = 1; q < groups; ++q)
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (i * g + t < a.nv)
#pragma unroll
                    for (int j = 0; j < 8; ++j) dw[i][j] += lds[(q - 1) * (8 * a.nv) + j * a.nv + i * g + t];
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int v = i * g + t;
        if (v < a.nv) {
            float *p = a.part + (int64_t)blockIdx.x * (8 * a.nv) + 8 * v;
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = dw[i][j];
        }
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
