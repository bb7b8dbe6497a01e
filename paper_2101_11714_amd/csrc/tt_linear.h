// What the gradients of a product with an activation need beside the products: the gradient in front of the activation, and the
// bias's, whose columns' sums are left per band of rows.
#pragma once

#include "tt_product.h"

namespace tt {

struct SlopeArgs {
    const void *dy, *pre;        // (pre is not looked at without an activation)
    void *dz;                    // rows of nv vectors, zeros behind the N-th column; null: not wanted
    float *part;                 // [bands][8 nv] sums of columns, null: not wanted, or
    BiasSum one;                 // of one band: the bias's gradient
    int64_t ld_dy, ld_pre, ld_dz;
    int64_t rows, band;          // rows of a band
    int N, nv, act;
    int groups;                  // workgroups of a band; those behind them copy the products' other operands
};

// dz is rounded to the operands' type, which the matrix cores take for both operands alike; the bias's sums take it as it is.  In 16 bits that makes the gradients'
// relative error 0.0023 where their own last rounding alone is 0.0017 (bfloat16, 8,192 x 4,096 x 4,096); dz as the sum of two such numbers would double the
// products, 424 of 456 us.  Who needs more has the call in 32 bits.
// 32 vectors of eight columns x 8 rows per workgroup at a time, down a band of rows; bound by memory (8,192 x 4,096 in 16 bits with SiLU 45 us, 4.5 TB/s).
template <typename T, bool WHOLE, bool ACT>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a, PackArgs p)
{
    if constexpr (sizeof(T) == 2)
        if ((int)blockIdx.x >= a.groups) return pack_rows<T>(p, (int64_t)(blockIdx.x - a.groups) * gridDim.y + blockIdx.y);
    __shared__ float sums[8][32][8];
    const int v = blockIdx.x * 32 + (threadIdx.x & 31), lane_row = threadIdx.x >> 5;
    const int n = a.N - 8 * v;
    const int64_t first = (int64_t)blockIdx.y * a.band, last = first + a.band < a.rows ? first + a.band : a.rows;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (v < a.nv) {
        constexpr int U = sizeof(T) == 4 ? 2 : 4;            // rows whose loads are on their way together
#pragma unroll 1
        for (int64_t r0 = first + lane_row; r0 < last; r0 += 8 * U) {
            Vec8<T> x[U], y[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int64_t r = r0 + 8 * i < last ? r0 + 8 * i : r0;
                x[i] = fetch8<WHOLE>((const T *)a.dy + row_at(r, a.ld_dy) + 8 * v, n, a.N);
                if (ACT) y[i] = fetch8<WHOLE>((const T *)a.pre + row_at(r, a.ld_pre) + 8 * v, n, a.N);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int64_t r = r0 + 8 * i;
                if (r >= last) break;
                float d[8];
                settle8<WHOLE>(x[i], n, a.N);
                widen8(x[i], d);
                if (ACT) {
                    float z[8];
                    settle8<WHOLE>(y[i], n, a.N);
                    widen8(y[i], z);
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] *= act_slope(z[j], a.act);
                }
                if (a.dz) put8<true>((T *)a.dz + row_at(r, a.ld_dz) + 8 * v, 8, d);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += d[j];
            }
        }
    }
    if (!a.part && !a.one.db) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[lane_row][threadIdx.x & 31][j] = s[j];
    __syncthreads();
    const int c = threadIdx.x, at = blockIdx.x * 256 + c;
    if (at >= 8 * a.nv) return;
    float y = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) y += sums[q][c >> 3][c & 7];
    if (a.part) a.part[(int64_t)blockIdx.y * 8 * a.nv + at] = y;
    else if (at < a.N) leave_bias(a.one, at, y);
}

}  // namespace tt
