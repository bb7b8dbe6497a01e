// Products of few rows, bound by one reading of the second operand: no tile in LDS, its rows go from memory to the matrix cores' registers.
#pragma once

#include "tt_product.h"

namespace tt {

constexpr int PF_WAVES = 8, PF_MOST = 64;                    // waves of a workgroup, rows

// A workgroup takes 16 columns of C and all of k, every wave an eighth of k (in turns of PF_FLIGHT steps of 64 bytes, all of
// whose loads are on their way together); the waves' sums are added through LDS, in their order.
// MB: blocks of 16 rows.  WHOLE: operands are whole 16-byte chunks.
template <typename T, typename O, int MB, bool WHOLE>
__global__ __launch_bounds__(PF_WAVES *WAVE) void product_few_kernel(ProductArgs p, EpilogueArgs e)
{
    constexpr int CH = 16 / sizeof(T), STEP = 4 * CH, FLIGHT = MB == 1 ? 8 : MB == 2 ? 5 : 3;
    __shared__ __attribute__((aligned(16))) float sums[PF_WAVES][MB][BLOCK][BLOCK + 4];
    const int64_t n0 = workgroup() * BLOCK;
    if (n0 >= p.N) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const T *wrow = (const T *)p.b + (n0 + r < p.N ? n0 + r : p.N - 1) * p.ldb;
    const T *xrow[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) xrow[i] = (const T *)p.a + (16 * i + r < p.M ? 16 * i + r : p.M - 1) * p.lda;
    auto chunk = [&](const T *line, int64_t k) {
        if (!WHOLE) return fetch_chunk(line, k, p.K);
        const bool in = k < p.K;                             // (no branch around the load: what it brings is dropped)
        uint4 x = *reinterpret_cast<const uint4 *>(line + (in ? k : 0));
        x.x = in ? x.x : 0u;
        x.y = in ? x.y : 0u;
        x.z = in ? x.z : 0u;
        x.w = in ? x.w : 0u;
        return x;
    };
    mfma_acc_t acc[MB][1];
#pragma unroll
    for (int i = 0; i < MB; ++i) acc[i][0] = mfma_acc_t{0.f, 0.f, 0.f, 0.f};
    for (int64_t k0 = (int64_t)wave * FLIGHT * STEP; k0 < p.K; k0 += PF_WAVES * FLIGHT * STEP) {
        uint4 w[FLIGHT][1], x[FLIGHT][MB];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) w[f][0] = chunk(wrow, k0 + f * STEP + q * CH);
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f)
#pragma unroll
            for (int i = 0; i < MB; ++i) x[f][i] = chunk(xrow[i], k0 + f * STEP + q * CH);
        __builtin_amdgcn_sched_barrier(0);                   // (or the compiler loads them one after the other)
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) block_products<T>(w[f], x[f], acc);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i) *reinterpret_cast<mfma_acc_t *>(&sums[wave][i][r][4 * q]) = acc[i][0];
    __syncthreads();
    const int m = threadIdx.x >> 1, c = 8 * (threadIdx.x & 1);
    const int have = p.N - (n0 + c) < 8 ? (int)(p.N - (n0 + c)) : 8;
    if (m >= p.M || m >= 16 * MB || have <= 0) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias[8];
#pragma unroll 4
    for (int s = 0; s < PF_WAVES; ++s) {
        const float4 lo = *reinterpret_cast<const float4 *>(&sums[s][m >> 4][m & 15][c]), hi = *reinterpret_cast<const float4 *>(&sums[s][m >> 4][m & 15][c + 4]);
        v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w;
        v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
    }
    load_bias(e, n0 + c, have, bias);
    finish8<T, O>(e, m, n0 + c, have, bias, v);
}

}  // namespace tt
