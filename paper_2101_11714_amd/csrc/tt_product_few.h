// Products of few rows, bound by one reading of the second operand: no tile in LDS, its rows go from memory to the matrix cores' registers.
#pragma once

#include "tt_product.h"

namespace tt {

constexpr int PF_WAVES = 8, PF_MOST = 64;                    // waves of a workgroup, rows

// A workgroup takes 16 * NB columns of C and all of k, every wave an eighth of k (in turns of FLIGHT steps of 64 bytes, all of whose loads are on their
// way together, from any address; the last turn looks at every chunk); the waves' sums are added through LDS, in their order.
// Workgroups begin at different places of k, so that rows of 2^n bytes do not keep a few channels of memory busy at a time (fp32, 1 x 4,096 x 12,288 44.6 -> 37.3 us, bf16, 8 x 8,192 x 8,192 33 -> 27.6).
// MB: blocks of 16 rows.  ODD: rows of 16-bit values begin at places that are no multiples of 4 bytes.
template <typename T, typename O, int MB, int NB, bool ODD>
__global__ __launch_bounds__(PF_WAVES *WAVE) void product_few_kernel(ProductArgs p, EpilogueArgs e)
{
    constexpr int CH = 16 / sizeof(T), STEP = 4 * CH, FLIGHT = MB + NB <= 2 ? 8 : MB + NB <= 4 ? 4 : 3, TURN = FLIGHT * STEP;
    __shared__ __attribute__((aligned(16))) float sums[PF_WAVES][MB][BLOCK][BLOCK * NB + 4];
    const int64_t n0 = workgroup() * (BLOCK * NB);
    if (n0 >= p.N) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const T *wrow[NB], *xrow[MB];
#pragma unroll
    for (int j = 0; j < NB; ++j) wrow[j] = (const T *)p.b + (n0 + 16 * j + r < p.N ? n0 + 16 * j + r : p.N - 1) * p.ldb;
#pragma unroll
    for (int i = 0; i < MB; ++i) xrow[i] = (const T *)p.a + (16 * i + r < p.M ? 16 * i + r : p.M - 1) * p.lda;
    mfma_acc_t acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = mfma_acc_t{0.f, 0.f, 0.f, 0.f};
    auto turn = [&](int64_t k0, auto load, auto get) {
        Chunk<T, ODD> w[FLIGHT][NB], x[FLIGHT][MB];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f)
#pragma unroll
            for (int j = 0; j < NB; ++j) load(w[f][j], wrow[j], k0 + f * STEP + q * CH);
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f)
#pragma unroll
            for (int i = 0; i < MB; ++i) load(x[f][i], xrow[i], k0 + f * STEP + q * CH);
        __builtin_amdgcn_sched_barrier(0);                   // (or the compiler loads them one after the other)
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            uint4 a[MB], b[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) b[j] = get(w[f][j], k0 + f * STEP + q * CH);
#pragma unroll
            for (int i = 0; i < MB; ++i) a[i] = get(x[f][i], k0 + f * STEP + q * CH);
            block_products<T>(b, a, acc);
        }
    };
    auto full = [&](int64_t k) { turn(k, [](Chunk<T, ODD> &c, const T *line, int64_t k) { c.load(line + k); }, [](const Chunk<T, ODD> &c, int64_t) { return c.get(); }); };
    const int rounds = (int)(p.K / (PF_WAVES * TURN));
    int at = rounds ? (int)(workgroup() % rounds) : 0;
#pragma unroll 1
    for (int i = 0; i < rounds; ++i, at = at + 1 < rounds ? at + 1 : 0) full(((int64_t)at * PF_WAVES + wave) * TURN);
    int64_t k0 = ((int64_t)rounds * PF_WAVES + wave) * TURN;
    if (k0 + TURN <= p.K) {
        full(k0);
        k0 = p.K;
    }
    if (k0 < p.K) turn(k0, [&](Chunk<T, ODD> &c, const T *line, int64_t k) { c.load(line, k, p.K); }, [&](const Chunk<T, ODD> &c, int64_t k) { return c.get(k, p.K); });
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) *reinterpret_cast<mfma_acc_t *>(&sums[wave][i][r][16 * j + 4 * q]) = acc[i][j];
    __syncthreads();
    for (int at = threadIdx.x; at < 16 * MB * 2 * NB; at += PF_WAVES * WAVE) {
        const int m = at / (2 * NB), c = 8 * (at % (2 * NB));
        const int have = p.N - (n0 + c) < 8 ? (int)(p.N - (n0 + c)) : 8;
        if (m >= p.M || have <= 0) continue;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias[8];
        load_bias(e, n0 + c, have, bias);
#pragma unroll 4
        for (int s = 0; s < PF_WAVES; ++s) {
            const float4 lo = *reinterpret_cast<const float4 *>(&sums[s][m >> 4][m & 15][c]), hi = *reinterpret_cast<const float4 *>(&sums[s][m >> 4][m & 15][c + 4]);
            v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w;
            v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
        }
        finish8<T, O>(e, m, n0 + c, have, bias, v);
    }
}

}  // namespace tt
