// The launches behind product_of, for the files that compile the kernels of a type.
#pragma once

#include "tt_product_launch.h"

namespace tt {

// C = A B^T; AK, BK: the operands' rows are dense in k
template <typename T, typename O, bool AK, bool BK>
int launch_product(Operand a, Operand b, int64_t M, int64_t N, int64_t K, const EpilogueArgs &e, void *workspace, hipStream_t st)
{
    if (M == 0 || N == 0) return TT_OK;
    const Plan p = plan_of(M, N, K, sizeof(T) == 4 ? TT_F32 : TT_BF16, AK && BK);
    if constexpr (sizeof(T) == 2)
        if (K > 0 && (a.packed || b.packed)) {
            PackArgs q{};
            int64_t wgs = 0;
            auto pack = [&](int i, Operand &o) {
                if (!o.packed) return;
                q.from[i] = o.data;
                q.to[i] = o.packed;
                q.ld[i] = o.ld;
                q.columns[i] = o.columns;
                q.row[i] = (int)ceil_div(o.columns, 8);
                q.chunks[i] = o.rows * q.row[i];
                wgs += ceil_div(q.chunks[i], WG * PACK_U);
                o.data = o.packed;
                o.ld = 8 * q.row[i];
            };
            pack(0, a);
            pack(1, b);
            hipLaunchKernelGGL((pack_kernel<T>), grid_of(wgs, WG), dim3(WG), 0, st, q);
        }
    ProductArgs q{a.data, b.data, a.ld, b.ld, M, N, K, (int)p.tiles_m, (int)p.tiles_n, p.k_part, p.parts > 1 ? (float *)workspace : nullptr, 8 * ceil_div(N, 8)};
    if (p.way == FEW) {
        if constexpr (AK && BK) {
            const bool odd = sizeof(T) == 2 && (a.ld % 2 || b.ld % 2 || (uintptr_t)a.data % 4 || (uintptr_t)b.data % 4);
            with_flag(odd, [&](auto o) {
                constexpr bool ODD = sizeof(T) == 2 && decltype(o)::value;
                auto launch = [&](auto mb, auto nb) {
                    constexpr int MB = decltype(mb)::value, NB = decltype(nb)::value;
                    hipLaunchKernelGGL((product_few_kernel<T, O, MB, NB, ODD>), grid_of(ceil_div(N, BLOCK * NB), PF_WAVES * WAVE), dim3(PF_WAVES * WAVE), 0, st, q, e);
                };
                constexpr std::integral_constant<int, 1> one{};
                constexpr std::integral_constant<int, 2> two{};
                constexpr std::integral_constant<int, 4> four{};
                // two blocks of columns share a reading of x where that leaves a workgroup for every compute unit
                if (M <= 16) launch(one, one);
                else if (M <= 32 && N < 256 * 32) launch(two, one);
                else if (M <= 32) launch(two, two);
                else if (N < 256 * 32) launch(four, one);
                else launch(four, two);
            });
        }
        return launched("product launch");
    }
    dim3 grid = grid_of(p.tiles_m * p.tiles_n, WG);
    grid.z = (unsigned)p.parts;
    if constexpr (sizeof(T) == 4) {
        if (p.way == TILES) hipLaunchKernelGGL((product_kernel<T, O, AK, BK, 64>), grid, dim3(WG), 0, st, q, e);
        else hipLaunchKernelGGL((product_kernel<T, O, AK, BK, 128>), grid, dim3(WG), 0, st, q, e);
    } else {
        int rc = TT_OK;
        with_flag(p.way == STREAM_WIDE, [&](auto w) {
            typedef StreamShape<decltype(w)::value> S;
            const auto kernel = product_stream_kernel<T, O, AK, BK, decltype(w)::value>;
            static OncePerDevice once;
            const hipError_t err = allow_dynamic_lds(once, (const void *)kernel, S::LDS);
            if (err != hipSuccess) {
                rc = hip_fail(err, "LDS of a product");
                return;
            }
            hipLaunchKernelGGL(kernel, grid, dim3(S::THREADS), S::LDS, st, q, e);
        });
        if (rc) return rc;
    }
    if (p.parts > 1) hipLaunchKernelGGL((join_parts_kernel<T, O>), grid_of(ceil_div(M * (q.ld_part / 8), WG), WG), dim3(WG), 0, st, q, e, p.parts);
    return launched("product launch");
}

template <typename T>
int product_of(Layout layout, int32_t out_type, const Operand &a, const Operand &b, int64_t M, int64_t N, int64_t K, const EpilogueArgs &e, void *workspace, hipStream_t st)
{
    if (layout == DENSE_STRIDED) return launch_product<T, T, true, false>(a, b, M, N, K, e, workspace, st);
    if (layout == STRIDED_STRIDED) {
        if (out_type == TT_F32) return launch_product<T, float, false, false>(a, b, M, N, K, e, workspace, st);
        return launch_product<T, T, false, false>(a, b, M, N, K, e, workspace, st);
    }
    if (out_type == TT_F32) return launch_product<T, float, true, true>(a, b, M, N, K, e, workspace, st);
    return launch_product<T, T, true, true>(a, b, M, N, K, e, workspace, st);
}

}  // namespace tt
