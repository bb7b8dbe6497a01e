// The launches behind product_of, for the files that compile the kernels of a type.
#pragma once

#include "tt_product_launch.h"

namespace tt {

template <typename T>
void pack(Operand &a, Operand &b, hipStream_t st)
{
    int64_t wgs;
    const PackArgs q = pack_args(a, b, wgs);
    if (wgs) hipLaunchKernelGGL((pack_kernel<T>), grid_of(wgs, WG), dim3(WG), 0, st, q);
}

inline ProductArgs args_of(const Product &x, const Plan &p)
{
    return {x.a.data, x.b.data, x.a.ld, x.b.ld, x.d.M, x.d.N, x.d.K, (int)p.tiles_m, (int)p.tiles_n, p.parts, p.k_part, p.parts > 1 ? x.parts : nullptr, 8 * ceil_div(x.d.N, 8)};
}

inline int64_t join_workgroups(const ProductArgs &q) { return q.parts > 1 ? ceil_div(q.M * (q.ld_part / 8), WG) : 0; }

// calls f with the rows of a kind's tiles
template <typename T, typename F>
void with_kind(int kind, F f)
{
    if constexpr (sizeof(T) == 4) {
        if (kind == 0) f(std::integral_constant<int, 128>{});
        else if (kind == 1) f(std::integral_constant<int, 64>{});
        else f(std::integral_constant<int, 32>{});
    } else {
        if (kind == 0) f(std::integral_constant<int, 256>{});
        else f(std::integral_constant<int, 128>{});
    }
}

// a kernel whose LDS is given with its launch
template <auto KERNEL, typename... A>
int launch_stream(dim3 grid, int threads, int lds, hipStream_t st, const A &...args)
{
    static OncePerDevice once;
    const hipError_t err = allow_dynamic_lds(once, (const void *)KERNEL, lds);
    if (err != hipSuccess) return hip_fail(err, "LDS of a product");
    hipLaunchKernelGGL(KERNEL, grid, dim3(threads), lds, st, args...);
    return TT_OK;
}

template <typename T, typename O>
int launch_product(Product x, hipStream_t st)
{
    const Size &d = x.d;
    if (d.M == 0 || d.N == 0) return TT_OK;
    if (x.few) {
        const ProductArgs q = args_of(x, Plan{0, 0, 1, d.K});
        const bool odd = sizeof(T) == 2 && (x.a.ld % 2 || x.b.ld % 2 || (uintptr_t)x.a.data % 4 || (uintptr_t)x.b.data % 4);
        with_flag(odd, [&](auto o) {
            constexpr bool ODD = sizeof(T) == 2 && decltype(o)::value;
            auto launch = [&](auto mb, auto nb) {
                constexpr int MB = decltype(mb)::value, NB = decltype(nb)::value;
                hipLaunchKernelGGL((product_few_kernel<T, O, MB, NB, ODD>), grid_of(ceil_div(d.N, BLOCK * NB), PF_WAVES * WAVE), dim3(PF_WAVES * WAVE), 0, st, q, x.e);
            };
            constexpr std::integral_constant<int, 1> one{};
            constexpr std::integral_constant<int, 2> two{};
            constexpr std::integral_constant<int, 4> four{};
            // two blocks of columns share a reading of x where that leaves a workgroup for every compute unit
            if (d.M <= 16) launch(one, one);
            else if (d.M <= 32 && d.N < 256 * 32) launch(two, one);
            else if (d.M <= 32) launch(two, two);
            else if (d.N < 256 * 32) launch(four, one);
            else launch(four, two);
        });
        return launched("product launch");
    }
    if constexpr (sizeof(T) == 2) pack<T>(x.a, x.b, st);
    const Plan &p = x.plan;
    const ProductArgs q = args_of(x, p);
    int rc = TT_OK;
    const dim3 grid = grid_of(p.tiles_m * p.tiles_n * p.parts, 512);
    with_kind<T>(x.kind, [&](auto size) {
        constexpr int TILE = decltype(size)::value;
        if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((product_kernel<T, O, TILE>), grid, dim3(WG), 0, st, q, x.e);
        else rc = launch_stream<product_stream_kernel<T, O, TILE == 256>>(grid, StreamShape<TILE == 256>::THREADS, StreamShape<TILE == 256>::LDS, st, q, x.e);
    });
    if (rc) return rc;
    if (p.parts > 1) hipLaunchKernelGGL((join_parts_kernel<T, O>), grid_of(join_workgroups(q), WG), dim3(WG), 0, st, q, x.e);
    return launched("product launch");
}

template <typename T, typename W>
int launch_gradients(Product dx, Product dw, const BiasSum &b, hipStream_t st)
{
    if constexpr (sizeof(T) == 2) pack<T>(dx.b, dw.b, st);
    const Plan &px = dx.plan, &pw = dw.plan;
    PairArgs g{{args_of(dx, px), args_of(dw, pw)}, {dx.e, dw.e}, pw.k_part > px.k_part, {px.tiles_m * px.tiles_n * px.parts, pw.tiles_m * pw.tiles_n * pw.parts}};
    int rc = TT_OK;
    const dim3 grid = grid_of(g.wgs[0] + g.wgs[1], 512);
    if (g.wgs[0] + g.wgs[1] > 0)
        with_kind<T>(dx.kind, [&](auto size) {
            constexpr int TILE = decltype(size)::value;
            if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((pair_kernel<T, W, TILE>), grid, dim3(WG), 0, st, g);
            else rc = launch_stream<pair_stream_kernel<T, W, TILE == 256>>(grid, StreamShape<TILE == 256>::THREADS, StreamShape<TILE == 256>::LDS, st, g);
        });
    if (rc) return rc;
    const int64_t wgs0 = g.wgs[0] ? join_workgroups(g.p[0]) : 0, wgs1 = g.wgs[1] ? join_workgroups(g.p[1]) : 0, all = wgs0 + wgs1 + (b.part ? ceil_div(b.N, 32) : 0);
    if (all) hipLaunchKernelGGL((finish_pair_kernel<T, W>), grid_of(all, WG), dim3(WG), 0, st, g, b, wgs0, wgs1);
    return g.wgs[0] + g.wgs[1] + all > 0 ? launched("gradient launch") : TT_OK;
}

template <typename T>
int product_of(int32_t out_type, const Product &x, hipStream_t st)
{
    return out_type == TT_F32 ? launch_product<T, float>(x, st) : launch_product<T, T>(x, st);
}

template <typename T>
int gradients_of(int32_t w_type, const Product &dx, const Product &dw, const BiasSum &b, hipStream_t st)
{
    return w_type == TT_F32 ? launch_gradients<T, float>(dx, dw, b, st) : launch_gradients<T, T>(dx, dw, b, st);
}

}  // namespace tt
