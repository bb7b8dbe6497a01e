// C-ABI entry points of the residual addition + RMS norm (declared in include/tt_emb.h): argument checks, workspace layout, kernel
// selection and launches.  Nothing here allocates device memory or waits for the stream.

#include "../../include/tt_emb.h"

#include "tt_rows_args.h"
#include "tt_rms_norm.h"

using namespace tt;

namespace {

struct NormShape {
    int lg, vpt;
};

// Threads per row (log) and vectors per thread.
NormShape norm_shape(int lg, int64_t nv)
{
    int vpt = 1;
    while ((int64_t)vpt << lg < nv) vpt <<= 1;
    return {lg, vpt};
}

// Few rows: as many threads as vectors, so that the call ends soon.  Enough rows: two vectors a thread, a wave's worth of threads
// at least (rows of 4,096, 16 bits, four vectors: 85 us instead of 81).  One / two, 16 bits: 512 rows of 4,096 columns 4.1 / 4.2 us, of 8,192 7.6 / 7.8;
// 1,024 rows 7.5 / 7.7 and 12.6 / 11.0; 2,048 rows 12.0 / 10.9 and 21.7 / 21.5.
NormShape norm_fwd_shape(int64_t rows, int64_t nv, int least_lg)
{
    int lg = lg_ceil(nv);
    if (rows > 512) {
        const int two = lg_ceil(ceil_div(nv, 2));
        lg = two > 6 ? two : lg < 6 ? lg : 6;
    }
    if (lg > 10) lg = 10;
    return norm_shape(lg < least_lg ? least_lg : lg, nv);
}

constexpr int64_t NORM_BWD_WORKGROUPS = 256;
// Rows that give so many workgroups work are left to one, whose sums are the weight's gradient: one launch instead of two (two rows of
// 4,096 columns 7.9 -> 6.0 us, three 8.5 -> 6.9, 128 of 64 7.9 -> 5.4; not three of 16,000: 13.8 -> 15.5).
constexpr int64_t NORM_BWD_ALONE = 3;

NormShape norm_bwd_shape(int64_t nv)
{
    const int lg = lg_ceil(nv), most = lg_ceil(RN_BWD_THREADS);
    return norm_shape(lg < most ? lg : most, nv);
}

int64_t norm_bwd_grid(int64_t rows, int64_t nv)
{
    const NormShape s = norm_bwd_shape(nv);
    const int64_t all = ceil_div(rows, RN_BWD_THREADS >> s.lg);
    if (all <= NORM_BWD_ALONE && s.vpt <= 2) return 1;
    return all < NORM_BWD_WORKGROUPS ? all : NORM_BWD_WORKGROUPS;
}

template <typename F>
void with_vpt(int vpt, F f)
{
    if (vpt == 1) f(std::integral_constant<int, 1>{});
    else if (vpt == 2) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 4>{});
}

// (activation, residual stream): the same type, or a stream of 32 bits
template <typename F>
void with_types(int32_t type, int32_t stream, F f)
{
    with_type(type, [&](auto t) {
        if (stream == TT_F32) f(t, float{});
        else f(t, t);
    });
}

int check_norm(int64_t rows, int64_t N)
{
    int rc = check_sizes(rows, N);
    if (rc) return rc;
    if (N > RN_MOST) return fail(TT_ERR_UNSUPPORTED, "more than %d columns", RN_MOST);
    if (N == 0 && rows > 0) return fail(TT_ERR_BAD_ARG, "rows without columns have no mean square");
    return TT_OK;
}

int check_weight(const void *weight, int32_t type)
{
    if (!weight) return TT_OK;
    if (type != TT_F32 && type != TT_BF16 && type != TT_F16) return fail(TT_ERR_UNSUPPORTED, "weight: type %d is not supported", (int)type);
    return (uintptr_t)weight % element_bytes(type) ? fail(TT_ERR_BAD_ARG, "weight is not aligned to its elements") : TT_OK;
}

}  // namespace

extern "C" {

int tt_add_rms_norm_fwd(const tt_rows_t *x, const tt_rows_t *residual, const tt_dropout_t *dropout, const void *weight, int32_t weight_type,
                        float eps, const tt_rows_t *sum, const tt_rows_t *output, float *rstd, const tt_rows_t *scales, int32_t group,
                        int64_t n_rows, int64_t N, void *stream)
{
    NormArgs a{};
    int rc = check_norm(n_rows, N);
    if (rc) return rc;
    if ((rc = check_rows(x, "x", n_rows, N, IN)) || (rc = check_rows(output, "output", n_rows, N, OUT, true)) || (rc = check_weight(weight, weight_type))) return rc;
    if (residual && (rc = check_rows(residual, "residual", n_rows, N, IN))) return rc;
    if (sum && (rc = check_rows(sum, "sum", n_rows, N, OUT))) return rc;
    const int32_t stream_type = residual ? residual->type : sum ? sum->type : x->type;
    if (stream_type != x->type && stream_type != TT_F32) return fail(TT_ERR_UNSUPPORTED, "the residual has x's type or 32 bits");
    if (sum && sum->type != stream_type) return fail(TT_ERR_UNSUPPORTED, "sum has the residual's type");
    const bool bits8 = output->type == TT_E4M3;
    if (!bits8 && output->type != x->type) return fail(TT_ERR_UNSUPPORTED, "output has x's type or 8 bits");
    if (!(eps >= 0.f)) return fail(TT_ERR_BAD_ARG, "eps must not be negative");
    if (bits8) {
        if (group != 0 && group != 32 && group != 64 && group != 128) return fail(TT_ERR_UNSUPPORTED, "groups of 32, 64 or 128 columns, or 0");
        if ((rc = check_rows(scales, "scales", n_rows, group ? ceil_div(N, group) : 1, OUT))) return rc;
        if (scales->type != TT_F32) return fail(TT_ERR_UNSUPPORTED, "scales have 32 bits");
    } else if (scales || group) {
        return fail(TT_ERR_BAD_ARG, "scales and groups belong to an output in 8 bits");
    }
    if ((uintptr_t)rstd % 4) return fail(TT_ERR_BAD_ARG, "rstd is not aligned");
    if ((rc = check_dropout(dropout, &a.drop))) return rc;
    if (n_rows == 0) return TT_OK;
    a.x = x->data;
    a.residual = residual ? residual->data : nullptr;
    a.weight = weight;
    a.weight_type = weight_type;
    a.sum = sum ? sum->data : nullptr;
    a.y = output->data;
    a.rstd = rstd;
    a.scales = bits8 ? (float *)scales->data : nullptr;
    a.ld_x = x->ld;
    a.ld_res = residual ? residual->ld : 0;
    a.ld_sum = sum ? sum->ld : 0;
    a.ld_y = output->ld;
    a.ld_scales = bits8 ? scales->ld : 0;
    a.rows = n_rows;
    a.N = (int)N;
    a.nv = (int)ceil_div(N, 8);
    a.group = group;
    a.eps = eps;
    const NormShape s = norm_fwd_shape(n_rows, a.nv, group ? lg_ceil(group / 8) : 0);
    const int threads = s.lg > 8 ? 1 << s.lg : WG;
    const dim3 grid = grid_of(ceil_div(n_rows, threads >> s.lg), threads);
    with_types(x->type, stream_type, [&](auto t, auto h) {
        with_vpt(s.vpt, [&](auto vpt) {
            with_whole(N, [&](auto whole) {
                with_flag(residual != nullptr, [&](auto res) {
                    with_flag(bits8, [&](auto y8) {
                        hipLaunchKernelGGL((norm_fwd_kernel<decltype(t), decltype(h), decltype(y8)::value, decltype(vpt)::value, decltype(whole)::value, decltype(res)::value>), grid,
                                           dim3(threads), 0, (hipStream_t)stream, a, s.lg);
                    });
                });
            });
        });
    });
    return launched("norm launch");
}

size_t tt_add_rms_norm_bwd_workspace_bytes(int64_t n_rows, int64_t N)
{
    if (n_rows <= 0 || N <= 0 || n_rows >= MOST_ROWS || N > RN_MOST) return 0;
    const int64_t nv = ceil_div(N, 8), grid = norm_bwd_grid(n_rows, nv);
    return grid > 1 ? (size_t)grid * (size_t)(8 * nv) * sizeof(float) : 0;
}

int tt_add_rms_norm_bwd(const tt_rows_t *grad_output, const tt_rows_t *h, const float *rstd, const void *weight, int32_t weight_type,
                        const tt_rows_t *grad_sum, const tt_dropout_t *dropout, const tt_rows_t *grad_x, const tt_rows_t *grad_residual,
                        void *grad_weight, int32_t grad_weight_type, int accumulate, int64_t n_rows, int64_t N,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    NormGradArgs a{};
    int rc = check_norm(n_rows, N);
    if (rc) return rc;
    if ((rc = check_rows(grad_output, "grad_output", n_rows, N, IN)) || (rc = check_rows(h, "h", n_rows, N, IN)) || (rc = check_weight(weight, weight_type))) return rc;
    if (h->type != grad_output->type && h->type != TT_F32) return fail(TT_ERR_UNSUPPORTED, "h has grad_output's type or 32 bits");
    if (grad_sum && (rc = check_rows(grad_sum, "grad_sum", n_rows, N, IN))) return rc;
    if (grad_x && (rc = check_rows(grad_x, "grad_x", n_rows, N, OUT))) return rc;
    if (grad_residual && (rc = check_rows(grad_residual, "grad_residual", n_rows, N, OUT))) return rc;
    if ((grad_sum && grad_sum->type != h->type) || (grad_residual && grad_residual->type != h->type))
        return fail(TT_ERR_UNSUPPORTED, "grad_sum and grad_residual have h's type");
    if (grad_x && grad_x->type != grad_output->type) return fail(TT_ERR_UNSUPPORTED, "grad_x has grad_output's type");
    if (grad_weight && (rc = check_weight(grad_weight, grad_weight_type))) return rc;
    if (n_rows > 0 && !rstd) return fail(TT_ERR_NULL, "rstd is NULL");
    if ((uintptr_t)rstd % 4) return fail(TT_ERR_BAD_ARG, "rstd is not aligned");
    if ((rc = check_dropout(dropout, &a.drop))) return rc;
    if (N == 0 || (n_rows == 0 && (!grad_weight || accumulate))) return TT_OK;
    if (n_rows > 0 && !grad_weight && !grad_x && !grad_residual) return TT_OK;
    const size_t need = grad_weight ? tt_add_rms_norm_bwd_workspace_bytes(n_rows, N) : 0;
    if (need && (!workspace || workspace_bytes < need)) return fail(TT_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    if ((uintptr_t)workspace & 15) return fail(TT_ERR_BAD_ARG, "workspace must be 16-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    a.dy = grad_output->data;
    a.h = h->data;
    a.weight = weight;
    a.weight_type = weight_type;
    a.dsum = grad_sum ? grad_sum->data : nullptr;
    a.rstd = rstd;
    a.dx = grad_x ? grad_x->data : nullptr;
    a.dres = grad_residual ? grad_residual->data : nullptr;
    a.dw_type = grad_weight_type;
    a.add = accumulate != 0;
    a.ld_dy = grad_output->ld;
    a.ld_h = h->ld;
    a.ld_dsum = grad_sum ? grad_sum->ld : 0;
    a.ld_dx = grad_x ? grad_x->ld : 0;
    a.ld_dres = grad_residual ? grad_residual->ld : 0;
    a.rows = n_rows;
    a.N = (int)N;
    a.nv = (int)ceil_div(N, 8);
    a.weight_type = weight_type;
    int64_t grid = 0;
    if (n_rows > 0) {
        const NormShape s = norm_bwd_shape(a.nv);
        const int threads = RN_BWD_THREADS, groups = threads >> s.lg, parts = s.lg < 6 ? threads / WAVE : groups;
        grid = norm_bwd_grid(n_rows, a.nv);
        if (grid > 1) a.part = grad_weight ? (float *)workspace : nullptr;
        else a.dw = grad_weight;
        const size_t lds = grad_weight && parts > 1 ? (size_t)parts * 8 * a.nv * sizeof(float) : 0;
        with_types(grad_output->type, h->type, [&](auto t, auto ht) {
            auto launch = [&](auto vpt) {
                with_whole(N, [&](auto whole) {
                    with_flag(grad_sum != nullptr, [&](auto dsum) {
                        hipLaunchKernelGGL((norm_bwd_kernel<decltype(t), decltype(ht), decltype(vpt)::value, decltype(whole)::value, decltype(dsum)::value>),
                                           dim3((unsigned)grid), dim3(threads), lds, st, a, s.lg);
                    });
                });
            };
            if (s.vpt > 4) launch(std::integral_constant<int, 8>{});
            else with_vpt(s.vpt, launch);
        });
    }
    if (grad_weight && !a.dw)
        with_type(grad_weight_type, [&](auto w) {
            hipLaunchKernelGGL(norm_dw_kernel<decltype(w)>, dim3((unsigned)ceil_div(N, 64)), dim3(1024), 0, st, (const float *)workspace, (int)grid, (int)N, a.nv,
                               (decltype(w) *)grad_weight, accumulate);
        });
    return launched("norm gradient launch");
}

}  // extern "C"
