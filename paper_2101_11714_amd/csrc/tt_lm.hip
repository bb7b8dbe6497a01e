// C-ABI entry points of the operators at a language model's way in (declared in include/tt_emb.h): token embedding, dropout,
// residual addition + RMS norm.  Argument checks, workspace layout, kernel selection and launches.  Nothing here allocates
// device memory or waits for the stream.

#include "../../include/tt_emb.h"

#include <type_traits>

#include "tt_error.h"
#include "tt_rms_norm.h"
#include "tt_token.h"

using namespace tt;

namespace {

constexpr int64_t MOST_ROWS = 1ll << 31;                     // rows and columns stay below (elements may be 2^62)

int element_bytes(int32_t type) { return type == TT_F32 ? 4 : type == TT_E4M3 ? 1 : 2; }

// calls f with a value of the C++ type of `type`
template <typename F>
void with_type(int32_t type, F f)
{
    if (type == TT_F32) f(float{});
    else if (type == TT_BF16) f(bf16_t{});
    else f(f16_t{});
}

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int lg_ceil(int64_t n)
{
    int lg = 0;
    while ((1ll << lg) < n) ++lg;
    return lg;
}

enum { IN, OUT };

// an array of n rows of N columns that the call reads (a row stride of 0 repeats one row) or writes
int check_rows(const tt_rows_t *a, const char *name, int64_t n, int64_t N, int way, bool bits8 = false)
{
    if (!a) return fail(TT_ERR_NULL, "%s is NULL", name);
    if (a->type != TT_F32 && a->type != TT_BF16 && a->type != TT_F16 && !(bits8 && a->type == TT_E4M3))
        return fail(TT_ERR_UNSUPPORTED, "%s: type %d is not supported here", name, (int)a->type);
    if (n == 0 || N == 0) return TT_OK;
    if (!a->data) return fail(TT_ERR_NULL, "%s is NULL", name);
    if ((uintptr_t)a->data % element_bytes(a->type)) return fail(TT_ERR_BAD_ARG, "%s is not aligned to its elements", name);
    if (n > 1 && (way == OUT ? a->ld < N : a->ld < 0)) return fail(TT_ERR_BAD_ARG, "%s: row stride %lld", name, (long long)a->ld);
    if (n > 1 && a->ld > (1ll << 31)) return fail(TT_ERR_UNSUPPORTED, "%s: row stride over 2^31", name);
    return TT_OK;
}

int check_sizes(int64_t rows, int64_t N)
{
    if (rows < 0 || N < 0) return fail(TT_ERR_BAD_ARG, "negative size");
    if (rows >= MOST_ROWS || N >= MOST_ROWS) return fail(TT_ERR_UNSUPPORTED, "2^31 rows or columns, or more");
    return TT_OK;
}

int check_dropout(const tt_dropout_t *d, DropArgs *out)
{
    *out = DropArgs{nullptr, 0u, 0u, 1.f};
    if (!d) return TT_OK;
    if (!(d->p >= 0.f && d->p <= 1.f)) return fail(TT_ERR_BAD_ARG, "dropout: p outside [0, 1]");
    const uint32_t q = (uint32_t)((double)d->p * 65536.0 + 0.5);
    if (q == 0) return TT_OK;                                // nothing is dropped
    if (!d->state) return fail(TT_ERR_NULL, "dropout: state is NULL");
    if ((uintptr_t)d->state % 8) return fail(TT_ERR_BAD_ARG, "dropout: state is not aligned");
    *out = DropArgs{d->state, d->site, q, q < 65536u ? (float)(65536.0 / (65536.0 - (double)q)) : 0.f};
    return TT_OK;
}

int check_tokens(const tt_tokens_t *t, int64_t *L)
{
    if (!t) return fail(TT_ERR_NULL, "tokens is NULL");
    if (t->bits != 32 && t->bits != 64) return fail(TT_ERR_BAD_ARG, "tokens of 32 or 64 bits are expected");
    if (t->L < 0) return fail(TT_ERR_BAD_ARG, "negative L");
    if (t->L >= MOST_ROWS) return fail(TT_ERR_UNSUPPORTED, "2^31 tokens or more");
    if (t->L > 0 && !t->data) return fail(TT_ERR_NULL, "tokens is NULL");
    if ((uintptr_t)t->data % (t->bits / 8)) return fail(TT_ERR_BAD_ARG, "tokens are not aligned");
    *L = t->L;
    return TT_OK;
}

int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : hip_fail(e, what);
}

// what a launch takes: less than 2^32 threads along x
int check_grid(int64_t workgroups, int threads)
{
    return workgroups * threads < (1ll << 32) ? TT_OK : fail(TT_ERR_UNSUPPORTED, "more rows than one launch takes");
}

int rows_lg(int nv) { return lg_ceil(nv < WG ? nv : WG); }

bool rows_four(const RowsArgs &a, int lg) { return a.rows * ceil_div(a.nv, 1 << lg) >= (int64_t)(WG >> lg) * 8192; }

// rows_kernel: a workgroup covers up to WG vectors of a row; several rows per thread where there are enough to fill the device
template <typename S, typename D>
void launch_rows(const RowsArgs &a, int lg, hipStream_t st)
{
    const int ty = WG >> lg;
    const int64_t chunks = ceil_div(a.nv, 1 << lg);
    if (rows_four(a, lg))
        hipLaunchKernelGGL((rows_kernel<S, D, 4>), dim3((unsigned)ceil_div(a.rows, ty * 4), (unsigned)chunks), dim3(WG), 0, st, a, lg);
    else
        hipLaunchKernelGGL((rows_kernel<S, D, 1>), dim3((unsigned)ceil_div(a.rows, ty), (unsigned)chunks), dim3(WG), 0, st, a, lg);
}

constexpr int64_t MOST_COLUMNS = 1 << 20;                    // of the kernels whose second grid dimension runs over the columns

int check_columns(int64_t N)
{
    return N > MOST_COLUMNS ? fail(TT_ERR_UNSUPPORTED, "more than 2^20 columns") : TT_OK;
}

// ---- gradient of a token table ----

constexpr int64_t MOST_GRAD_TOKENS = 1ll << 28;              // (a workgroup per tile of sorted positions)

struct GradWs {
    uint32_t *k[2], *v[2], *hist, *total;
    float *part;
    size_t bytes;
};

// entries per tile of sorted positions
int grad_entries(int64_t L) { return L < 16384 ? 8 : 32; }

GradWs grad_ws(void *ws, int64_t L, int64_t N)
{
    GradWs w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = ws ? (char *)ws + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return p;
    };
    const int64_t sort_tiles = ceil_div(L, TS_TILE);
    int64_t tiles = ceil_div(L, grad_entries(L));
    if (L >= 16384 && tiles < 2048) tiles = 2048;            // (what a shorter call needs at most)
    for (int i = 0; i < 2; ++i) {
        w.k[i] = (uint32_t *)take((size_t)L * 4);
        w.v[i] = (uint32_t *)take((size_t)L * 4);
    }
    w.hist = (uint32_t *)take((size_t)sort_tiles * TS_BINS * 4);
    w.total = (uint32_t *)take(TS_BINS * 4);
    w.part = (float *)take((size_t)tiles * 2 * (size_t)(8 * ceil_div(N, 8)) * 4);
    w.bytes = at;
    return w;
}

hipError_t sort_tokens(const tt_tokens_t *t, int64_t num_rows, const GradWs &w, hipStream_t st, const uint32_t **ks, const uint32_t **vs)
{
    SortPass s{};
    s.tokens = t->data;
    s.wide = t->bits == 64;
    s.n = t->L;
    s.num_rows = num_rows;
    s.tiles = (int)ceil_div(t->L, TS_TILE);
    s.hist = w.hist;
    s.total = w.total;
    int bits = 1;                                            // num_rows itself is the key of no token
    while (bits < 32 && (1ll << bits) <= num_rows) ++bits;
    int at = 0;
    for (s.shift = 0; s.shift < bits; s.shift += 9, at ^= 1) {
        s.kout = w.k[at];
        s.vout = w.v[at];
        hipLaunchKernelGGL(token_hist_kernel, dim3(s.tiles), dim3(TS_WG), 0, st, s);
        if (s.tiles > TS_SCAN_TILES) {
            hipLaunchKernelGGL(token_scan_kernel, dim3(TS_BINS / WAVE), dim3(TS_WG), 0, st, s);
            hipLaunchKernelGGL(token_scatter_kernel<true>, dim3(s.tiles), dim3(TS_WG), 0, st, s);
        } else {
            hipLaunchKernelGGL(token_scatter_kernel<false>, dim3(s.tiles), dim3(TS_WG), 0, st, s);
        }
        s.tokens = nullptr;
        s.kin = s.kout;
        s.vin = s.vout;
    }
    *ks = s.kin;
    *vs = s.vin;
    return hipGetLastError();
}

// the table's rows become old * row + factor * (sums of the gradient's rows)
int token_grad(const tt_tokens_t *tokens, const tt_rows_t *grad, const tt_dropout_t *dropout, const tt_rows_t *table, const char *name,
               int64_t num_rows, int64_t N, float factor, bool old, void *workspace, size_t workspace_bytes, void *stream)
{
    int64_t L;
    GradArgs a{};
    int rc = check_tokens(tokens, &L);
    if (rc) return rc;
    if (L >= MOST_GRAD_TOKENS) return fail(TT_ERR_UNSUPPORTED, "2^28 tokens or more");
    if ((rc = check_sizes(num_rows, N)) || (rc = check_columns(N))) return rc;
    if ((rc = check_rows(table, name, num_rows, N, OUT)) || (rc = check_rows(grad, "grad_output", L, N, IN))) return rc;
    if ((rc = check_dropout(dropout, &a.drop))) return rc;
    if (N == 0 || num_rows == 0 || (old && L == 0)) return TT_OK;
    const size_t need = tt_token_bwd_workspace_bytes(L, N);
    if (L > 0 && (!workspace || workspace_bytes < need))
        return fail(TT_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    if ((uintptr_t)workspace & 15) return fail(TT_ERR_BAD_ARG, "workspace must be 16-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    const GradWs w = grad_ws(workspace, L, N);
    a.g = grad->data;
    a.table = table->data;
    a.part = w.part;
    a.ld_g = grad->ld;
    a.ld_table = table->ld;
    a.n = L;
    a.num_rows = num_rows;
    a.N = (int)N;
    a.nv = (int)ceil_div(N, 8);
    a.entries = grad_entries(L);
    a.tiles = (int)ceil_div(L, a.entries);
    a.factor = factor;
    a.old = old;
    const int lg = lg_ceil(a.nv < WAVE ? a.nv : WAVE);
    const unsigned chunks = (unsigned)ceil_div(a.nv, 1 << lg);
    if (L > 0) {
        const hipError_t e = sort_tokens(tokens, num_rows, w, st, &a.ks, &a.vs);
        if (e != hipSuccess) return hip_fail(e, "token sort");
        with_type(grad->type, [&](auto g) {
            with_type(table->type, [&](auto o) {
                hipLaunchKernelGGL((token_grad_kernel<decltype(g), decltype(o)>), dim3((unsigned)ceil_div(a.tiles, WG >> lg), chunks), dim3(WG), 0, st, a, lg);
            });
        });
    }
    const int64_t blocks = ceil_div(num_rows, NWAVE * TZ_ROWS);
    const unsigned zero_grid = (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20);
    with_type(table->type, [&](auto o) {
        if (a.tiles > 1) hipLaunchKernelGGL(token_join_kernel<decltype(o)>, dim3(a.tiles, chunks), dim3(WG), 0, st, a, lg);
        if (!old) hipLaunchKernelGGL(token_zero_kernel<decltype(o)>, dim3(zero_grid), dim3(WG), 0, st, a, lg);
    });
    return launched("token gradient launch");
}

// ---- norm ----

struct NormShape {
    int lg, vpt, block;
};

// Threads per row and vectors per thread.
NormShape norm_shape(int64_t rows, int64_t nv, int least_lg)
{
    int lg = lg_ceil(nv);
    if (lg > 10) lg = 10;
    if (rows > 512) {                                        // enough rows: four vectors a thread, a wave's worth of threads at least
        const int four = lg_ceil(ceil_div(nv, 4));
        lg = four > 6 ? four : lg < 6 ? lg : 6;
    }
    if (lg < least_lg) lg = least_lg;
    int vpt = 1;
    while ((int64_t)vpt << lg < nv) vpt <<= 1;
    return {lg, vpt, lg > 8 ? 1024 : 256};
}

template <typename F>
void with_norm_shape(const NormShape &s, F f)
{
    auto block = [&](auto b) {
        if (s.vpt == 1) f(b, std::integral_constant<int, 1>{});
        else if (s.vpt == 2) f(b, std::integral_constant<int, 2>{});
        else f(b, std::integral_constant<int, 4>{});
    };
    if (s.block == 1024) block(std::integral_constant<int, 1024>{});
    else block(std::integral_constant<int, 256>{});
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

int norm_bwd_groups(const NormShape &s) { return s.block >> s.lg; }

constexpr int64_t NORM_BWD_WORKGROUPS = 1024;

int64_t norm_bwd_grid(int64_t rows, const NormShape &s)
{
    const int64_t all = ceil_div(rows, norm_bwd_groups(s));
    return all < NORM_BWD_WORKGROUPS ? all : NORM_BWD_WORKGROUPS;
}

}  // namespace

extern "C" {

int tt_token_fwd(const tt_rows_t *table, int64_t num_rows, int64_t N, const tt_tokens_t *tokens, float scale,
                 const tt_dropout_t *dropout, const tt_rows_t *output, void *stream)
{
    int64_t L;
    RowsArgs a{};
    int rc = check_tokens(tokens, &L);
    if (rc) return rc;
    if ((rc = check_sizes(num_rows, N)) || (rc = check_columns(N))) return rc;
    if ((rc = check_rows(table, "table", num_rows, N, IN)) || (rc = check_rows(output, "output", L, N, OUT))) return rc;
    if ((rc = check_dropout(dropout, &a.drop))) return rc;
    if (L == 0 || N == 0) return TT_OK;
    a.src = table->data;
    a.dst = output->data;
    a.tokens = tokens->data;
    a.ld_src = table->ld;
    a.ld_dst = output->ld;
    a.rows = L;
    a.num_rows = num_rows;
    a.N = (int)N;
    a.nv = (int)ceil_div(N, 8);
    a.wide = tokens->bits == 64;
    a.scale = scale;
    const int lg = rows_lg(a.nv);
    if ((rc = check_grid(ceil_div(L, (WG >> lg) * (rows_four(a, lg) ? 4 : 1)), WG))) return rc;
    with_type(table->type, [&](auto s) { with_type(output->type, [&](auto d) { launch_rows<decltype(s), decltype(d)>(a, lg, (hipStream_t)stream); }); });
    return launched("token lookup launch");
}

size_t tt_token_bwd_workspace_bytes(int64_t L, int64_t N)
{
    if (L <= 0 || N <= 0 || L >= MOST_GRAD_TOKENS || N > MOST_COLUMNS) return 0;
    return grad_ws(nullptr, L, N).bytes;
}

int tt_token_bwd(const tt_tokens_t *tokens, const tt_rows_t *grad_output, float scale, const tt_dropout_t *dropout,
                 const tt_rows_t *grad_table, int64_t num_rows, int64_t N, int accumulate,
                 void *workspace, size_t workspace_bytes, void *stream)
{
    return token_grad(tokens, grad_output, dropout, grad_table, "grad_table", num_rows, N, scale, accumulate != 0, workspace, workspace_bytes, stream);
}

int tt_token_bwd_sgd(const tt_tokens_t *tokens, const tt_rows_t *grad_output, float scale, const tt_dropout_t *dropout,
                     const tt_rows_t *table, int64_t num_rows, int64_t N, float lr,
                     void *workspace, size_t workspace_bytes, void *stream)
{
    return token_grad(tokens, grad_output, dropout, table, "table", num_rows, N, -lr * scale, true, workspace, workspace_bytes, stream);
}

static int dropout_rows(const tt_rows_t *x, const tt_rows_t *residual, const tt_dropout_t *dropout, const tt_rows_t *out,
                        const char *in_name, const char *out_name, int64_t rows, int64_t N, void *stream)
{
    RowsArgs a{};
    int rc = check_sizes(rows, N);
    if (rc) return rc;
    if ((rc = check_columns(N)) || (rc = check_rows(x, in_name, rows, N, IN)) || (rc = check_rows(out, out_name, rows, N, OUT))) return rc;
    if (residual && (rc = check_rows(residual, "residual", rows, N, IN))) return rc;
    if (out->type != x->type || (residual && residual->type != x->type)) return fail(TT_ERR_UNSUPPORTED, "arrays of one type are expected");
    if (!dropout) return fail(TT_ERR_NULL, "dropout is NULL");
    if ((rc = check_dropout(dropout, &a.drop))) return rc;
    if (rows == 0 || N == 0) return TT_OK;
    a.src = x->data;
    a.residual = residual ? residual->data : nullptr;
    a.dst = out->data;
    a.ld_src = x->ld;
    a.ld_res = residual ? residual->ld : 0;
    a.ld_dst = out->ld;
    a.rows = a.num_rows = rows;
    a.N = (int)N;
    a.nv = (int)ceil_div(N, 8);
    a.scale = 1.f;
    const int lg = rows_lg(a.nv);
    if ((rc = check_grid(ceil_div(rows, (WG >> lg) * (rows_four(a, lg) ? 4 : 1)), WG))) return rc;
    with_type(x->type, [&](auto s) { launch_rows<decltype(s), decltype(s)>(a, lg, (hipStream_t)stream); });
    return launched("dropout launch");
}

int tt_dropout_fwd(const tt_rows_t *x, const tt_rows_t *residual, const tt_dropout_t *dropout, const tt_rows_t *output,
                   int64_t n_rows, int64_t N, void *stream)
{
    return dropout_rows(x, residual, dropout, output, "x", "output", n_rows, N, stream);
}

int tt_dropout_bwd(const tt_rows_t *grad_output, const tt_dropout_t *dropout, const tt_rows_t *grad_x, int64_t n_rows, int64_t N, void *stream)
{
    return dropout_rows(grad_output, nullptr, dropout, grad_x, "grad_output", "grad_x", n_rows, N, stream);
}

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
    const NormShape s = norm_shape(n_rows, a.nv, group ? lg_ceil(group / 8) : 0);
    if ((rc = check_grid(ceil_div(n_rows, s.block >> s.lg), s.block))) return rc;
    with_types(x->type, stream_type, [&](auto t, auto h) {
        with_norm_shape(s, [&](auto block, auto vpt) {
            constexpr int BLOCK = decltype(block)::value, VPT = decltype(vpt)::value;
            const dim3 grid((unsigned)ceil_div(n_rows, BLOCK >> s.lg));
            if (bits8)
                hipLaunchKernelGGL((norm_fwd_kernel<decltype(t), decltype(h), true, VPT, BLOCK>), grid, dim3(BLOCK), 0, (hipStream_t)stream, a, s.lg);
            else
                hipLaunchKernelGGL((norm_fwd_kernel<decltype(t), decltype(h), false, VPT, BLOCK>), grid, dim3(BLOCK), 0, (hipStream_t)stream, a, s.lg);
        });
    });
    return launched("norm launch");
}

size_t tt_add_rms_norm_bwd_workspace_bytes(int64_t n_rows, int64_t N)
{
    if (n_rows <= 0 || N <= 0 || n_rows >= MOST_ROWS || N > RN_MOST) return 0;
    const int64_t most = n_rows < NORM_BWD_WORKGROUPS ? n_rows : NORM_BWD_WORKGROUPS;
    return (size_t)most * (size_t)(8 * ceil_div(N, 8)) * sizeof(float);
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
    a.part = grad_weight ? (float *)workspace : nullptr;
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
        const NormShape s = norm_shape(n_rows, a.nv, 0);
        grid = norm_bwd_grid(n_rows, s);
        const size_t lds = grad_weight ? (size_t)(norm_bwd_groups(s) - 1) * 8 * a.nv * sizeof(float) : 0;
        with_types(grad_output->type, h->type, [&](auto t, auto ht) {
            with_norm_shape(s, [&](auto block, auto vpt) {
                constexpr int BLOCK = decltype(block)::value, VPT = decltype(vpt)::value;
                hipLaunchKernelGGL((norm_bwd_kernel<decltype(t), decltype(ht), VPT, BLOCK>), dim3((unsigned)grid), dim3(BLOCK), lds, st, a, s.lg);
            });
        });
    }
    if (grad_weight)
        with_type(grad_weight_type, [&](auto w) {
            hipLaunchKernelGGL(norm_dw_kernel<decltype(w)>, dim3((unsigned)ceil_div(N, 64)), dim3(1024), 0, st, (const float *)workspace, (int)grid, (int)N, a.nv,
                               (decltype(w) *)grad_weight, accumulate);
        });
    return launched("norm gradient launch");
}

}  // extern "C"
