// C-ABI entry points of token embedding and dropout (declared in include/tt_emb.h): argument checks, workspace layout, kernel
// selection and launches.  Nothing here allocates device memory or waits for the stream.

#include "../../include/tt_emb.h"

#include "tt_rows_args.h"
#include "tt_token.h"

using namespace tt;

namespace {

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

template <typename S, typename D, int U, bool TOKENS, bool RESIDUAL>
void launch_rows(RowsArgs &a, hipStream_t st)
{
    const dim3 grid = grid_of(ceil_div(a.rows * a.nv, WG * U), WG);
    a.nv_d = (double)a.nv;
    a.inv_nv = 1.0 / a.nv_d;
    a.half_nv = 0.5 * a.inv_nv;
    with_whole(a.N, [&](auto whole) {
        hipLaunchKernelGGL((rows_kernel<S, D, U, decltype(whole)::value, TOKENS, RESIDUAL>), grid, dim3(WG), 0, st, a);
    });
}

constexpr int64_t MOST_COLUMNS = 1 << 20;                    // of the kernels whose second grid dimension runs over the columns

int check_columns(int64_t N)
{
    return N > MOST_COLUMNS ? fail(TT_ERR_UNSUPPORTED, "more than 2^20 columns") : TT_OK;
}

// ---- gradient of a token table ----

constexpr int64_t MOST_GRAD_TOKENS = 1ll << 28;              // (a workgroup per tile of sorted positions)

// Workgroups that clear (they take turns beyond that).  With less than MOST_ELEMENTS there are less than 2^32 parts to be cleared, and less
// than 2^23 + 2^21 workgroups that add, so that all of them fit a launch along x.
constexpr int64_t MOST_CLEAR = 1 << 22;

struct GradWs {
    uint32_t *k[2], *v[2], *hist, *total;
    uint8_t *named;
    float *part;
    size_t bytes;
};

// Entries per tile of sorted positions: as many as leave 4,096 waves some work, and at least 8 and at most 64 (then fewer sums of
// runs cross tiles).  16-bit gradients added to a 16-bit table, 8 / 16 / 32 / 64 entries: 2^21 vectors (16,384 tokens of 1,024 columns) 46 / 45 / 51 / 66 us,
// 2^22 (32,768 of 1,024) 61 / 54 / 56 / 69, 2^23 (65,536 of 1,024) 109 / 93 / 88 / 99, 2^24 (32,768 of 4,096) 175 / 151 / 139 / 141, 2^25 (65,536 of
// 4,096) 317 / 268 / 245 / 232.
constexpr int64_t GRAD_SHORT = 1 << 22;                      // vectors of the gradient up to which it is 8
int grad_entries(int64_t L, int64_t nv)
{
    if (L * nv < GRAD_SHORT) return 8;
    if (L * nv < 2 * GRAD_SHORT) return 16;
    return L * nv < 4 * GRAD_SHORT || nv <= 1 << TG_LEAST_LG ? 32 : 64;      // (the shortest rows: as many as a workgroup's LDS holds)
}
static_assert((WG >> TG_LEAST_LG) * 32 <= TG_MOST && (WG >> (TG_LEAST_LG + 1)) * 64 <= TG_MOST, "a workgroup's entries fit its LDS");

// The path without a sort, whose workgroups each look at all tokens: up to 4,096 of them.  16-bit gradients of 1,024 columns added to a
// table, sort / without: 30 tokens 13.6 / 4.2 us, 500 15.7 / 5.5, 1,000 16.5 / 8.1 (all of one token 17 / 27); of 4,096 columns,
// 500 tokens (4,000 workgroups) 16.2 / 13.7, 1,000 19.5 / 25.3.
bool few_tokens(int64_t L, int64_t nv) { return L <= TF_MOST && L * ceil_div(nv, WAVE) <= 4096; }

GradWs grad_ws(void *ws, int64_t L, int64_t num_rows, int64_t N)
{
    GradWs w;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = ws ? (char *)ws + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return p;
    };
    const int64_t sort_tiles = ceil_div(L, TS_TILE);
    const int64_t nv = ceil_div(N, 8);
    int64_t tiles = ceil_div(L, grad_entries(L, nv));
    const int64_t shorter = ceil_div(ceil_div(GRAD_SHORT, nv), 8);           // what a call below the limit needs at most
    if (L * nv >= GRAD_SHORT && tiles < shorter) tiles = shorter;
    for (int i = 0; i < 2; ++i) {
        w.k[i] = (uint32_t *)take((size_t)L * 4);
        w.v[i] = (uint32_t *)take((size_t)L * 4);
    }
    w.hist = (uint32_t *)take((size_t)sort_tiles * TS_BINS * 4);
    w.total = (uint32_t *)take(TS_BINS * 4);
    w.named = (uint8_t *)take((size_t)num_rows);
    w.part = (float *)take((size_t)tiles * 2 * (size_t)(8 * nv) * 4);
    w.bytes = at;
    return w;
}

// Rows up to which the first kernel of the sort, of one workgroup or of a few, clears their bytes itself.  By another kernel / itself, 16
// columns: 4,000 tokens (one workgroup), 2^17 rows 29.1 / 28.2 us, 2^18 30.4 / 30.5, 2^19 32.0 / 33.7; 16,384 tokens, 2^19 rows 46.9 / 45.3, 2^20 58.9 / 58.0,
// 2^22 78.1 / 79.2.
constexpr int64_t BLANK_ONE = 1 << 18, BLANK_FEW = 1 << 20;

hipError_t sort_tokens(const tt_tokens_t *t, int64_t num_rows, const GradWs &w, bool named, hipStream_t st, const uint32_t **ks, const uint32_t **vs)
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
    const int passes = (bits + TS_BITS - 1) / TS_BITS;
    s.bits = (bits + passes - 1) / passes;
    const bool one = t->L <= TO_MOST;
    if (named) {
        s.named = w.named;
        s.blank = num_rows <= (one ? BLANK_ONE : BLANK_FEW);
        if (!s.blank) hipLaunchKernelGGL(token_blank_kernel, dim3(1024), dim3(WG), 0, st, s);
    }
    if (one) {
        s.kout = w.k[0];
        s.vout = w.v[0];
        *ks = s.kout;
        *vs = s.vout;
        auto launch = [&](auto r) {
            constexpr int R = decltype(r)::value;
            static OncePerDevice once;
            const hipError_t e = allow_dynamic_lds(once, (const void *)token_sort_one_kernel<R>, sort_one_lds(R));
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL(token_sort_one_kernel<R>, dim3(1), dim3(TS_WG), sort_one_lds(R), st, s, passes);
            return hipGetLastError();
        };
        if (t->L <= TS_WG) return launch(std::integral_constant<int, 1>{});
        if (t->L <= 4 * TS_WG) return launch(std::integral_constant<int, 4>{});
        return launch(std::integral_constant<int, 8>{});
    }
    int at = 0;
    for (s.shift = 0; s.shift < bits; s.shift += s.bits, at ^= 1) {
        s.kout = w.k[at];
        s.vout = w.v[at];
        hipLaunchKernelGGL(token_hist_kernel, dim3(s.tiles), dim3(TS_WG), 0, st, s);
        s.blank = false;
        if (s.tiles > TS_SCAN_TILES) {
            hipLaunchKernelGGL(token_scan_kernel, dim3(TS_BINS / WAVE), dim3(TS_WG), 0, st, s);
            hipLaunchKernelGGL(token_scatter_kernel<true>, dim3(s.tiles), dim3(TS_WG), 0, st, s);
        } else {
            hipLaunchKernelGGL(token_scatter_kernel<false>, dim3(s.tiles), dim3(TS_WG), 0, st, s);
        }
        s.tokens = nullptr;
        s.named = nullptr;
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
    if ((rc = check_sizes(num_rows, N)) || (rc = check_sizes(L, N)) || (rc = check_columns(N))) return rc;
    if ((rc = check_rows(table, name, num_rows, N, OUT)) || (rc = check_rows(grad, "grad_output", L, N, IN))) return rc;
    if ((rc = check_dropout(dropout, &a.drop))) return rc;
    if (N == 0 || num_rows == 0 || (old && L == 0)) return TT_OK;
    const size_t need = tt_token_bwd_workspace_bytes(L, num_rows, N);
    if (need && (!workspace || workspace_bytes < need))
        return fail(TT_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    if ((uintptr_t)workspace & 15) return fail(TT_ERR_BAD_ARG, "workspace must be 16-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    const GradWs w = grad_ws(workspace, L, num_rows, N);
    a.g = grad->data;
    a.table = table->data;
    a.part = w.part;
    a.ld_g = grad->ld;
    a.ld_table = table->ld;
    a.n = L;
    a.num_rows = num_rows;
    a.N = (int)N;
    a.nv = (int)ceil_div(N, 8);
    a.entries = grad_entries(L, a.nv);
    a.tiles = (int)ceil_div(L, a.entries);
    a.factor = factor * a.drop.factor;
    a.old = old;
    const bool few = few_tokens(L, a.nv);
    int lg = lg_ceil(a.nv < WAVE ? a.nv : WAVE), lg_join = lg;
    if (!few && lg < TG_LEAST_LG) lg = TG_LEAST_LG;
    const unsigned chunks = (unsigned)ceil_div(a.nv, 1 << lg), join_chunks = (unsigned)ceil_div(a.nv, 1 << lg_join);
    const int64_t sum_blocks = (few ? L : ceil_div(a.tiles, WG >> lg)) * chunks;
    ClearArgs k{};
    int64_t clear_blocks = 0;
    if (!old) {
        const int64_t pieces = ceil_div(N * element_bytes(table->type), 32);
        k.named = w.named;
        k.lg = lg_ceil(pieces < WG ? pieces : WG);
        const int64_t along = ceil_div(pieces, 1 << k.lg), parts = ceil_div(num_rows, WG >> k.lg) * along;
        k.chunks = (uint32_t)along;
        k.parts = (uint32_t)parts;
        clear_blocks = ceil_div(parts, TZ_SWEEPS) < MOST_CLEAR ? ceil_div(parts, TZ_SWEEPS) : MOST_CLEAR;
    }
    if (!few) {
        const hipError_t e = sort_tokens(tokens, num_rows, w, !old, st, &a.ks, &a.vs);
        if (e != hipSuccess) return hip_fail(e, "token sort");
    }
    const dim3 grid((unsigned)(sum_blocks + clear_blocks));
    with_whole(N, [&](auto whole) {
        with_type(grad->type, [&](auto g) {
            with_type(table->type, [&](auto o) {
                using G = decltype(g);
                using O = decltype(o);
                constexpr bool WHOLE = decltype(whole)::value;
                if (few)
                    hipLaunchKernelGGL((token_few_kernel<G, O, WHOLE>), grid, dim3(WG), 0, st, a, tokens->data, (int)(tokens->bits == 64), lg, (int)chunks, (uint32_t)sum_blocks, k);
                else
                    hipLaunchKernelGGL((token_grad_kernel<G, O, WHOLE>), grid, dim3(WG), 0, st, a, lg, (int)chunks, (uint32_t)sum_blocks, k);
            });
        });
    });
    if (!few && a.tiles > 1)
        with_type(table->type, [&](auto o) { hipLaunchKernelGGL(token_join_kernel<decltype(o)>, dim3(a.tiles, join_chunks), dim3(WG), 0, st, a, lg_join); });
    return launched("token gradient launch");
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
    if ((rc = check_sizes(num_rows, N)) || (rc = check_sizes(L, N)) || (rc = check_columns(N))) return rc;
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
    a.scale = scale * a.drop.factor;
    if (num_rows == 0) {                                     // no token is one: rows of zeros, for which nothing has to be there to be read
        a.src = output->data;
        a.ld_src = 0;
        a.drop.state = nullptr;
    }
    with_type(num_rows ? table->type : output->type, [&](auto s) {
        with_type(output->type, [&](auto d) {
            // few tokens: one vector per thread, so that more of the device has some; else two (32,768 tokens of 4,096 columns in 16 bits
            // under dropout, 1 / 2 / 4 vectors: 97 / 75 / 77 us; 1 / 2, 2^20 vectors 5.7 / 5.9, under dropout 6.5 / 6.2, 2^21 9.9 / 9.9 and 10.4 / 9.9)
            if (L * a.nv < (1 << 20)) launch_rows<decltype(s), decltype(d), 1, true, false>(a, (hipStream_t)stream);
            else launch_rows<decltype(s), decltype(d), 2, true, false>(a, (hipStream_t)stream);
        });
    });
    return launched("token lookup launch");
}

size_t tt_token_bwd_workspace_bytes(int64_t L, int64_t num_rows, int64_t N)
{
    if (L <= 0 || few_tokens(L, ceil_div(N, 8)) || num_rows <= 0 || num_rows >= MOST_ROWS || N <= 0 || L >= MOST_GRAD_TOKENS || N > MOST_COLUMNS) return 0;
    return grad_ws(nullptr, L, num_rows, N).bytes;
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
    a.scale = a.drop.factor;
    with_type(x->type, [&](auto s) {
        if (residual) launch_rows<decltype(s), decltype(s), 1, false, true>(a, (hipStream_t)stream);
        else launch_rows<decltype(s), decltype(s), 1, false, false>(a, (hipStream_t)stream);
    });
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

}  // extern "C"
