// C-ABI entry points of the log probabilities of tokens (declared in include/tt_emb.h): argument checks, workspace layout, kernel
// selection and launches.  Nothing here allocates device memory or waits for the stream.

#include "../../include/tt_emb.h"

#include "tt_rows_args.h"
#include "tt_logprob.h"

using namespace tt;

namespace {

constexpr int64_t MOST_VOCAB = 1ll << 30;

// How a row is cut: into pieces enough for 512 workgroups, of 512 vectors at least, whose alternatives one workgroup can rank.
struct Pieces {
    int n, size;
};

Pieces pieces_of(int64_t rows, int64_t V, int32_t k)
{
    const int64_t nv = ceil_div(V, 8);
    int64_t n = rows > 0 ? ceil_div(512, rows) : 1;
    if (n > ceil_div(nv, 512)) n = ceil_div(nv, 512);
    if (k > 0 && n > LP_LIST / k) n = LP_LIST / k;
    if (n < 1) n = 1;
    const int64_t size = ceil_div(nv, n);
    return {(int)ceil_div(nv, size), (int)size};
}

size_t sums_bytes(int64_t rows, const Pieces &p) { return p.n > 1 ? (size_t)rows * (size_t)p.n * 4 * sizeof(float) : 0; }
size_t keys_bytes(int64_t rows, const Pieces &p, int32_t k) { return p.n > 1 ? (size_t)rows * (size_t)p.n * (size_t)k * sizeof(uint64_t) : 0; }

int check_logits(int64_t rows, int64_t V)
{
    int rc = check_sizes(rows, V);
    if (rc) return rc;
    if (V > MOST_VOCAB) return fail(TT_ERR_UNSUPPORTED, "more than 2^30 columns");
    if (V == 0 && rows > 0) return fail(TT_ERR_BAD_ARG, "rows without columns");
    return TT_OK;
}

int check_tokens(const tt_tokens_t *t, int64_t rows)
{
    if (!t) return fail(TT_ERR_NULL, "tokens is NULL");
    if (t->L != rows) return fail(TT_ERR_BAD_SHAPE, "%lld tokens for %lld rows", (long long)t->L, (long long)rows);
    if (t->bits != 32 && t->bits != 64) return fail(TT_ERR_BAD_ARG, "tokens of %d bits", (int)t->bits);
    if (rows > 0 && !t->data) return fail(TT_ERR_NULL, "tokens is NULL");
    return (uintptr_t)t->data % (t->bits / 8) ? fail(TT_ERR_BAD_ARG, "tokens are not aligned") : TT_OK;
}

int check_floats(const float *p, const char *name) { return (uintptr_t)p % 4 ? fail(TT_ERR_BAD_ARG, "%s is not aligned", name) : TT_OK; }

int check_scale(float scale)
{
    // (with less, logits whose difference 32 bits do not hold could both have a probability)
    return scale >= 1e-36f && scale <= 1e30f ? TT_OK : fail(TT_ERR_BAD_ARG, "scale must be 1e-36 at least, and 1e30 at most");
}

}  // namespace

extern "C" {

size_t tt_token_logprob_fwd_workspace_bytes(int64_t n_rows, int64_t V, int32_t k)
{
    if (n_rows <= 0 || V <= 0 || check_logits(n_rows, V) || k < 0 || k > LP_MOST_K) return 0;
    // (rows times pieces is at most 512 + rows while there are pieces, that is up to 511 rows)
    const int64_t most = ceil_div(ceil_div(V, 8), 512) > 1 ? 1024 : 0;
    return (size_t)(most < n_rows * 512 ? most : n_rows * 512) * (4 * sizeof(float) + (size_t)k * sizeof(uint64_t));
}

int tt_token_logprob_fwd(const tt_rows_t *logits, const tt_tokens_t *tokens, float scale, float *logprob, float *lse, float *entropy,
                         int32_t k, void *top_ids, int32_t top_ids_bits, float *top_logprobs, int64_t n_rows, int64_t V,
                         void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_logits(n_rows, V);
    if (rc || (rc = check_rows(logits, "logits", n_rows, V, IN)) || (rc = check_scale(scale))) return rc;
    if ((logprob || tokens) && (rc = check_tokens(tokens, n_rows))) return rc;
    if (k < 0 || k > LP_MOST_K) return fail(TT_ERR_UNSUPPORTED, "0 to %d alternatives", LP_MOST_K);
    if (k > 0 && n_rows > 0 && !top_ids) return fail(TT_ERR_NULL, "top_ids is NULL");
    if (k > 0 && top_ids_bits != 32 && top_ids_bits != 64) return fail(TT_ERR_BAD_ARG, "top_ids of %d bits", (int)top_ids_bits);
    if (k > 0 && (uintptr_t)top_ids % (top_ids_bits / 8)) return fail(TT_ERR_BAD_ARG, "top_ids is not aligned");
    if ((rc = check_floats(logprob, "logprob")) || (rc = check_floats(lse, "lse")) || (rc = check_floats(entropy, "entropy")) || (rc = check_floats(top_logprobs, "top_logprobs"))) return rc;
    if (n_rows == 0) return TT_OK;
    const Pieces p = pieces_of(n_rows, V, k);
    const size_t sums = sums_bytes(n_rows, p), need = sums + keys_bytes(n_rows, p, k);
    if (need && (!workspace || workspace_bytes < need)) return fail(TT_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    if ((uintptr_t)workspace & 15) return fail(TT_ERR_BAD_ARG, "workspace must be 16-byte aligned");
    LogprobArgs a{};
    a.logits = logits->data;
    a.ld = logits->ld;
    a.tokens = tokens ? tokens->data : nullptr;
    a.tokens64 = tokens && tokens->bits == 64;
    a.scale = scale;
    a.logprob = logprob;
    a.lse = lse;
    a.entropy = entropy;
    a.k = k;
    a.ids = top_ids;
    a.ids64 = top_ids_bits == 64;
    a.top = top_logprobs;
    a.rows = n_rows;
    a.V = (int)V;
    a.nv = (int)ceil_div(V, 8);
    a.pieces = p.n;
    a.piece = p.size;
    a.sums = (float *)workspace;
    a.keys = (uint64_t *)((char *)workspace + sums);
    with_type(logits->type, [&](auto t) {
        typedef decltype(t) T;
        with_whole(V, [&](auto w) {
            constexpr bool WHOLE = decltype(w)::value;
            const dim3 grid = grid_of(n_rows * p.n, WG);
            if (k > 0) {
                hipLaunchKernelGGL((logprob_kernel<T, true, true, WHOLE>), grid, dim3(WG), 0, (hipStream_t)stream, a);
            } else {
                with_flag(entropy != nullptr, [&](auto h) {
                    hipLaunchKernelGGL((logprob_kernel<T, false, decltype(h)::value, WHOLE>), grid, dim3(WG), 0, (hipStream_t)stream, a);
                });
            }
        });
        if (p.n > 1 && k > 0) hipLaunchKernelGGL((logprob_join_kernel<T, true>), grid_of(n_rows, LP_JOIN), dim3(LP_JOIN), 0, (hipStream_t)stream, a);
        else if (p.n > 1) hipLaunchKernelGGL((logprob_join_kernel<T, false>), grid_of(n_rows, WAVE), dim3(WAVE), 0, (hipStream_t)stream, a);
    });
    return launched("log probability launch");
}

int tt_token_logprob_bwd(const tt_rows_t *logits, const tt_tokens_t *tokens, float scale, const float *lse, const float *entropy,
                         const float *grad_logprob, const float *grad_entropy, const tt_rows_t *grad_logits, int64_t n_rows, int64_t V, void *stream)
{
    int rc = check_logits(n_rows, V);
    if (rc || (rc = check_rows(logits, "logits", n_rows, V, IN)) || (rc = check_rows(grad_logits, "grad_logits", n_rows, V, OUT)) || (rc = check_scale(scale))) return rc;
    if (grad_logits->type != logits->type) return fail(TT_ERR_UNSUPPORTED, "grad_logits has the logits' type");
    if ((grad_logprob || tokens) && (rc = check_tokens(tokens, n_rows))) return rc;
    if (n_rows > 0 && !lse) return fail(TT_ERR_NULL, "lse is NULL");
    if (n_rows > 0 && grad_entropy && !entropy) return fail(TT_ERR_NULL, "entropy is NULL");
    if ((rc = check_floats(lse, "lse")) || (rc = check_floats(entropy, "entropy")) || (rc = check_floats(grad_logprob, "grad_logprob")) || (rc = check_floats(grad_entropy, "grad_entropy"))) return rc;
    if (n_rows == 0) return TT_OK;
    LogprobGradArgs a{};
    a.logits = logits->data;
    a.tokens = tokens ? tokens->data : nullptr;
    a.out = grad_logits->data;
    a.ld = logits->ld;
    a.ld_out = grad_logits->ld;
    a.lse = lse;
    a.entropy = entropy;
    a.g = grad_logprob;
    a.ge = grad_entropy;
    a.rows = n_rows;
    a.tokens64 = tokens && tokens->bits == 64;
    a.V = (int)V;
    a.nv = (int)ceil_div(V, 8);
    a.pieces = (int)ceil_div(a.nv, WG * LP_UNROLL);
    a.piece = WG * LP_UNROLL;
    a.scale = scale;
    with_type(logits->type, [&](auto t) {
        with_whole(V, [&](auto whole) {
            hipLaunchKernelGGL((logprob_bwd_kernel<decltype(t), decltype(whole)::value>), grid_of(n_rows * a.pieces, WG), dim3(WG), 0, (hipStream_t)stream, a);
        });
    });
    return launched("log probability gradient launch");
}

}  // extern "C"
