// C-ABI entry points of the norm and rotation of queries and keys (declared in include/tt_emb.h): argument checks, workspace layout, kernel
// selection and launches.  Nothing here allocates device memory or waits for the stream.

#include "../../include/tt_emb.h"

#include "tt_rows_args.h"
#include "tt_rotate.h"

using namespace tt;

namespace {

constexpr int MOST_HEAD = 512;                               // columns of a head: 34 units at most, whatever its pairs
constexpr int64_t BWD_WORKGROUPS = 512;

int check_heads(const tt_heads_t *h, const char *name, int64_t rows, int64_t D, int32_t type, int32_t heads, int way)
{
    if (!h) return fail(TT_ERR_NULL, "%s is NULL", name);
    if (h->type != TT_F32 && h->type != TT_BF16 && h->type != TT_F16) return fail(TT_ERR_UNSUPPORTED, "%s: type %d is not supported here", name, (int)h->type);
    if (h->type != type) return fail(TT_ERR_UNSUPPORTED, "%s has another type than the others", name);
    if (h->heads < 0) return fail(TT_ERR_BAD_ARG, "%s: negative number of heads", name);
    if (h->heads != heads) return fail(TT_ERR_BAD_SHAPE, "%s has another number of heads", name);
    if (rows == 0 || D == 0 || heads == 0) return TT_OK;
    if (!h->data) return fail(TT_ERR_NULL, "%s is NULL", name);
    if ((uintptr_t)h->data % element_bytes(h->type)) return fail(TT_ERR_BAD_ARG, "%s is not aligned to its elements", name);
    if (h->ld < 0 || h->ld_head < 0) return fail(TT_ERR_BAD_ARG, "%s: negative stride", name);
    if (h->ld > (1ll << 31) || h->ld_head > (1ll << 31)) return fail(TT_ERR_UNSUPPORTED, "%s: stride over 2^31", name);
    if (way == IN) return TT_OK;
    // heads of an output may not overlap: heads within rows, or rows within heads
    const bool one_head = heads == 1, one_row = rows == 1;
    const bool inner = (one_head || h->ld_head >= D) && (one_row || h->ld >= (one_head ? D : (heads - 1) * h->ld_head + D));
    const bool outer = (one_row || h->ld >= D) && (one_head || h->ld_head >= (one_row ? D : (rows - 1) * h->ld + D));
    return inner || outer ? TT_OK : fail(TT_ERR_BAD_ARG, "%s: its heads overlap", name);
}

int check_weight(const void *w, const char *name, int32_t type)
{
    if (!w) return TT_OK;
    if (type != TT_F32 && type != TT_BF16 && type != TT_F16) return fail(TT_ERR_UNSUPPORTED, "%s: type %d is not supported", name, (int)type);
    return (uintptr_t)w % element_bytes(type) ? fail(TT_ERR_BAD_ARG, "%s is not aligned to its elements", name) : TT_OK;
}

int check_rotation(const tt_rotation_t *t, int64_t rows, int64_t D, RotateArgs *a)
{
    a->pairs = 0;
    a->ends[0] = a->ends[1] = a->ends[2] = a->ends[3] = 0;
    if (!t) return TT_OK;
    if (t->axes < 1 || t->axes > 4) return fail(TT_ERR_BAD_ARG, "rotation: %d axes", (int)t->axes);
    if (t->bits != 32 && t->bits != 64) return fail(TT_ERR_BAD_ARG, "rotation: positions of %d bits", (int)t->bits);
    if (t->pairs < 0 || 2ll * t->pairs > D) return fail(TT_ERR_BAD_ARG, "rotation: %d pairs of %lld columns", (int)t->pairs, (long long)D);
    int64_t end = 0;
    for (int i = 0; i < 4; ++i) {
        if (i < t->axes) {
            if (t->sections[i] < 0) return fail(TT_ERR_BAD_ARG, "rotation: a negative section");
            end += t->sections[i];
        }
        a->ends[i] = (int)(end < t->pairs ? end : t->pairs);
    }
    if (end != t->pairs) return fail(TT_ERR_BAD_ARG, "rotation: sections of %lld pairs, not of %d", (long long)end, (int)t->pairs);
    if (t->pairs == 0 || rows == 0) return TT_OK;
    if (!t->positions || !t->freqs) return fail(TT_ERR_NULL, "rotation: positions or freqs is NULL");
    if ((uintptr_t)t->positions % (t->bits / 8) || (uintptr_t)t->freqs % 4) return fail(TT_ERR_BAD_ARG, "rotation: positions or freqs are not aligned");
    if (t->ld_positions < 0) return fail(TT_ERR_BAD_ARG, "rotation: negative stride");
    a->positions = t->positions;
    a->ld_positions = t->ld_positions;
    a->freqs = t->freqs;
    a->positions64 = t->bits == 64;
    a->pairs = t->pairs;
    a->neighbours = t->neighbours != 0;
    return TT_OK;
}

int check_sizes_of(int64_t rows, int64_t D, int64_t heads)
{
    if (rows < 0 || D < 0) return fail(TT_ERR_BAD_ARG, "negative size");
    if (D > MOST_HEAD) return fail(TT_ERR_UNSUPPORTED, "heads of more than %d columns", MOST_HEAD);
    if (heads > (1 << 20)) return fail(TT_ERR_UNSUPPORTED, "more than 2^20 heads");
    if (rows >= MOST_ROWS || rows * D * (heads > 0 ? heads : 1) >= MOST_ELEMENTS) return fail(TT_ERR_UNSUPPORTED, "2^31 rows or 2^40 elements, or more");
    return TT_OK;
}

void shape_of(RotateArgs &a)
{
    a.turned = (int)ceil_div(a.pairs, 8);
    a.units = a.turned + (int)ceil_div(a.D - 2 * a.pairs, 16);
    a.lg = lg_ceil(a.units);
}

// Heads of a group: up to eight, which then share its cosines and sines, where that leaves every compute unit 16 waves.
void slices_of(RotateArgs &a)
{
    const int64_t wanted = 256 * 16 * (WAVE >> a.lg), heads = a.rows * ((int64_t)a.q_heads + a.k_heads);
    int64_t each = heads / wanted;
    a.each = each < 1 ? 1 : each > 8 ? 8 : (int)each;
    a.q_slices = (int)ceil_div(a.q_heads, a.each);
    a.k_slices = (int)ceil_div(a.k_heads, a.each);
}

// Workgroups of the backward pass: no more than have heads to take, BWD_WORKGROUPS shared out by the numbers of heads.
int64_t bwd_workgroups(const RotateArgs &a, bool keys)
{
    const int64_t heads = keys ? a.k_heads : a.q_heads, items = a.rows * (keys ? a.k_slices : a.q_slices);
    const int64_t most = BWD_WORKGROUPS * heads / ((int64_t)a.q_heads + a.k_heads), all = ceil_div(items, WG >> a.lg);
    return all < most || most < 1 ? (most < 1 && all > 1 ? 1 : all) : most;
}

template <typename F>
void with_shape(const RotateArgs &a, bool norm, F f)
{
    with_flag(norm, [&](auto nm) {
        with_flag(a.pairs % (a.neighbours ? 4 : 8) == 0 && (a.D - 2 * a.pairs) % 8 == 0, [&](auto whole) { with_flag(a.neighbours != 0, [&](auto nb) { f(nm, whole, nb); }); });
    });
}

Heads of(const tt_heads_t *h) { return h ? Heads{h->data, h->ld, h->ld_head} : Heads{}; }

}  // namespace

extern "C" {

int tt_qk_norm_rotate_fwd(const tt_heads_t *q, const tt_heads_t *k, const tt_rotation_t *rotation, int norm, float eps,
                          const void *q_weight, int32_t q_weight_type, const void *k_weight, int32_t k_weight_type,
                          const tt_heads_t *q_output, const tt_heads_t *k_output, int64_t n_rows, int64_t D, void *stream)
{
    RotateArgs a{};
    if (!q) return fail(TT_ERR_NULL, "q is NULL");
    if ((k == nullptr) != (k_output == nullptr)) return fail(TT_ERR_NULL, "k and its output go together");
    int rc = check_sizes_of(n_rows, D, (int64_t)q->heads + (k ? k->heads : 0));
    if (rc) return rc;
    if ((rc = check_heads(q, "q", n_rows, D, q->type, q->heads, IN)) || (rc = check_heads(q_output, "q_output", n_rows, D, q->type, q->heads, OUT))) return rc;
    if (k && ((rc = check_heads(k, "k", n_rows, D, q->type, k->heads, IN)) || (rc = check_heads(k_output, "k_output", n_rows, D, q->type, k->heads, OUT)))) return rc;
    if ((rc = check_rotation(rotation, n_rows, D, &a))) return rc;
    if (norm && !(eps >= 0.f)) return fail(TT_ERR_BAD_ARG, "eps must not be negative");
    if (!norm && (q_weight || k_weight)) return fail(TT_ERR_BAD_ARG, "weights belong to a norm");
    if ((rc = check_weight(q_weight, "q_weight", q_weight_type)) || (rc = check_weight(k_weight, "k_weight", k_weight_type))) return rc;
    a.q = of(q);
    a.k = of(k);
    a.oq = of(q_output);
    a.ok = of(k_output);
    a.wq = q_weight;
    a.wk = k_weight;
    a.wq_type = q_weight_type;
    a.wk_type = k_weight_type;
    a.q_heads = q->heads;
    a.k_heads = k ? k->heads : 0;
    a.rows = n_rows;
    a.D = (int)D;
    a.eps = eps;
    if (n_rows == 0 || D == 0 || a.q_heads + a.k_heads == 0) return TT_OK;
    shape_of(a);
    slices_of(a);
    const dim3 grid = grid_of(ceil_div(n_rows * ((int64_t)a.q_slices + a.k_slices), WG >> a.lg), WG);
    with_type(q->type, [&](auto t) {
        with_shape(a, norm != 0, [&](auto nm, auto whole, auto nb) {
            hipLaunchKernelGGL((rotate_kernel<decltype(t), decltype(nm)::value, decltype(whole)::value, decltype(nb)::value>), grid, dim3(WG), 0, (hipStream_t)stream, a);
        });
    });
    return launched("rotation launch");
}

size_t tt_qk_norm_rotate_bwd_workspace_bytes(int64_t n_rows, int64_t q_heads, int64_t k_heads, int64_t D)
{
    if (n_rows <= 0 || D <= 0 || q_heads < 0 || k_heads < 0 || check_sizes_of(n_rows, D, q_heads + k_heads)) return 0;
    const int64_t heads = n_rows * (q_heads + k_heads);      // (a workgroup has one at least)
    return (size_t)(heads < BWD_WORKGROUPS + 2 ? heads : BWD_WORKGROUPS + 2) * (size_t)D * sizeof(float);
}

int tt_qk_norm_rotate_bwd(const tt_heads_t *grad_q_output, const tt_heads_t *grad_k_output, const tt_heads_t *q, const tt_heads_t *k,
                          const tt_rotation_t *rotation, int norm, float eps,
                          const void *q_weight, int32_t q_weight_type, const void *k_weight, int32_t k_weight_type,
                          const tt_heads_t *grad_q, const tt_heads_t *grad_k, void *grad_q_weight, int32_t grad_q_weight_type,
                          void *grad_k_weight, int32_t grad_k_weight_type, int accumulate, int64_t n_rows, int64_t D,
                          void *workspace, size_t workspace_bytes, void *stream)
{
    RotateArgs a{};
    if (!grad_q_output) return fail(TT_ERR_NULL, "grad_q_output is NULL");
    if ((grad_k_output == nullptr) != (grad_k == nullptr)) return fail(TT_ERR_NULL, "grad_k and the output's gradient go together");
    const int32_t type = grad_q_output->type, q_heads = grad_q_output->heads, k_heads = grad_k_output ? grad_k_output->heads : 0;
    int rc = check_sizes_of(n_rows, D, (int64_t)q_heads + k_heads);
    if (rc) return rc;
    if ((rc = check_heads(grad_q_output, "grad_q_output", n_rows, D, type, q_heads, IN)) || (rc = check_heads(grad_q, "grad_q", n_rows, D, type, q_heads, OUT))) return rc;
    if (grad_k && ((rc = check_heads(grad_k_output, "grad_k_output", n_rows, D, type, k_heads, IN)) || (rc = check_heads(grad_k, "grad_k", n_rows, D, type, k_heads, OUT)))) return rc;
    if ((rc = check_rotation(rotation, n_rows, D, &a))) return rc;
    if (norm) {
        if (!(eps >= 0.f)) return fail(TT_ERR_BAD_ARG, "eps must not be negative");
        if ((rc = check_heads(q, "q", n_rows, D, type, q_heads, IN))) return rc;
        if (grad_k && (rc = check_heads(k, "k", n_rows, D, type, k_heads, IN))) return rc;
    } else if (q_weight || k_weight || grad_q_weight || grad_k_weight) {
        return fail(TT_ERR_BAD_ARG, "weights belong to a norm");
    }
    if (grad_k_weight && !grad_k) return fail(TT_ERR_BAD_ARG, "grad_k_weight without keys");
    if ((rc = check_weight(q_weight, "q_weight", q_weight_type)) || (rc = check_weight(k_weight, "k_weight", k_weight_type)) ||
        (rc = check_weight(grad_q_weight, "grad_q_weight", grad_q_weight_type)) || (rc = check_weight(grad_k_weight, "grad_k_weight", grad_k_weight_type))) return rc;
    if (D == 0) return TT_OK;
    const bool weights = grad_q_weight || grad_k_weight;
    const bool some = n_rows > 0 && q_heads + k_heads > 0;
    if (!some && (!weights || accumulate)) return TT_OK;
    a.q = of(q);
    a.k = of(k);
    a.gq = of(grad_q_output);
    a.gk = of(grad_k_output);
    a.oq = of(grad_q);
    a.ok = of(grad_k);
    a.wq = q_weight;
    a.wk = k_weight;
    a.wq_type = q_weight_type;
    a.wk_type = k_weight_type;
    a.q_heads = q_heads;
    a.k_heads = k_heads;
    a.rows = n_rows;
    a.D = (int)D;
    a.eps = eps;
    a.gwq = grad_q_weight;
    a.gwk = grad_k_weight;
    a.gwq_type = grad_q_weight_type;
    a.gwk_type = grad_k_weight_type;
    a.add = accumulate;
    hipStream_t st = (hipStream_t)stream;
    int64_t grid = 0;
    // (queries and keys have sums of their own, and of two that go to one place one would be lost)
    const char *const gwq = (const char *)grad_q_weight, *const gwk = (const char *)grad_k_weight;
    const bool apart = !gwq || !gwk || gwq + D * element_bytes(grad_q_weight_type) <= gwk || gwk + D * element_bytes(grad_k_weight_type) <= gwq;
    auto overlap = [] { return fail(TT_ERR_BAD_ARG, "grad_q_weight and grad_k_weight overlap"); };
    if (some) {
        shape_of(a);
        slices_of(a);
        a.q_workgroups = (int)bwd_workgroups(a, false);
        const int64_t k_workgroups = bwd_workgroups(a, true);
        grid = a.q_workgroups + k_workgroups;
        // (a weight whose heads are none has a gradient of zeros, which only the second launch writes)
        const bool alone = a.q_workgroups == 1 && k_workgroups == (grad_k_weight ? 1 : k_workgroups);
        const size_t need = weights && !alone ? (size_t)grid * (size_t)D * sizeof(float) : 0;
        if (need && (!workspace || workspace_bytes < need)) return fail(TT_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace_bytes);
        if ((uintptr_t)workspace & 15) return fail(TT_ERR_BAD_ARG, "workspace must be 16-byte aligned");
        if (!apart) return overlap();
        a.part = need ? (float *)workspace : nullptr;
        const size_t lds = weights ? (size_t)NWAVE * 16 * a.units * sizeof(float) : 0;
        with_type(type, [&](auto t) {
            with_shape(a, norm != 0, [&](auto nm, auto whole, auto nb) {
                hipLaunchKernelGGL((rotate_bwd_kernel<decltype(t), decltype(nm)::value, decltype(whole)::value, decltype(nb)::value>), dim3((unsigned)grid), dim3(WG), lds, st, a);
            });
        });
    } else if (!apart) {
        return overlap();
    }
    if (weights && (a.part || !some)) hipLaunchKernelGGL(rotate_weight_kernel, dim3((unsigned)ceil_div(D, 32), 2), dim3(1024), 0, st, a, (int)grid);
    return launched("rotation gradient launch");
}

}  // extern "C"
