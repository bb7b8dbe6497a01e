// C-ABI entry points of the matrix product with its epilogue (declared in include/tt_emb.h): argument checks, workspace layout, kernel
// selection and launches.  Nothing here allocates device memory or waits for the stream.

#include "../../include/tt_emb.h"

#include "tt_rows_args.h"
#include "tt_linear.h"
#include "tt_product_launch.h"

using namespace tt;

namespace {

constexpr int64_t MOST_COLUMNS = PS_MOST_STRIDE;             // of x, weight and output, so that copies in whole chunks can be loaded

int check_product(int64_t M, int64_t K, int64_t N)
{
    int rc = check_sizes(M, K);
    if (!rc) rc = check_sizes(M, N);
    if (!rc) rc = check_sizes(N, K);
    if (rc) return rc;
    if (K > MOST_COLUMNS || N > MOST_COLUMNS) return fail(TT_ERR_UNSUPPORTED, "more than 2^22 columns");
    return TT_OK;
}

int check_vector(const void *v, const char *name, int32_t type)
{
    if (!v) return TT_OK;
    if (type != TT_F32 && type != TT_BF16 && type != TT_F16) return fail(TT_ERR_UNSUPPORTED, "%s: type %d is not supported", name, (int)type);
    return (uintptr_t)v % element_bytes(type) ? fail(TT_ERR_BAD_ARG, "%s is not aligned to its elements", name) : TT_OK;
}

int check_workspace(size_t need, const void *workspace, size_t bytes)
{
    if (need && (!workspace || bytes < need)) return fail(TT_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, bytes);
    if ((uintptr_t)workspace & 15) return fail(TT_ERR_BAD_ARG, "workspace must be 16-byte aligned");
    return TT_OK;
}

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// Where what lies in the workspace of a product: parts of sums, copies of x and of the weight in whole chunks where they are not.  The parts' room is the
// call's own by its plan; a query's, which is to do for fewer rows and so for any plan, is product_bytes.
struct Room {
    bool few;                    // (few rows are loaded as they lie)
    size_t parts, x, w, all;
};

Room product_room(int64_t M, int64_t K, int64_t N, int32_t type, bool whole_x, bool whole_w, Product *call = nullptr)
{
    Room r{};
    r.few = few_rows(M, N, K, type, whole_x && whole_w);
    if (r.few) return r;
    if (call) {
        double us;
        const Size d{M, N, K};
        call->kind = plan_of(&d, 1, type, &call->plan, us);
        r.parts = up(parts_bytes(d, call->plan));
    } else {
        r.parts = up(product_bytes(M, N, K, type));
    }
    r.x = whole_x ? 0 : up(packed_bytes(M, K, type));
    r.w = whole_w ? 0 : up(packed_bytes(N, K, type));
    r.all = r.parts + r.x + r.w;
    return r;
}

// The same of a gradient: parts of sums of both products, the gradient in front of the activation, or a copy of the output's in rows of whole chunks,
// copies of x and of the weight, the columns' sums of the bands.
struct GradRoom {
    size_t parts_x, parts_w, dz, x, w, bands, all;
    int64_t band, n_bands;
};

GradRoom grad_room(int64_t M, int64_t K, int64_t N, int32_t type, bool copy, bool copy_x, bool copy_w, bool x, bool w, bool b, const Product *dx = nullptr, const Product *dw = nullptr)
{
    GradRoom r{};
    r.parts_x = dx ? up(parts_bytes(dx->d, dx->plan)) : x ? up(product_bytes(M, K, N, type)) : 0;
    r.parts_w = dw ? up(parts_bytes(dw->d, dw->plan)) : w ? up(product_bytes(N, K, M, type)) : 0;
    r.dz = copy && (x || w) ? up(packed_bytes(M, N, type)) : 0;
    r.x = copy_x ? up(packed_bytes(M, K, type)) : 0;
    r.w = copy_w ? up(packed_bytes(N, K, type)) : 0;
    r.n_bands = M < 64 * 256 ? ceil_div(M, 64) : 256;
    r.band = ceil_div(M, r.n_bands > 0 ? r.n_bands : 1);
    r.bands = b && r.n_bands > 1 ? up((size_t)r.n_bands * (size_t)(8 * ceil_div(N, 8)) * sizeof(float)) : 0;
    r.all = r.parts_x + r.parts_w + r.dz + r.x + r.w + r.bands;
    return r;
}

}  // namespace

extern "C" {

size_t tt_linear_fwd_workspace_bytes(int64_t n_rows, int64_t K, int64_t N, int32_t type, int whole)
{
    if (check_product(n_rows, K, N) || (type != TT_F32 && type != TT_BF16 && type != TT_F16)) return 0;
    // fewer rows may go another way, and so may arrays that are whole after all
    size_t most = 0;
    for (const bool w : {true, whole || type == TT_F32})
        for (const int64_t up_to : {PF_CLASS[0], PF_CLASS[1], PF_CLASS[2], n_rows}) {
            const size_t need = product_room(n_rows < up_to ? n_rows : up_to, K, N, type, w, w).all;
            if (need > most) most = need;
        }
    return most;
}

int tt_linear_fwd(const tt_rows_t *x, const tt_rows_t *weight, const void *bias, int32_t bias_type, int32_t activation,
                  const tt_rows_t *residual, const tt_rows_t *pre, const tt_rows_t *output, int64_t n_rows, int64_t K, int64_t N,
                  void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_product(n_rows, K, N);
    if (rc) return rc;
    if ((rc = check_rows(x, "x", n_rows, K, IN)) || (rc = check_rows(weight, "weight", N, K, IN)) || (rc = check_rows(output, "output", n_rows, N, OUT))) return rc;
    if (residual && (rc = check_rows(residual, "residual", n_rows, N, IN))) return rc;
    if (pre && (rc = check_rows(pre, "pre", n_rows, N, OUT))) return rc;
    if ((rc = check_vector(bias, "bias", bias_type))) return rc;
    if (weight->type != x->type) return fail(TT_ERR_UNSUPPORTED, "weight has x's type");
    if (output->type != x->type && output->type != TT_F32) return fail(TT_ERR_UNSUPPORTED, "output has x's type or 32 bits");
    if (residual && residual->type != output->type) return fail(TT_ERR_UNSUPPORTED, "residual has the output's type");
    if (pre && pre->type != x->type) return fail(TT_ERR_UNSUPPORTED, "pre has x's type");
    if (activation < 0 || activation >= ACT_COUNT) return fail(TT_ERR_BAD_ARG, "activation %d", (int)activation);
    Product p{};
    const Room room = product_room(n_rows, K, N, x->type, whole_chunks(*x, K), whole_chunks(*weight, K), &p);
    if ((rc = check_workspace(room.all, workspace, workspace_bytes))) return rc;
    char *ws = (char *)workspace;
    p.a = {x->data, x->ld, n_rows, K, room.x ? ws + room.parts : nullptr};
    p.b = {weight->data, weight->ld, N, K, room.w ? ws + room.parts + room.x : nullptr};
    p.d = {n_rows, N, K};
    p.e = {bias, bias_type, activation, residual ? residual->data : nullptr, pre ? pre->data : nullptr, output->data, residual ? residual->ld : 0, pre ? pre->ld : 0, output->ld};
    p.parts = (float *)ws;
    p.few = room.few;
    with_type(x->type, [&](auto t) { rc = product_of<decltype(t)>(output->type, p, (hipStream_t)stream); });
    return rc;
}

size_t tt_linear_bwd_workspace_bytes(int64_t n_rows, int64_t K, int64_t N, int32_t type, int32_t activation, int whole)
{
    if (check_product(n_rows, K, N) || (type != TT_F32 && type != TT_BF16 && type != TT_F16)) return 0;
    const bool copy = !whole && type != TT_F32;
    return grad_room(n_rows, K, N, type, copy || activation != TT_ACT_NONE, copy, copy, true, true, true).all;
}

int tt_linear_bwd(const tt_rows_t *grad_output, const tt_rows_t *x, const tt_rows_t *weight, const tt_rows_t *pre, int32_t activation,
                  const tt_rows_t *grad_x, const tt_rows_t *grad_weight, void *grad_bias, int32_t grad_bias_type, int accumulate,
                  int64_t n_rows, int64_t K, int64_t N, void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_product(n_rows, K, N);
    if (rc) return rc;
    if ((rc = check_rows(grad_output, "grad_output", n_rows, N, IN))) return rc;
    if (activation < 0 || activation >= ACT_COUNT) return fail(TT_ERR_BAD_ARG, "activation %d", (int)activation);
    const int32_t type = grad_output->type;
    if (activation != TT_ACT_NONE) {
        if ((rc = check_rows(pre, "pre", n_rows, N, IN))) return rc;
        if (pre->type != type) return fail(TT_ERR_UNSUPPORTED, "pre has grad_output's type");
    }
    if (grad_x) {
        if ((rc = check_rows(grad_x, "grad_x", n_rows, K, OUT)) || (rc = check_rows(weight, "weight", N, K, IN))) return rc;
        if (grad_x->type != type || weight->type != type) return fail(TT_ERR_UNSUPPORTED, "weight and grad_x have grad_output's type");
    }
    if (grad_weight) {
        if ((rc = check_rows(grad_weight, "grad_weight", N, K, OUT)) || (rc = check_rows(x, "x", n_rows, K, IN))) return rc;
        if (x->type != type) return fail(TT_ERR_UNSUPPORTED, "x has grad_output's type");
        if (grad_weight->type != type && grad_weight->type != TT_F32) return fail(TT_ERR_UNSUPPORTED, "grad_weight has grad_output's type or 32 bits");
    }
    if ((rc = check_vector(grad_bias, "grad_bias", grad_bias_type))) return rc;
    const bool copy = activation != TT_ACT_NONE || !whole_chunks(*grad_output, N);
    const bool copy_x = grad_weight && !whole_chunks(*x, K), copy_w = grad_x && !whole_chunks(*weight, K);
    Product dx{}, dw{};
    const bool some_w = grad_weight && !(accumulate && n_rows == 0);             // (else there is nothing to add)
    if (grad_x) dx.d = {n_rows, K, N};
    if (some_w) dw.d = {N, K, n_rows};
    const Size sizes[2] = {dx.d, dw.d};
    Plan plans[2];
    double us;
    dx.kind = dw.kind = plan_of(sizes, 2, type, plans, us);
    dx.plan = plans[0];
    dw.plan = plans[1];
    const GradRoom room = grad_room(n_rows, K, N, type, copy, copy_x, copy_w, grad_x != nullptr, grad_weight != nullptr, grad_bias != nullptr, &dx, &dw);
    if ((rc = check_workspace(room.all, workspace, workspace_bytes))) return rc;
    hipStream_t st = (hipStream_t)stream;
    char *ws = (char *)workspace;
    const void *dz = grad_output->data;
    int64_t ld_dz = grad_output->ld;
    char *const at_dz = ws + room.parts_x + room.parts_w, *const at_x = at_dz + room.dz, *const at_w = at_x + room.x;
    BiasSum bias{nullptr, grad_bias, grad_bias_type, accumulate, (int)room.n_bands, (int)N, (int)(8 * ceil_div(N, 8))};
    if (grad_bias && n_rows == 0) bias.part = (const float *)grad_bias;          // (no bands: nothing of it is read)
    if (room.dz) {
        dz = at_dz;
        ld_dz = 8 * ceil_div(N, 8);
    }
    if (grad_x) {
        dx.a = {dz, ld_dz, n_rows, N, nullptr};
        dx.b = {weight->data, weight->ld, N, K, copy_w ? at_w : nullptr};
        dx.e.out = grad_x->data;
        dx.e.ld_out = grad_x->ld;
        dx.parts = (float *)ws;
    }
    if (some_w) {
        dw.a = {dz, ld_dz, n_rows, N, nullptr};
        dw.b = {x->data, x->ld, n_rows, K, copy_x ? at_x : nullptr};
        dw.e.out = grad_weight->data;
        dw.e.ld_out = grad_weight->ld;
        if (accumulate) {
            dw.e.add = dw.e.out;
            dw.e.ld_add = dw.e.ld_out;
        }
        dw.parts = (float *)(ws + room.parts_x);
    }
    if (N > 0 && (room.dz || grad_bias) && n_rows > 0) {
        SlopeArgs a{};
        a.dy = grad_output->data;
        a.ld_dy = grad_output->ld;
        if (activation != TT_ACT_NONE) {
            a.pre = pre->data;
            a.ld_pre = pre->ld;
        }
        a.N = (int)N;
        a.nv = (int)ceil_div(N, 8);
        a.groups = (int)ceil_div(a.nv, 32);
        if (room.dz) {
            a.dz = at_dz;
            a.ld_dz = ld_dz;
        }
        if (room.bands) bias.part = a.part = (float *)(at_w + room.w);
        else a.one = bias;
        a.rows = n_rows;
        a.band = room.band;
        a.act = activation;
        int64_t copies;
        const PackArgs pack = pack_args(dx.b, dw.b, copies);
        const dim3 grid((unsigned)(a.groups + ceil_div(copies, room.n_bands)), (unsigned)room.n_bands);
        with_type(type, [&](auto t) {
            with_whole(N, [&](auto whole) {
                with_flag(activation != TT_ACT_NONE, [&](auto act) {
                    hipLaunchKernelGGL((slope_kernel<decltype(t), decltype(whole)::value, decltype(act)::value>), grid, dim3(WG), 0, st, a, pack);
                });
            });
        });
        if ((rc = launched("gradient launch"))) return rc;
    }
    with_type(type, [&](auto t) { rc = gradients_of<decltype(t)>(grad_weight ? grad_weight->type : type, dx, dw, bias, st); });
    return rc;
}

}  // extern "C"
