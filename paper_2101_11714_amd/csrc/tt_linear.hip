// C-ABI entry points of the matrix product with its epilogue (declared in include/tt_emb.h): argument checks, workspace layout, kernel
// selection and launches.  Nothing here allocates device memory or waits for the stream.

#include "../../include/tt_emb.h"

#include "tt_rows_args.h"
#include "tt_linear.h"
#include "tt_product_few.h"
#include "tt_product_stream.h"

using namespace tt;

namespace {

constexpr int64_t MOST_COLUMNS = 1ll << 24;                  // of x, weight and output

// How a product is computed.
enum Way { FEW, TILES, STREAM, STREAM_WIDE };

struct Plan {
    Way way;
    int64_t tiles_m, tiles_n;
    int parts;
    int64_t k_part;
};

constexpr int64_t MOST_TILES = 512;                          // workgroups that parts are made for

// Parts of k, of four steps at least, where the tiles alone are too few for the device.
int64_t parts_of(int64_t tiles, int64_t steps)
{
    int64_t parts = tiles < 256 ? MOST_TILES / (tiles > 0 ? tiles : 1) : 1;
    if (parts > steps / 4) parts = steps / 4;
    return parts < 1 ? 1 : parts;
}

Plan plan_of(int64_t M, int64_t N, int64_t K, int32_t type, bool dense, bool whole)
{
    Plan p{};
    const int64_t step = 128 / element_bytes(type);
    p.parts = 1;
    p.k_part = K;
    if (dense && M <= PF_MOST) {
        p.way = FEW;
        return p;
    }
    p.way = !whole || type == TT_F32 ? TILES : ceil_div(M, 256) * ceil_div(N, 256) >= 128 ? STREAM_WIDE : STREAM;
    const int64_t tile = p.way == STREAM_WIDE ? 256 : 128, steps = ceil_div(K, step);
    p.tiles_m = ceil_div(M, p.way == TILES && M <= 32 ? 32 : tile);
    p.tiles_n = ceil_div(N, tile);
    const int64_t parts = parts_of(p.tiles_m * p.tiles_n, steps);
    p.k_part = ceil_div(steps, parts) * step;
    p.parts = K > 0 ? (int)ceil_div(K, p.k_part) : 1;
    return p;
}

// What the parts' sums of a product of M rows, or of fewer, take at most, whatever its way: with more rows there are fewer parts, but a part is
// no larger than its tiles.
size_t parts_bytes(int64_t M, int64_t N, int64_t K, int32_t type)
{
    if (M <= 0 || N <= 0) return 0;
    const int64_t most = ceil_div(K, 128 / element_bytes(type)) / 4, wide = ceil_div(N, 256);
    if (wide >= 256 || most < 2) return 0;
    const int64_t rows = M * (most < MOST_TILES ? most : MOST_TILES), tiled = MOST_TILES * 256 / wide;
    return (size_t)(rows < tiled ? rows : tiled) * (size_t)(8 * ceil_div(N, 8)) * sizeof(float);
}

bool whole_chunks(const void *p, int64_t ld, int64_t columns, int32_t type)
{
    return type != TT_F32 && columns % 8 == 0 && ld % 8 == 0 && (uintptr_t)p % 16 == 0 && ld <= PS_MOST_STRIDE;
}

// C = A B^T; AK, BK: the operands' rows are dense in k
template <typename T, typename O, bool AK, bool BK>
int product(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t M, int64_t N, int64_t K, const EpilogueArgs &e, void *workspace, hipStream_t st)
{
    if (M == 0 || N == 0) return TT_OK;
    const int32_t type = sizeof(T) == 4 ? TT_F32 : TT_BF16;
    const bool whole = whole_chunks(a, lda, AK ? K : M, type) && whole_chunks(b, ldb, BK ? K : N, type);
    const Plan p = plan_of(M, N, K, type, AK && BK, whole);
    ProductArgs q{a, b, lda, ldb, M, N, K, (int)p.tiles_m, (int)p.tiles_n, p.k_part, p.parts > 1 ? (float *)workspace : nullptr, 8 * ceil_div(N, 8)};
    if (p.way == FEW) {
        if constexpr (AK && BK) {
            const dim3 grid = grid_of(ceil_div(N, BLOCK), PF_WAVES * WAVE);
            const bool chunks = whole || (type == TT_F32 && K % 4 == 0 && lda % 4 == 0 && ldb % 4 == 0 && (uintptr_t)a % 16 == 0 && (uintptr_t)b % 16 == 0);
            with_flag(chunks && K > 0, [&](auto w) {
                auto launch = [&](auto mb) { hipLaunchKernelGGL((product_few_kernel<T, O, decltype(mb)::value, decltype(w)::value>), grid, dim3(PF_WAVES * WAVE), 0, st, q, e); };
                if (M <= 16) launch(std::integral_constant<int, 1>{});
                else if (M <= 32) launch(std::integral_constant<int, 2>{});
                else launch(std::integral_constant<int, 4>{});
            });
        }
        return launched("product launch");
    }
    if (p.way == TILES) {
        dim3 grid = grid_of(p.tiles_m * p.tiles_n, WG);
        grid.z = (unsigned)p.parts;
        if (M <= 32) hipLaunchKernelGGL((product_kernel<T, O, AK, BK, 32, 128>), grid, dim3(WG), 0, st, q, e);
        else hipLaunchKernelGGL((product_kernel<T, O, AK, BK, 128, 128>), grid, dim3(WG), 0, st, q, e);
    } else if constexpr (sizeof(T) == 2) {
        int rc = TT_OK;
        with_flag(p.way == STREAM_WIDE, [&](auto w) {
            typedef StreamShape<decltype(w)::value> S;
            dim3 grid = grid_of(p.tiles_m * p.tiles_n, S::THREADS);
            grid.z = (unsigned)p.parts;
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

int check_product(int64_t M, int64_t K, int64_t N)
{
    int rc = check_sizes(M, K);
    if (!rc) rc = check_sizes(M, N);
    if (!rc) rc = check_sizes(N, K);
    if (rc) return rc;
    if (K > MOST_COLUMNS || N > MOST_COLUMNS) return fail(TT_ERR_UNSUPPORTED, "more than 2^24 columns");
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

// Where what lies in the workspace of a gradient: parts of sums first (of one product, then of the other), the gradient in front of the
// activation, the columns' sums of the bands.
struct GradRoom {
    size_t parts, dz, bands, all;
    int64_t band, n_bands;
};

GradRoom grad_room(int64_t M, int64_t K, int64_t N, int32_t type, int32_t act, bool x, bool w, bool b)
{
    GradRoom r{};
    const size_t px = x ? parts_bytes(M, K, N, type) : 0, pw = w ? parts_bytes(N, K, M, type) : 0;
    const int64_t cols = 8 * ceil_div(N, 8);
    r.parts = up(px > pw ? px : pw);
    r.dz = act != TT_ACT_NONE && (x || w) ? up((size_t)M * (size_t)cols * element_bytes(type)) : 0;
    r.n_bands = M < 64 * 256 ? ceil_div(M, 64) : 256;
    r.band = ceil_div(M, r.n_bands > 0 ? r.n_bands : 1);
    r.bands = b ? up((size_t)r.n_bands * (size_t)cols * sizeof(float)) : 0;
    r.all = r.parts + r.dz + r.bands;
    return r;
}

template <typename F>
void with_output(int32_t type, int32_t out, F f)
{
    with_type(type, [&](auto t) {
        if (out == TT_F32) f(t, float{});
        else f(t, t);
    });
}

}  // namespace

extern "C" {

size_t tt_linear_fwd_workspace_bytes(int64_t n_rows, int64_t K, int64_t N, int32_t type)
{
    if (check_product(n_rows, K, N) || (type != TT_F32 && type != TT_BF16 && type != TT_F16)) return 0;
    return n_rows <= PF_MOST ? 0 : parts_bytes(n_rows, N, K, type);
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
    if ((rc = check_workspace(tt_linear_fwd_workspace_bytes(n_rows, K, N, x->type), workspace, workspace_bytes))) return rc;
    EpilogueArgs e{bias, bias_type, activation, residual ? residual->data : nullptr, pre ? pre->data : nullptr, output->data, residual ? residual->ld : 0, pre ? pre->ld : 0, output->ld};
    with_output(x->type, output->type, [&](auto t, auto o) {
        rc = product<decltype(t), decltype(o), true, true>(x->data, x->ld, weight->data, weight->ld, n_rows, N, K, e, workspace, (hipStream_t)stream);
    });
    return rc;
}

size_t tt_linear_bwd_workspace_bytes(int64_t n_rows, int64_t K, int64_t N, int32_t type, int32_t activation)
{
    if (check_product(n_rows, K, N) || (type != TT_F32 && type != TT_BF16 && type != TT_F16)) return 0;
    return grad_room(n_rows, K, N, type, activation, true, true, true).all;
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
    const GradRoom room = grad_room(n_rows, K, N, type, activation, grad_x != nullptr, grad_weight != nullptr, grad_bias != nullptr);
    if ((rc = check_workspace(room.all, workspace, workspace_bytes))) return rc;
    hipStream_t st = (hipStream_t)stream;
    char *ws = (char *)workspace;
    const void *dz = grad_output->data;
    int64_t ld_dz = grad_output->ld;
    if (N > 0 && (room.dz || room.bands) && n_rows > 0) {
        SlopeArgs a{};
        a.dy = grad_output->data;
        a.ld_dy = grad_output->ld;
        if (activation != TT_ACT_NONE) {
            a.pre = pre->data;
            a.ld_pre = pre->ld;
        }
        a.N = (int)N;
        a.nv = (int)ceil_div(N, 8);
        if (room.dz) {
            a.dz = ws + room.parts;
            a.ld_dz = 8 * a.nv;
            dz = a.dz;
            ld_dz = a.ld_dz;
        }
        a.part = room.bands ? (float *)(ws + room.parts + room.dz) : nullptr;
        a.rows = n_rows;
        a.band = room.band;
        a.act = activation;
        with_type(type, [&](auto t) {
            with_whole(N, [&](auto whole) {
                hipLaunchKernelGGL((slope_kernel<decltype(t), decltype(whole)::value>), dim3((unsigned)ceil_div(a.nv, 32), (unsigned)room.n_bands), dim3(WG), 0, st, a);
            });
        });
        if ((rc = launched("gradient launch"))) return rc;
    }
    if (grad_bias && N > 0) {
        with_type(grad_bias_type, [&](auto w) {
            hipLaunchKernelGGL((bias_sum_kernel<decltype(w)>), dim3((unsigned)ceil_div(N, 64)), dim3(WG), 0, st, (const float *)(ws + room.parts + room.dz), (int)room.n_bands, (int)N,
                               (int)(8 * ceil_div(N, 8)), (decltype(w) *)grad_bias, accumulate);
        });
        if ((rc = launched("gradient launch"))) return rc;
    }
    if (grad_x) {
        EpilogueArgs e{};
        e.out = grad_x->data;
        e.ld_out = grad_x->ld;
        with_type(type, [&](auto t) {
            typedef decltype(t) T;
            rc = product<T, T, true, false>(dz, ld_dz, weight->data, weight->ld, n_rows, K, N, e, ws, st);
        });
        if (rc) return rc;
    }
    if (grad_weight && !(accumulate && n_rows == 0)) {
        EpilogueArgs e{};
        e.out = grad_weight->data;
        e.ld_out = grad_weight->ld;
        if (accumulate) {
            e.add = e.out;
            e.ld_add = e.ld_out;
        }
        with_output(type, grad_weight->type, [&](auto t, auto o) {
            rc = product<decltype(t), decltype(o), false, false>(dz, ld_dz, x->data, x->ld, N, K, n_rows, e, ws, st);
        });
    }
    return rc;
}

}  // extern "C"
