// Checks of arguments and choice of types that the operators on rows of arrays share (tt_token.hip, tt_norm.hip).
#pragma once

#include <type_traits>

#include "tt_error.h"
#include "tt_rows_io.h"

namespace tt {

constexpr int64_t MOST_ROWS = 1ll << 31;                     // rows and columns stay below
constexpr int64_t MOST_ELEMENTS = 1ll << 40;                 // so do rows times columns: what every launch here takes, and no card holds

inline int element_bytes(int32_t type) { return type == TT_F32 ? 4 : type == TT_E4M3 ? 1 : 2; }

// calls f with b as a type
template <typename F>
void with_flag(bool b, F f)
{
    if (b) f(std::true_type{});
    else f(std::false_type{});
}

// calls f with whether rows of N columns consist of whole vectors
template <typename F>
void with_whole(int64_t N, F f)
{
    with_flag(N % 8 == 0, f);
}

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
inline int check_rows(const tt_rows_t *a, const char *name, int64_t n, int64_t N, int way, bool bits8 = false)
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

inline int check_sizes(int64_t rows, int64_t N)
{
    if (rows < 0 || N < 0) return fail(TT_ERR_BAD_ARG, "negative size");
    if (rows >= MOST_ROWS || N >= MOST_ROWS) return fail(TT_ERR_UNSUPPORTED, "2^31 rows or columns, or more");
    if (rows * N >= MOST_ELEMENTS) return fail(TT_ERR_UNSUPPORTED, "2^40 elements or more");
    return TT_OK;
}

inline int check_dropout(const tt_dropout_t *d, DropArgs *out)
{
    *out = DropArgs{nullptr, 0u, 0u, 1.f};
    if (!d) return TT_OK;
    if (!(d->p >= 0.f && d->p <= 1.f)) return fail(TT_ERR_BAD_ARG, "dropout: p outside [0, 1]");
    const uint32_t q = (uint32_t)((double)d->p * 65536.0 + 0.5);
    if (q == 0) return TT_OK;                                // nothing is dropped
    if (!d->state) return fail(TT_ERR_NULL, "dropout: state is NULL");
    if ((uintptr_t)d->state % 8) return fail(TT_ERR_BAD_ARG, "dropout: state is not aligned");
    *out = DropArgs{d->state, d->site, (uint32_t)(65536ull * q - 1), q < 65536u ? (float)(65536.0 / (65536.0 - (double)q)) : 0.f};
    return TT_OK;
}

inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TT_OK : hip_fail(e, what);
}

// A grid for kernels that take their number from workgroup().  A launch takes less than 2^32 threads along x; where there are more, y goes on
// (with MOST_ELEMENTS to about 2^10), and the last row's surplus workgroups find nothing to do.
inline dim3 grid_of(int64_t workgroups, int threads)
{
    if (workgroups * threads < (1ll << 32)) return dim3((unsigned)workgroups);
    return dim3(1u << GRID_LG, (unsigned)ceil_div(workgroups, 1ll << GRID_LG));
}

}  // namespace tt
