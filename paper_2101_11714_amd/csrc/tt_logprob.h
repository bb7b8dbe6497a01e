// Log probabilities of tokens under rows of logits, with entropy and the likeliest alternatives, and the gradient.
//
// One pass over a row holds the largest logit m so far, S = sum of exp(z - m) and T = sum of exp(z - m) (z - m) / log 2 in 32 bits, and multiplies the two
// sums when m grows; lse = m + log S, entropy = log S - T log 2 / S, both without a difference of large numbers.  Few rows are cut into
// pieces, a workgroup each, which a second launch joins.
// The k likeliest: the k-th largest of the threads' largest logits is no larger than the k-th largest of all, so that few more than k logits
// are left to be ranked.  Logits are ordered by a 64-bit key, value first and column after it, so that no two are equal.
#pragma once

#include "tt_rows_io.h"

namespace tt {

constexpr int LP_UNROLL = 4;                                 // vectors of eight logits a thread loads at a time
constexpr int LP_LIST = 1024;                                // candidates that a workgroup can rank
constexpr int LP_MOST_K = 64;
constexpr float LP_LEAST = -3.402823466e38f, LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct LogprobArgs {
    const void *logits;
    int64_t ld;
    const void *tokens;          // null: none
    int tokens64;
    float scale;
    float *logprob, *lse, *entropy;
    int k, ids64;
    void *ids;
    float *top;
    int64_t rows;
    int V, nv;                   // vectors of eight of a row
    int pieces, piece;           // of a row, vectors of one
    float *sums;                 // [rows][pieces][4]: m, S, T of pieces
    uint64_t *keys;              // [rows][pieces][k]
};

struct Sums {
    float m, s, t;
};

// the sums about another maximum, no smaller than theirs; 0 for what has none
__device__ __forceinline__ Sums about(const Sums &a, float m, float c)
{
    const float d = fmaxf((a.m - m) * c, LP_LEAST), f = __builtin_amdgcn_exp2f(d);
    return {m, a.s * f, f == 0.f ? a.s * f : f * (a.t + d * a.s)};
}

// a wave's sums, in every lane
__device__ __forceinline__ Sums joined(Sums a, float c)
{
    auto add = [](float x, float y) { return x + y; };
    a = about(a, lanes_reduce(a.m, 6, [](float x, float y) { return fmaxf(x, y); }), c);
    a.s = lanes_reduce(a.s, 6, add);
    a.t = lanes_reduce(a.t, 6, add);
    return a;
}

__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);             // (-0 is 0)
    if (x != x) return 0xffffffffu;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) { return order == 0xffffffffu ? __uint_as_float(0x7fc00000u) : __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }

// 0: no alternative
__device__ __forceinline__ uint64_t key_of(float x, uint32_t column)
{
    return x == -INFINITY ? 0ull : (uint64_t)order_of(x) << 32 | (uint32_t)~column;
}

// The upper halves of the n-th and of the k-th largest of a wave's 64 values (1 to 64), bit by bit: no larger than these, and nearly
// as good as bounds, in half the steps.
__device__ __forceinline__ void upper_halves(uint32_t x, int n, int k, uint32_t &nth, uint32_t &kth)
{
    nth = kth = 0;
#pragma unroll
    for (uint32_t bit = 0x80000000u; bit > 0xffffu; bit >>= 1) {
        const int c = __popcll(__ballot(x >= (nth | bit))), d = __popcll(__ballot(x >= (kth | bit)));
        nth |= c >= n ? bit : 0u;
        kth |= d >= k ? bit : 0u;
    }
}

// how many of n keys are larger
__device__ __forceinline__ int rank_of(const uint64_t *keys, int n, uint64_t key)
{
    int r = 0;
#pragma unroll 8
    for (int i = 0; i < n; ++i) r += keys[i] > key;
    return r;
}

__device__ __forceinline__ int64_t token_at(const LogprobArgs &a, int64_t row) { return a.tokens64 ? ((const int64_t *)a.tokens)[row] : ((const int32_t *)a.tokens)[row]; }

// the logit of a row's token, and whether there is one
struct Given {
    float z;
    bool there;
};

template <typename T>
__device__ __forceinline__ Given given_logit(const LogprobArgs &a, int64_t row)
{
    if (!a.logprob) return {0.f, false};
    const int64_t token = token_at(a, row);
    const bool there = token >= 0 && token < a.V;
    return {(float)((const T *)a.logits)[row * a.ld + (there ? token : 0)], there};
}

// What a row's sums say.  Log probabilities are taken from the largest logit and not from lse, which has lost log S in rows of the lowest
// values of a type.
__device__ __forceinline__ void leave_row(const LogprobArgs &a, int64_t row, const Sums &r, float log_s, const Given &given)
{
    const bool none = r.s == 0.f;
    if (a.lse) a.lse[row] = none ? -INFINITY : r.m * a.scale + log_s;
    if (a.entropy) a.entropy[row] = none ? 0.f : log_s - LN2 * (r.t / r.s);
    if (a.logprob) a.logprob[row] = !given.there ? 0.f : none ? -INFINITY : a.scale * (given.z - r.m) - log_s;
}

__device__ __forceinline__ void leave_top(const LogprobArgs &a, int64_t row, int place, uint64_t key, float m, float log_s)
{
    const int64_t at = row * a.k + place, column = key ? (int64_t)(uint32_t)~(uint32_t)key : -1;
    if (a.ids64) ((int64_t *)a.ids)[at] = column;
    else ((int32_t *)a.ids)[at] = (int32_t)column;
    if (a.top) a.top[at] = key ? a.scale * (value_of((uint32_t)(key >> 32)) - m) - log_s : -INFINITY;
}

// the vectors [from, to) of a row, U of a thread's at a time: f(vector's number, its eight logits), -inf where there is no column.
// go(): whether to go on, asked when U loads are on their way.
template <typename T, bool WHOLE, int U, typename F, typename G>
__device__ __forceinline__ void each_vector(const T *line, int from, int to, int V, F f, G go)
{
#pragma unroll 1
    for (int v0 = from + threadIdx.x; v0 < to; v0 += WG * U) {
        Vec8<T> r[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int v = v0 + i * WG < to ? v0 + i * WG : to - 1;
            r[i] = fetch8<WHOLE>(line + 8 * (int64_t)v, V - 8 * v, V);
        }
        __builtin_amdgcn_sched_barrier(0);                   // (or the compiler loads them one after the other)
        if (!go()) return;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int v = v0 + i * WG;
            if (v >= to) break;
            float x[8];
            settle8<WHOLE>(r[i], V - 8 * v, V);
            widen8(r[i], x);
            if (!WHOLE && 8 * v + 8 > V)
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = 8 * v + j < V ? x[j] : -INFINITY;
            f(v, x);
        }
    }
}

template <typename T, bool WHOLE, int U, typename F>
__device__ __forceinline__ void each_vector(const T *line, int from, int to, int V, F f)
{
    each_vector<T, WHOLE, U>(line, from, to, V, f, [] { return true; });
}

// a thread's sums over its vectors of [from, to)
template <typename T, bool ENTROPY, bool WHOLE, int U = LP_UNROLL>
__device__ __forceinline__ Sums thread_sums(const T *line, int from, int to, int V, float c)
{
    Sums r{LP_LEAST, 0.f, 0.f};
    each_vector<T, WHOLE, U>(line, from, to, V, [&](int v, const float (&x)[8]) {
        float m = r.m;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, x[j]);
        if (m > r.m) {
            const float d = fmaxf((r.m - m) * c, LP_LEAST), f = __builtin_amdgcn_exp2f(d);
            if (ENTROPY) r.t = f == 0.f ? 0.f : f * (r.t + d * r.s);
            r.s *= f;
            r.m = m;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = (x[j] - m) * c, e = __builtin_amdgcn_exp2f(d);
            r.s += e;
            if (ENTROPY) r.t += e * fmaxf(d, LP_LEAST);
        }
    });
    return r;
}

// the workgroup's, in every thread
__device__ __forceinline__ Sums workgroup_sums(Sums r, Sums *waves, float c)
{
    r = joined(r, c);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = r;
    __syncthreads();
    r.m = fmaxf(fmaxf(waves[0].m, waves[1].m), fmaxf(waves[2].m, waves[3].m));
    r.s = r.t = 0.f;
#pragma unroll
    for (int w = 0; w < NWAVE; ++w) {
        const Sums o = about(waves[w], r.m, c);
        r.s += o.s;
        r.t += o.t;
    }
    return r;
}

// The workgroup's k largest keys into out[0 .. k), 0 where there are fewer.  order: of the thread's largest logit (or of a smaller one of its own), 0
// where it has none; only threads that have one of the candidates look at their logits again (`again`: those whose order may be too small do).
// Two bounds leave k candidates at least: the smallest over the waves of the k / 4-th largest order of a wave, and the largest over the waves of the
// k-th largest (which alone says something where the logits are too few for all waves).
template <typename T, bool WHOLE>
__device__ __forceinline__ void largest_keys(const T *line, int from, int to, int V, int k, uint32_t order, bool again, uint64_t *list, int *count, uint64_t *least, uint64_t *out)
{
    uint32_t *bounds = reinterpret_cast<uint32_t *>(out);
    uint32_t nth, kth;
    upper_halves(order, (k + NWAVE - 1) / NWAVE, k, nth, kth);
    if ((threadIdx.x & 63) == 0) {
        bounds[threadIdx.x >> 6] = nth;
        bounds[NWAVE + (threadIdx.x >> 6)] = kth;
    }
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t low = bounds[0];
#pragma unroll
        for (int w = 1; w < NWAVE; ++w) low = min(low, bounds[w]);
#pragma unroll
        for (int w = 0; w < NWAVE; ++w) low = max(low, bounds[NWAVE + w]);
        *least = low ? (uint64_t)low << 32 : 1;
    }
    __syncthreads();
    int n;
    for (;;) {
        const uint64_t bound = *least;
        const uint32_t high = (uint32_t)(bound >> 32);
        if (again || (order && order >= high))
            each_vector<T, WHOLE, LP_UNROLL>(line, from, to, V, [&](int v, const float (&x)[8]) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint64_t key = key_of(x[j], 8 * v + j);
                    if (key >= bound) {
                        const int at = atomicAdd(count, 1);
                        if (at < LP_LIST) list[at] = key;
                    }
                }
            });
        __syncthreads();
        n = *count;
        if (n <= LP_LIST) break;
        // more than the list takes: the k-th largest of those that it took is a closer bound
        uint64_t closer = 0;
        for (int i = threadIdx.x; i < LP_LIST; i += WG)
            if (rank_of(list, LP_LIST, list[i]) == k - 1) closer = list[i];
        __syncthreads();
        if (closer) *least = closer;
        if (threadIdx.x == 0) *count = 0;
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += WG) {
        const uint64_t key = list[i];
        const int r = rank_of(list, n, key);
        if (r < k) out[r] = key;
    }
    for (int i = n + threadIdx.x; i < k; i += WG) out[i] = 0;
}

template <typename T, bool TOP, bool ENTROPY, bool WHOLE>
__global__ __launch_bounds__(WG) void logprob_kernel(LogprobArgs a)
{
    __shared__ Sums waves[NWAVE];
    __shared__ __attribute__((aligned(16))) uint64_t list[TOP ? LP_LIST : 1];
    __shared__ uint64_t found[TOP ? LP_MOST_K : 1], least;
    static_assert(!TOP || LP_MOST_K >= NWAVE, "the bounds' room");
    __shared__ int count;
    const int64_t id = workgroup(), row = id / a.pieces;
    if (row >= a.rows) return;
    const int piece = (int)(id - row * a.pieces), from = piece * a.piece, to = min(from + a.piece, a.nv);
    const T *line = (const T *)a.logits + row * a.ld;
    const float c = a.scale * LOG2E;
    Given given{0.f, false};
    if (a.pieces == 1 && threadIdx.x == 0) given = given_logit<T>(a, row);
    Sums r = thread_sums<T, ENTROPY, WHOLE>(line, from, to, a.V, c);
    // a sum that is no number: a NaN among the logits, or an infinity (and maybe a NaN beside it)
    const bool odd = r.s != r.s;
    const uint32_t order = r.s == 0.f ? 0u : odd && r.m != INFINITY ? 0xffffffffu : order_of(r.m);
    r = workgroup_sums(r, waves, c);
    if (TOP) largest_keys<T, WHOLE>(line, from, to, a.V, a.k, order, odd, list, &count, &least, found);
    if (a.pieces > 1) {
        if (threadIdx.x == 0) *reinterpret_cast<float4 *>(a.sums + id * 4) = make_float4(r.m, r.s, r.t, 0.f);
        if (TOP) {
            __syncthreads();
            for (int i = threadIdx.x; i < a.k; i += WG) a.keys[id * a.k + i] = found[i];
        }
        return;
    }
    const float log_s = logf(r.s);
    if (threadIdx.x == 0) leave_row(a, row, r, log_s, given);
    if (TOP) {
        __syncthreads();
        for (int i = threadIdx.x; i < a.k; i += WG) leave_top(a, row, i, found[i], r.m, log_s);
    }
}

// A row's pieces joined, in their order: a workgroup of one wave per row without alternatives, with them of LP_JOIN threads.
// Where c pieces have t-th keys of a bound at least, and c t >= k, so have k of all keys: every wave looks for another t, and the largest bound leaves few
// more than k of the keys to be ranked.  (All of them, by searches in the pieces' lists: 24 rows of 22 pieces, k = 20, 8.4 us; so 4.9.)
constexpr int LP_JOIN = 1024;

template <typename T, bool TOP>
__global__ __launch_bounds__(TOP ? LP_JOIN : WAVE) void logprob_join_kernel(LogprobArgs a)
{
    __shared__ __attribute__((aligned(16))) uint64_t list[TOP ? LP_LIST : 1];
    __shared__ uint32_t bound;
    __shared__ int count;
    __shared__ float row_m, row_log_s;
    const int64_t row = workgroup();
    if (row >= a.rows) return;
    const float c = a.scale * LOG2E;
    const int n = a.pieces * a.k, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;      // (n: at most LP_LIST)
    uint64_t key = 0;
    uint32_t head = 0;
    const int t = TOP ? wave * a.k / (LP_JOIN / WAVE) : 0;       // (0 .. k - 1)
    if (TOP) {
        const uint64_t *keys = a.keys + row * n;
        if (threadIdx.x < n) key = keys[threadIdx.x];
        if (lane < a.pieces) head = (uint32_t)(keys[lane * a.k + t] >> 32);
        if (threadIdx.x == 0) bound = count = 0;
    }
    if (threadIdx.x < WAVE) {
        Given given{0.f, false};
        if (threadIdx.x == 0) given = given_logit<T>(a, row);
        Sums r{LP_LEAST, 0.f, 0.f};
        for (int p = threadIdx.x; p < a.pieces; p += WAVE) {
            const float4 s = *reinterpret_cast<const float4 *>(a.sums + (row * a.pieces + p) * 4);
            const Sums x{s.x, s.y, s.z};
            const float m = fmaxf(r.m, x.m);
            const Sums y = about(r, m, c), z = about(x, m, c);
            r = {m, y.s + z.s, y.t + z.t};
        }
        r = joined(r, c);
        if (threadIdx.x == 0) {
            row_m = r.m;
            row_log_s = logf(r.s);
            leave_row(a, row, r, row_log_s, given);
        }
    }
    if (!TOP) return;
    __syncthreads();
    uint32_t low, none;
    const int lists = (a.k + t) / (t + 1);
    if (lists <= min(a.pieces, WAVE)) {
        upper_halves(head, lists, WAVE, low, none);
        if (lane == 0 && low) atomicMax(&bound, low);
    }
    __syncthreads();
    if (key && (uint32_t)(key >> 32) >= bound) list[atomicAdd(&count, 1)] = key;
    __syncthreads();
    const int m = count;
    if ((int)threadIdx.x < m) {
        const uint64_t mine = list[threadIdx.x];
        const int r = rank_of(list, m, mine);
        if (r < a.k) leave_top(a, row, r, mine, row_m, row_log_s);
    }
    if ((int)threadIdx.x < a.k && (int)threadIdx.x >= m) leave_top(a, row, threadIdx.x, 0, row_m, row_log_s);
}

struct LogprobGradArgs {
    const void *logits, *tokens;
    void *out;
    int64_t ld, ld_out;
    const float *lse, *entropy, *g, *ge;
    int64_t rows;
    int tokens64, V, nv, pieces, piece;
    float scale;
};

// An lse beyond LP_FAR has lost 2^-12 of the sum that it holds, or more, and all of it where the row has nothing but its type's lowest value (which under a
// scale above 1 make it -inf).  There the row's first workgroup takes all of the row: it finds the largest logit and the sum once more and goes by these, if
// they are what the lse was made of; an lse of more columns than the row has is taken as it is.  The row's other workgroups do nothing, since out may be
// the logits, which are read as a whole before the first of them is written (4,096 x 50,257 in bfloat16 148 us, with a tenth of the rows of lowest values 178, with half of them 235).
constexpr float LP_FAR = 4096.f;

template <typename T, bool WHOLE>
__global__ __launch_bounds__(WG) void logprob_bwd_kernel(LogprobGradArgs a)
{
    __shared__ Sums waves[NWAVE];
    const int64_t id = workgroup(), row = id / a.pieces;
    if (row >= a.rows) return;
    const int piece = (int)(id - row * a.pieces), from = piece * a.piece, to = min(from + a.piece, a.nv);
    const T *line = (const T *)a.logits + row * a.ld;
    T *out = (T *)a.out + row * a.ld_out;
    // (what a row has is loaded together, whether it is there or not: one after the other they took as long as a short row's logits)
    const float lse = a.lse[row], at_g = (a.g ? a.g : a.lse)[row], at_ge = (a.ge ? a.ge : a.lse)[row], at_h = (a.ge ? a.entropy : a.lse)[row];
    int64_t token = -1;
    if (a.tokens && a.g) token = a.tokens64 ? ((const int64_t *)a.tokens)[row] : ((const int32_t *)a.tokens)[row];
    if (token < 0 || token >= a.V) token = -1;
    const float g = token >= 0 ? at_g : 0.f, ge = a.ge ? at_ge : 0.f, h = a.ge ? at_h : 0.f;
    // log p = scale (logit - m) - log_s
    auto leave = [&](int v, float (&x)[8], float m, float log_s, bool none) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float l = fmaf(x[j] - m, a.scale, -log_s), p = __builtin_amdgcn_exp2f(l * LOG2E);
            float d = -p * (g + (ge != 0.f && p != 0.f ? ge * (l + h) : 0.f));       // (p log p is 0 where p is, however large the log: masks of a type's lowest value)
            if (8 * v + j == token) d += g;
            x[j] = none || x[j] == -INFINITY ? 0.f : d * a.scale;
        }
        put8<WHOLE>(out + 8 * (int64_t)v, a.V - 8 * v, x);
    };
    const bool far = fabsf(lse) > LP_FAR;
    each_vector<T, WHOLE, LP_UNROLL>(line, from, to, a.V, [&](int v, float (&x)[8]) { leave(v, x, 0.f, lse, false); }, [&] { return !far; });
    if (!far || piece) return;
    const float c = a.scale * LOG2E;
    const Sums r = workgroup_sums(thread_sums<T, false, WHOLE, 1>(line, 0, a.nv, a.V, c), waves, c);
    const float log_r = logf(r.s), own = r.m * a.scale + log_r;
    const bool same = r.s > 0.f && (own == lse || fabsf(own - lse) < fabsf(lse) * 0x1p-22f);            // (sums in another order: a unit of the last place; < is false of infinities)
    const float m = same ? r.m : 0.f, log_s = same ? log_r : lse;
    each_vector<T, WHOLE, 1>(line, 0, a.nv, a.V, [&](int v, float (&x)[8]) { leave(v, x, m, log_s, !same && lse == -INFINITY); });
}

}  // namespace tt
