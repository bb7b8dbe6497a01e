// Token embedding: rows of a table by token, scaled, with dropout or without; and the table's gradient by sorted tokens.
//
// Forward: out[t] = m_t . (scale table[token_t]); a token outside [0, num_rows) is none and gets a row of zeros.
// Backward: G[v] = scale sum_{t: token_t = v} m_t . g[t], in 32 bits, in the order of t within a tile of sorted positions
// and tile after tile, so that the result is the same in every run; nothing is added with atomics.
// Both are bound by HBM; the gather reads whole rows, the gradient is one pass over g and one over the rows it writes.
#pragma once

#include "tt_rows_io.h"

namespace tt {

// ---- rows of one array to rows of another: gather, scaling, dropout, residual addition ---------------------------------

struct RowsArgs {
    const void *src, *residual;  // residual: of the source's type, or null
    void *dst;
    const void *tokens;          // null: row r of the source
    int64_t ld_src, ld_res, ld_dst, rows, num_rows;
    int N, nv, wide;             // columns, vectors per row, tokens of 64 bits
    float scale;
    DropArgs drop;
};

__device__ __forceinline__ int64_t token_at(const void *tokens, int wide, int64_t i)
{
    return wide ? ((const int64_t *)tokens)[i] : (int64_t)((const int32_t *)tokens)[i];
}

// tx threads (a power of two) along a row, WG / tx rows side by side, U rows per thread one after the other: their tokens
// are loaded together, then their vectors.
template <typename S, typename D, int U>
__global__ __launch_bounds__(WG) void rows_kernel(const RowsArgs a, int lg_tx)
{
    const int tx = 1 << lg_tx, ty = WG >> lg_tx;
    const int v = blockIdx.y * tx + (threadIdx.x & (tx - 1));
    if (v >= a.nv) return;
    const int64_t r0 = (int64_t)blockIdx.x * (ty * U) + (threadIdx.x >> lg_tx);
    const int n = a.N - 8 * v;
    const DropKey key = drop_key(a.drop);
    int64_t from[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * ty;
        from[u] = -1;
        if (r < a.rows) {
            from[u] = a.tokens ? token_at(a.tokens, a.wide, r) : r;
            if (from[u] >= a.num_rows) from[u] = -1;
        }
    }
    Vec8<S> x[U], res[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * ty;
        if (from[u] >= 0) x[u] = fetch8((const S *)a.src + from[u] * a.ld_src + 8 * v, n);
        if (a.residual && r < a.rows) res[u] = fetch8((const S *)a.residual + r * a.ld_res + 8 * v, n);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * ty;
        if (r >= a.rows) break;
        float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (from[u] >= 0) {
            widen8(x[u], y);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= a.scale;
        }
        if (a.drop.state) drop8(a.drop, drop_mask(a.drop, key, (uint64_t)r * (uint64_t)a.nv + (uint64_t)v), y);
        if (a.residual) {
            float z[8];
            widen8(res[u], z);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += z[j];
        }
        put8((D *)a.dst + r * a.ld_dst + 8 * v, n, y);
    }
}

// ---- stable sort of (token, position) ------------------------------------------------------------------------------

constexpr int TS_WG = 512, TS_SUB = 4, TS_TILE = TS_WG * TS_SUB;             // keys per workgroup and pass
constexpr int TS_BINS = 512;                                                // digits of up to 9 bits
constexpr int TS_WAVES = TS_WG / WAVE;
constexpr int TS_SCAN_TILES = 64;                                           // more tiles: their counts are scanned by a kernel

struct SortPass {
    const void *tokens;          // first pass: the keys come from here
    const uint32_t *kin, *vin;
    uint32_t *kout, *vout;
    uint32_t *hist;              // [tile][bin] counts; scanned: of the earlier tiles
    uint32_t *total;             // [bin], scanned only
    int64_t n;
    int64_t num_rows;
    int wide, shift, tiles;
};

// no token sorts behind all rows
__device__ __forceinline__ uint32_t sort_key(const SortPass &s, int64_t i)
{
    if (!s.tokens) return s.kin[i];
    const int64_t t = token_at(s.tokens, s.wide, i);
    return t >= 0 && t < s.num_rows ? (uint32_t)t : (uint32_t)s.num_rows;
}

__global__ __launch_bounds__(TS_WG) void token_hist_kernel(const SortPass s)
{
    __shared__ uint32_t h[TS_BINS];
    const int t = threadIdx.x;
    const int64_t base = (int64_t)blockIdx.x * TS_TILE;
    h[t] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < TS_SUB; ++q) {
        const int64_t i = base + q * TS_WG + t;
        if (i < s.n) atomicAdd(&h[(sort_key(s, i) >> s.shift) & (TS_BINS - 1)], 1u);
    }
    __syncthreads();
    s.hist[(int64_t)blockIdx.x * TS_BINS + t] = h[t];
}

// Counts become the counts of the earlier tiles.  64 bins a workgroup, 8 stretches of tiles side by side.
__global__ __launch_bounds__(TS_WG) void token_scan_kernel(const SortPass s)
{
    __shared__ uint32_t sum[TS_WAVES][WAVE];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int bin = blockIdx.x * WAVE + lane;
    const int per = (s.tiles + TS_WAVES - 1) / TS_WAVES;
    const int b0 = min(w * per, s.tiles), b1 = min(b0 + per, s.tiles);
    uint32_t mine = 0;
    for (int b = b0; b < b1; ++b) mine += s.hist[(int64_t)b * TS_BINS + bin];
    sum[w][lane] = mine;
    __syncthreads();
    uint32_t run = 0, all = 0;
    for (int q = 0; q < TS_WAVES; ++q) {
        if (q < w) run += sum[q][lane];
        all += sum[q][lane];
    }
    for (int b = b0; b < b1; ++b) {
        const uint32_t c = s.hist[(int64_t)b * TS_BINS + bin];
        s.hist[(int64_t)b * TS_BINS + bin] = run;
        run += c;
    }
    if (w == 0) s.total[bin] = all;
}

// Thread t works for bin t: where the bin starts (keys of smaller bins, then the bin's keys of earlier tiles), then the
// bin's places by (round, wave) of this tile; a key's rank among its wave's equal digits comes from ballots.
template <bool SCANNED>
__global__ __launch_bounds__(TS_WG) void token_scatter_kernel(const SortPass s)
{
    __shared__ uint16_t cnt[TS_SUB * TS_WAVES][TS_BINS];
    __shared__ uint32_t start[TS_BINS], wsum[TS_WAVES];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int64_t base = (int64_t)blockIdx.x * TS_TILE;
    uint32_t key[TS_SUB], pos[TS_SUB];
#pragma unroll
    for (int q = 0; q < TS_SUB; ++q) {
        const int64_t i = base + q * TS_WG + t;
        key[q] = i < s.n ? sort_key(s, i) : 0u;
        pos[q] = i < s.n && !s.tokens ? s.vin[i] : (uint32_t)i;
    }
    uint32_t all = 0, before = 0;
    if constexpr (SCANNED) {
        all = s.total[t];
        before = s.hist[(int64_t)blockIdx.x * TS_BINS + t];
    } else {
#pragma unroll 8
        for (int b = 0; b < s.tiles; ++b) {
            const uint32_t c = s.hist[b * TS_BINS + t];
            all += c;
            before += b < (int)blockIdx.x ? c : 0u;
        }
    }
    for (int g = 0; g < TS_SUB * TS_WAVES; ++g) cnt[g][t] = 0;
    uint32_t inc = all;
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) {
        const uint32_t o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == WAVE - 1) wsum[w] = inc;
    __syncthreads();
    uint32_t first = inc - all + before;
    for (int q = 0; q < w; ++q) first += wsum[q];
    int rank[TS_SUB];
#pragma unroll
    for (int q = 0; q < TS_SUB; ++q) {
        const bool in = base + q * TS_WG + t < s.n;
        const uint32_t dg = (key[q] >> s.shift) & (TS_BINS - 1);
        uint64_t same = __ballot(in);
#pragma unroll
        for (int b = 0; b < 9; ++b) {
            const bool bit = (dg >> b) & 1u;
            const uint64_t bal = __ballot(bit);
            same &= bit ? bal : ~bal;
        }
        rank[q] = __popcll(same & lanemask_lt());
        if (in && rank[q] == 0) cnt[q * TS_WAVES + w][dg] = (uint16_t)__popcll(same);
    }
    __syncthreads();
    {
        uint32_t run = 0;
        for (int g = 0; g < TS_SUB * TS_WAVES; ++g) {
            const uint32_t c = cnt[g][t];
            cnt[g][t] = (uint16_t)run;
            run += c;
        }
        start[t] = first;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < TS_SUB; ++q) {
        if (base + q * TS_WG + t >= s.n) continue;
        const uint32_t dg = (key[q] >> s.shift) & (TS_BINS - 1);
        const uint32_t to = start[dg] + cnt[q * TS_WAVES + w][dg] + (uint32_t)rank[q];
        s.kout[to] = key[q];
        s.vout[to] = pos[q];
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------------

// new row = old * table row (not read where old is 0) + sum * factor
struct GradArgs {
    const uint32_t *ks, *vs;     // sorted tokens and their positions
    const void *g;
    void *table;
    float *part;                 // [tile][2][nv * 8]
    int64_t ld_g, ld_table, n, num_rows;
    int N, nv, entries, tiles;   // entries per tile
    float factor;
    bool old;
    DropArgs drop;
};

template <typename O>
__device__ __forceinline__ void apply_row(const GradArgs &a, int64_t row, int v, const float (&sum)[8])
{
    O *p = (O *)a.table + row * a.ld_table + 8 * v;
    const int n = a.N - 8 * v;
    float y[8];
    if (a.old) {
        widen8(fetch8(p, n), y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = fmaf(sum[j], a.factor, y[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = sum[j] * a.factor;
    }
    put8(p, n, y);
}

// A tile of sorted entries for tx lanes, each with a vector of columns.  A run of equal tokens that lies inside the tile is
// applied here; the part of a run that goes on in the next tile is left in part[tile][1], the part of one that began in an
// earlier tile in part[tile][0].
template <typename G, typename O>
__global__ __launch_bounds__(WG) void token_grad_kernel(const GradArgs a, int lg_tx)
{
    constexpr int NB = 8;
    const int tx = 1 << lg_tx;
    const int tile = blockIdx.x * (WG >> lg_tx) + (threadIdx.x >> lg_tx);
    const int v = blockIdx.y * tx + (threadIdx.x & (tx - 1));
    if (tile >= a.tiles || v >= a.nv) return;
    const int64_t i0 = (int64_t)tile * a.entries;
    const int cnt = (int)(a.n - i0 < a.entries ? a.n - i0 : a.entries);
    const uint32_t none = (uint32_t)a.num_rows;
    uint32_t cur = a.ks[i0];
    if (cur == none) return;
    const uint32_t next = i0 + cnt < a.n ? a.ks[i0 + cnt] : none;
    bool first = i0 > 0 && a.ks[i0 - 1] == cur;              // the first run began in an earlier tile
    const DropKey dk = drop_key(a.drop);
    const int n = a.N - 8 * v;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto flush = [&](bool goes_on) {
        if (first || goes_on) {
            float *p = a.part + ((int64_t)tile * 2 + (first ? 0 : 1)) * (8 * a.nv) + 8 * v;
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = sum[j];
        } else {
            apply_row<O>(a, cur, v, sum);
        }
        first = false;
    };
    for (int e0 = 0; e0 < cnt; e0 += NB) {
        uint32_t key[NB], pos[NB];
        Vec8<G> x[NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            const int e = min(e0 + q, cnt - 1);
            key[q] = a.ks[i0 + e];
            pos[q] = a.vs[i0 + e];
        }
#pragma unroll
        for (int q = 0; q < NB; ++q) x[q] = fetch8((const G *)a.g + (int64_t)pos[q] * a.ld_g + 8 * v, n);
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            if (e0 + q >= cnt) break;
            if (key[q] != cur) {
                flush(false);
                cur = key[q];
                if (cur == none) return;                     // what is left has no token
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = 0.f;
            }
            float y[8];
            widen8(x[q], y);
            if (a.drop.state) drop8(a.drop, drop_mask(a.drop, dk, (uint64_t)pos[q] * (uint64_t)a.nv + (uint64_t)v), y);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += y[j];
        }
    }
    flush(cur == next);
}

// A run that crosses tiles is put together by the workgroup of the tile where it begins: its part[tile][1], then
// part[u][0] of the later tiles u that it reaches; the workgroup's WG / tx groups of lanes take every (WG / tx)-th of them,
// and their sums are added in the groups' order.
template <typename O>
__global__ __launch_bounds__(WG) void token_join_kernel(const GradArgs a, int lg_tx)
{
    __shared__ float lds[WG * 8];
    const int tile = blockIdx.x;
    const int64_t i0 = (int64_t)tile * a.entries, i1 = i0 + a.entries;
    if (i1 >= a.n) return;
    const uint32_t key = a.ks[i1 - 1];
    if (key == (uint32_t)a.num_rows || a.ks[i1] != key) return;              // no token, or the run ends with the tile
    if (i0 > 0 && a.ks[i0] == key && a.ks[i0 - 1] == key) return;            // it began in an earlier tile
    int lo = tile + 1, hi = a.tiles;                         // the tiles whose first entry is of the run: [tile + 1, lo) at the end
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (a.ks[(int64_t)mid * a.entries] == key) lo = mid + 1; else hi = mid;
    }
    const int tx = 1 << lg_tx, groups = WG >> lg_tx, gi = threadIdx.x >> lg_tx, v = blockIdx.y * tx + (threadIdx.x & (tx - 1));
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (v < a.nv) {
        if (gi == 0) {
            const float *p = a.part + ((int64_t)tile * 2 + 1) * (8 * a.nv) + 8 * v;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] = p[j];
        }
#pragma unroll 4
        for (int u = tile + 1 + gi; u < lo; u += groups) {
            const float *p = a.part + (int64_t)u * 2 * (8 * a.nv) + 8 * v;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += p[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[j * WG + threadIdx.x] = sum[j];
    __syncthreads();
    if (gi || v >= a.nv) return;
    for (int q = 1; q < groups; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += lds[j * WG + q * tx + threadIdx.x];
    apply_row<O>(a, key, v, sum);
}

// Rows that no token names are zero: a wave looks up 16 neighbouring rows in the sorted tokens and clears the absent ones.
constexpr int TZ_ROWS = 16;

template <typename O>
__global__ __launch_bounds__(WG) void token_zero_kernel(const GradArgs a, int lg_tx)
{
    const int lane = threadIdx.x & 63, tx = 1 << lg_tx;
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int64_t step = (int64_t)gridDim.x * NWAVE * TZ_ROWS;
    for (int64_t v0 = ((int64_t)blockIdx.x * NWAVE + (threadIdx.x >> 6)) * TZ_ROWS; v0 < a.num_rows; v0 += step) {
        const int64_t row = v0 + lane;
        bool absent = false;
        if (lane < TZ_ROWS && row < a.num_rows) {
            int64_t lo = 0, hi = a.n;
            while (lo < hi) {
                const int64_t mid = (lo + hi) >> 1;
                if ((int64_t)a.ks[mid] < row) lo = mid + 1; else hi = mid;
            }
            absent = lo >= a.n || (int64_t)a.ks[lo] != row;
        }
        const uint32_t clear = (uint32_t)__ballot(absent);
        for (int r = lane >> lg_tx; r < TZ_ROWS; r += WAVE >> lg_tx) {
            if (!((clear >> r) & 1u)) continue;
            for (int v = lane & (tx - 1); v < a.nv; v += tx) put8((O *)a.table + (v0 + r) * a.ld_table + 8 * v, a.N - 8 * v, zero);
        }
    }
}

}  // namespace tt
