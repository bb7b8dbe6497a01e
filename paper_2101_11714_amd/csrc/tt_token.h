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
    float scale;                 // with the dropout's factor
    DropArgs drop;
};

__device__ __forceinline__ int64_t token_at(const void *tokens, int wide, int64_t i)
{
    return wide ? ((const int64_t *)tokens)[i] : (int64_t)((const int32_t *)tokens)[i];
}

// tx threads (a power of two) along a row, WG / tx rows side by side, U rows per thread.  No load stands in a branch: what is loaded
// there is waited for there, one load after the other; a row or a token that does not exist reads the first one instead.
// U = 1 for dropout alone (U = 2 and 4 took 10 and 20 % longer: more workgroups hide more than longer ones), 2 for lookups, whose
// loads wait for the tokens.
template <typename S, typename D, int U, bool WHOLE, bool TOKENS, bool RESIDUAL>
__global__ __launch_bounds__(WG) void rows_kernel(const RowsArgs a, int lg_tx)
{
    const int tx = 1 << lg_tx, ty = WG >> lg_tx;
    const int v = blockIdx.y * tx + (threadIdx.x & (tx - 1));
    if (v >= a.nv) return;
    const int64_t r0 = (int64_t)blockIdx.x * (ty * U) + (threadIdx.x >> lg_tx);
    const int n = a.N - 8 * v;
    const DropKey key = drop_key(a.drop);
    int64_t from[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * ty;
        from[u] = r < a.rows ? r : 0;
        there[u] = true;
        if constexpr (TOKENS) {
            const int64_t t = token_at(a.tokens, a.wide, from[u]);
            there[u] = t >= 0 && t < a.num_rows;
            from[u] = there[u] ? t : 0;
        }
    }
    Vec8<S> x[U], res[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * ty;
        x[u] = fetch8<WHOLE>((const S *)a.src + row_at(from[u], a.ld_src) + 8 * v, n);
        if constexpr (RESIDUAL) res[u] = fetch8<WHOLE>((const S *)a.residual + row_at(r < a.rows ? r : 0, a.ld_res) + 8 * v, n);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * ty;
        if (r >= a.rows) break;
        float y[8];
        widen8(x[u], y);
        if (a.drop.state) {
            drop8(a.drop, key, (uint64_t)row_at(r, a.nv) + (uint64_t)v, a.scale, y);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= a.scale;
        }
        if constexpr (TOKENS) {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = there[u] ? y[j] : 0.f;
        }
        if constexpr (RESIDUAL) {
            float z[8];
            widen8(res[u], z);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += z[j];
        }
        put8<WHOLE>((D *)a.dst + row_at(r, a.ld_dst) + 8 * v, n, y);
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

// Up to 8,192 tokens: the whole sort in one workgroup, in LDS.  A wave owns R * 64 neighbouring entries and ranks 64 of them at a
// time among the wave's earlier ones with the same digit; the counts by (digit, wave) become starting places.  One launch instead
// of two per digit.  Not beyond: one workgroup took 48 us for 16,384 tokens of 1,000,000 rows, the launches per digit 32.
constexpr int TO_WG = 1024, TO_WAVES = TO_WG / WAVE, TO_BINS = 256, TO_MOST = 8 * TO_WG;

static inline size_t sort_one_lds(int R) { return (size_t)R * TO_WG * 6 + (size_t)TO_WAVES * TO_BINS * 4 + 32; }

template <int R>
__global__ __launch_bounds__(TO_WG) void token_sort_one_kernel(const SortPass s, int passes)
{
    extern __shared__ uint32_t lds_u32[];
    uint32_t *keys = lds_u32, *cnt = keys + R * TO_WG;       // cnt[wave][digit]
    uint32_t *wsum = cnt + TO_WAVES * TO_BINS;
    uint16_t *poss = (uint16_t *)(wsum + 8);
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, n = (int)s.n;
    uint32_t key[R], pos[R];                                 // pos: and, in the high half, the rank
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = (w * R + r) * WAVE + lane;
        key[r] = i < n ? sort_key(s, i) : 0xffffffffu;       // places without a token sort behind all
        pos[r] = (uint32_t)i;
    }
    for (int pass = 0, shift = 0; pass < passes; ++pass, shift += 8) {
        uint32_t *mine = cnt + w * TO_BINS;
#pragma unroll
        for (int q = 0; q < TO_BINS / WAVE; ++q) mine[q * WAVE + lane] = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t dg = (key[r] >> shift) & (TO_BINS - 1);
            uint64_t same = ~0ull;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const bool bit = (dg >> b) & 1u;
                const uint64_t bal = __ballot(bit);
                same &= bit ? bal : ~bal;
            }
            const int rank = __popcll(same & lanemask_lt());
            const uint32_t before = mine[dg];                // (a wave's LDS accesses are done in their order)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (rank == 0) mine[dg] = before + (uint32_t)__popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            pos[r] |= (before + (uint32_t)rank) << 16;
        }
        __syncthreads();
        if (t < TO_BINS) {
            uint32_t c[TO_WAVES], all = 0;
#pragma unroll
            for (int q = 0; q < TO_WAVES; ++q) {
                c[q] = cnt[q * TO_BINS + t];
                all += c[q];
            }
            uint32_t inc = all;
#pragma unroll
            for (int d = 1; d < WAVE; d <<= 1) {
                const uint32_t o = __shfl_up(inc, d);
                if (lane >= d) inc += o;
            }
            if (lane == WAVE - 1) wsum[w] = inc;
            uint32_t run = inc - all;
#pragma unroll
            for (int q = 0; q < TO_WAVES; ++q) {
                cnt[q * TO_BINS + t] = run;
                run += c[q];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t dg = (key[r] >> shift) & (TO_BINS - 1);
            uint32_t to = mine[dg] + (pos[r] >> 16);
            for (uint32_t q = 0; q < dg >> 6; ++q) to += wsum[q];
            keys[to] = key[r];
            poss[to] = (uint16_t)pos[r];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = (w * R + r) * WAVE + lane;
            key[r] = keys[i];
            pos[r] = poss[i];
        }
        // (the next pass writes cnt, which nobody reads any more, and keys only behind its barriers)
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = (w * R + r) * WAVE + lane;
        if (i < n) {
            s.kout[i] = key[r];
            s.vout[i] = pos[r];
        }
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------------

constexpr int TG_LEAST_LG = 2, TG_ENTRIES = 32;              // lanes per tile (log), entries per tile: least and most
constexpr int TG_MOST = (WG >> TG_LEAST_LG) * TG_ENTRIES;

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

template <typename O, bool WHOLE>
__device__ __forceinline__ void apply_row(const GradArgs &a, int64_t row, int v, const float (&sum)[8])
{
    O *p = (O *)a.table + row_at(row, a.ld_table) + 8 * v;
    const int n = a.N - 8 * v;
    float y[8];
    if (a.old) {
        widen8(fetch8<WHOLE>(p, n), y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = fmaf(sum[j], a.factor, y[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = sum[j] * a.factor;
    }
    put8<WHOLE>(p, n, y);
}

// The first place of the sorted tokens whose token is at least `row`, found by a wave 64 places at a time.
__device__ __forceinline__ int64_t first_at_least(const uint32_t *ks, int64_t n, uint32_t row)
{
    int64_t lo = 0, len = n;                                 // the answer is in [lo, lo + len]
    const int lane = threadIdx.x & 63;
    while (len > 0) {
        const int64_t step = (len + WAVE - 1) / WAVE;
        const int64_t i = lo + (int64_t)lane * step;         // the last place of the lane's stretch decides
        const int64_t last = i + step - 1 < lo + len - 1 ? i + step - 1 : lo + len - 1;
        const bool below = i < lo + len && ks[last] < row;
        const int k = __popcll(__ballot(below));             // whole stretches below `row`
        const int64_t at = lo + k * step;
        if (at >= lo + len) return lo + len;
        len = step < lo + len - at ? step : lo + len - at;
        lo = at;
        if (len == 1) return lo;                             // its one place is not below
        len -= 1;                                            // the last place of the stretch is known not to be
    }
    return lo;
}

constexpr int TZ_MOST = 1024;                                // rows of a clearing workgroup, at most

// Rows that no token names are zero.  A workgroup takes `rows` neighbouring ones, marks those that occur among the sorted tokens
// in LDS and clears the others, 16 bytes a thread; 64 KB or so, so that the workgroups at work sweep through memory together.
template <typename O>
__device__ __forceinline__ void clear_absent(const GradArgs &a, int64_t block, int rows, uint32_t *marks, int64_t *range)
{
    constexpr int E = 16 / sizeof(O);
    struct __attribute__((packed, aligned(sizeof(O)))) Piece { O v[E]; };
    const int64_t v0 = block * rows, v1 = v0 + rows < a.num_rows ? v0 + rows : a.num_rows;
    const int t = threadIdx.x, w = t >> 6;
    if (t < TZ_MOST / 32) marks[t] = 0;
    if (w < 2) {
        const int64_t at = first_at_least(a.ks, a.n, (uint32_t)(w ? v1 : v0));
        if ((t & 63) == 0) range[w] = at;
    }
    __syncthreads();
    for (int64_t i = range[0] + t; i < range[1]; i += WG) {
        const uint32_t r = a.ks[i] - (uint32_t)v0;
        if (!((marks[r >> 5] >> (r & 31)) & 1u)) atomicOr(&marks[r >> 5], 1u << (r & 31));
    }
    __syncthreads();
    const int pieces = (a.N + E - 1) / E;
    int lg = 0;
    while (lg < 8 && (1 << lg) < pieces) ++lg;
    const Piece zero{};
    for (int r = t >> lg; r < (int)(v1 - v0); r += WG >> lg) {
        if ((marks[r >> 5] >> (r & 31)) & 1u) continue;
        O *p = (O *)a.table + (v0 + r) * a.ld_table;
        for (int c = t & ((1 << lg) - 1); c < pieces; c += 1 << lg) {
            const int n = a.N - E * c;
            if (n >= E) {
                *reinterpret_cast<Piece *>(p + E * c) = zero;
            } else {
                for (int j = 0; j < n; ++j) p[E * c + j] = (O)0.f;
            }
        }
    }
}

// A tile of sorted entries for tx lanes, each with a vector of columns.  A run of equal tokens that lies inside the tile is
// applied here; the part of a run that goes on in the next tile is left in part[tile][1], the part of one that began in an
// earlier tile in part[tile][0].  The workgroups behind the tiles' clear the rows that no token names.
template <typename G, typename O, bool WHOLE>
__global__ __launch_bounds__(WG) void token_grad_kernel(const GradArgs a, int lg_tx, int chunks, int64_t tile_blocks, int clear_rows)
{
    constexpr int NB = 8;
    __shared__ uint32_t marks[TZ_MOST / 32];
    __shared__ int64_t range[2];
    __shared__ uint32_t keys[TG_MOST + 2], poss[TG_MOST + 2];
    if ((int64_t)blockIdx.x >= tile_blocks) {
        for (int64_t b = (int64_t)blockIdx.x - tile_blocks; b * clear_rows < a.num_rows; b += (int64_t)gridDim.x - tile_blocks) {
            clear_absent<O>(a, b, clear_rows, marks, range);
            __syncthreads();
        }
        return;
    }
    const int tx = 1 << lg_tx, in_wg = WG >> lg_tx;
    const int tile0 = (int)(blockIdx.x / (unsigned)chunks) * in_wg, tile = tile0 + (threadIdx.x >> lg_tx);
    const int v = (int)(blockIdx.x % (unsigned)chunks) * tx + (threadIdx.x & (tx - 1));
    const uint32_t none = (uint32_t)a.num_rows;
    {   // the workgroup's entries, and the ones beside them
        const int64_t first = (int64_t)tile0 * a.entries - 1;
        for (int e = threadIdx.x; e < in_wg * a.entries + 2; e += WG) {
            const int64_t i = first + e;
            const bool in = i >= 0 && i < a.n;
            keys[e] = in ? a.ks[i] : none;
            poss[e] = in ? a.vs[i] : 0u;
        }
    }
    __syncthreads();
    if (tile >= a.tiles || v >= a.nv) return;
    const int64_t i0 = (int64_t)tile * a.entries;
    const int cnt = (int)(a.n - i0 < a.entries ? a.n - i0 : a.entries);
    const uint32_t *tk = keys + (tile - tile0) * a.entries + 1, *tp = poss + (tile - tile0) * a.entries + 1;
    uint32_t cur = tk[0];
    if (cur == none) return;
    bool first = i0 > 0 && tk[-1] == cur;                    // the first run began in an earlier tile
    const DropKey dk = drop_key(a.drop);
    const int n = a.N - 8 * v;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto flush = [&](bool goes_on) {
        if (first || goes_on) {
            float *p = a.part + ((int64_t)tile * 2 + (first ? 0 : 1)) * (8 * a.nv) + 8 * v;
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = sum[j];
        } else {
            apply_row<O, WHOLE>(a, cur, v, sum);
        }
        first = false;
    };
    for (int e0 = 0; e0 < cnt; e0 += NB) {
        Vec8<G> x[NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) x[q] = fetch8<WHOLE>((const G *)a.g + row_at(tp[min(e0 + q, cnt - 1)], a.ld_g) + 8 * v, n);
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            if (e0 + q >= cnt) break;
            const uint32_t key = tk[e0 + q];
            if (key != cur) {
                flush(false);
                cur = key;
                if (cur == none) return;                     // what is left has no token
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = 0.f;
            }
            float y[8];
            widen8(x[q], y);
            if (a.drop.state) drop8(a.drop, dk, (uint64_t)row_at(tp[e0 + q], a.nv) + (uint64_t)v, 1.f, y);   // (a.factor has the dropout's)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += y[j];
        }
    }
    flush(tk[cnt] == cur);                                   // (behind the last entry of all: no token)
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
    apply_row<O, false>(a, key, v, sum);
}

}  // namespace tt
