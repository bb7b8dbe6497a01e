// Token embedding: rows of a table by token, scaled, with dropout or without; and the table's gradient by sorted tokens.
//
// Forward: out[t] = m_t . (scale table[token_t]); a token outside [0, num_rows) is none and gets a row of zeros.
// Backward: G[v] = scale sum_{t: token_t = v} m_t . g[t], in 32 bits: in the order of t within a tile of sorted positions, the tiles' sums by
// groups of lanes that take every so many-th of them each, the groups' sums in their order (few tokens: the positions by such groups).  The order
// depends on the tokens alone, so that the result is the same in every run; nothing is added with atomics.
// Both are bound by HBM where there is work; the gather reads whole rows, the gradient is one pass over g and one over the rows it
// writes.  32,768 tokens of 4,096 columns in 16 bits: lookup with dropout 74 us (4.9 TB/s of distinct rows and output), gradient of
// 131,072 rows in 32 bits 478 us (5.0 TB/s), of which sorting takes 25 and joining 13.
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
    double nv_d, inv_nv, half_nv;            // nv, 1 / nv, 0.5 / nv
    float scale;                 // with the dropout's factor
    DropArgs drop;
};

__device__ __forceinline__ int64_t token_at(const void *tokens, int wide, int64_t i)
{
    return wide ? ((const int64_t *)tokens)[i] : (int64_t)((const int32_t *)tokens)[i];
}

// A thread per vector, in the order of the rows, U of them per thread, WG apart; a vector's number is parted into row and place in
// 64-bit floating point (exact below 2^51; one division of whole numbers would take longer than all the rest).  No load stands in a
// branch: what is loaded there is waited for there, one load after the other; a row or a token that does not exist reads the first
// one instead.
// U = 1 for dropout alone (2 and 4 took 10 and 20 % longer: more workgroups hide more than longer ones), more for lookups, whose
// loads wait for the tokens.
template <typename S, typename D, int U, bool WHOLE, bool TOKENS, bool RESIDUAL>
__global__ __launch_bounds__(WG) void rows_kernel(const RowsArgs a)
{
    int64_t row[U];
    int v[U], n[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const double i = (double)workgroup() * (double)(U * WG) + (double)(u * WG + (int)threadIdx.x);
        const double r = floor(fma(i, a.inv_nv, a.half_nv));
        row[u] = (int64_t)(uint32_t)r;                       // (behind the last row: cut off where it is looked at)
        v[u] = (int)fma(-r, a.nv_d, i);
        n[u] = a.N - 8 * v[u];
    }
    const DropKey key = drop_key(a.drop);
    int64_t from[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        from[u] = row[u] < a.rows ? row[u] : 0;
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
        x[u] = fetch8<WHOLE>((const S *)a.src + row_at(from[u], a.ld_src) + 8 * v[u], n[u], a.N);
        if constexpr (RESIDUAL) res[u] = fetch8<WHOLE>((const S *)a.residual + row_at(row[u] < a.rows ? row[u] : 0, a.ld_res) + 8 * v[u], n[u], a.N);
    }
    DropWords words[U];                                      // (while the vectors are on their way)
    if (a.drop.state) {
#pragma unroll
        for (int u = 0; u < U; ++u) words[u] = drop_words(a.drop, key, (uint64_t)row_at(row[u], a.nv) + (uint64_t)v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (row[u] >= a.rows) break;
        if constexpr (TOKENS) keep8(there[u], x[u]);
        const float scale = !TOKENS || there[u] ? a.scale : 0.f;     // (zeros by any scale)
        float y[8];
        settle8<WHOLE>(x[u], n[u], a.N);
        widen8(x[u], y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= scale;
        if (a.drop.state) drop8(a.drop, words[u], y);
        if constexpr (RESIDUAL) {
            float z[8];
            settle8<WHOLE>(res[u], n[u], a.N);
            widen8(res[u], z);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += z[j];
        }
        put8<WHOLE>((D *)a.dst + row_at(row[u], a.ld_dst) + 8 * v[u], n[u], y);
    }
}

// ---- stable sort of (token, position) ------------------------------------------------------------------------------

// By digits of up to 10 bits, low ones first, as few passes as that allows.  Counts of the tiles added up by each workgroup itself / scanned by
// a kernel, gradient of 64 columns: 16 tiles 37 / 39 us, 32 46 / 48, 64 61 / 61, 128 91 / 85, 256 128 / 113.
constexpr int TS_WG = 1024, TS_SUB = 2, TS_TILE = TS_WG * TS_SUB;           // keys per workgroup and pass
constexpr int TS_BITS = 10, TS_BINS = 1 << TS_BITS;
constexpr int TS_WAVES = TS_WG / WAVE;
constexpr int TS_SCAN_TILES = 64;                                           // more tiles: their counts are scanned by a kernel
static_assert(TS_BINS == TS_WG, "a thread per bin");

struct SortPass {
    const void *tokens;          // first pass: the keys come from here
    const uint32_t *kin, *vin;
    uint32_t *kout, *vout;
    uint32_t *hist;              // [tile][bin] counts; scanned: of the earlier tiles
    uint32_t *total;             // [bin], scanned only
    uint8_t *named;              // a byte per row, or null: cleared by the first kernel, set by the next one
    bool blank;                  // (by this kernel)
    int64_t n;
    int64_t num_rows;
    int wide, shift, bits, tiles;
};

// (16-byte aligned, with room up to a multiple of 16)
__device__ __forceinline__ void blank_named(const SortPass &s)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; 16 * i < s.num_rows; i += (int64_t)gridDim.x * blockDim.x)
        reinterpret_cast<uint4 *>(s.named)[i] = make_uint4(0u, 0u, 0u, 0u);
}

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
    if (s.blank) blank_named(s);
    h[t] = 0;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < TS_SUB; ++q) {
        const int64_t i = base + q * TS_WG + t;
        if (i < s.n) atomicAdd(&h[(sort_key(s, i) >> s.shift) & ((1u << s.bits) - 1u)], 1u);
    }
    __syncthreads();
    s.hist[(int64_t)blockIdx.x * TS_BINS + t] = h[t];
}

// Counts become the counts of the earlier tiles.  64 bins a workgroup, a stretch of the tiles per wave.
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

// Among a wave's lanes that are `in`: how many have this lane's digit, in lower lanes (low half) and in all (high half).
__device__ __forceinline__ uint32_t rank_digit(uint32_t digit, int bits, bool in)
{
    const uint64_t there = __ballot(in);
    uint32_t lo = (uint32_t)there, hi = (uint32_t)(there >> 32);
#pragma unroll
    for (int b = 0; b < TS_BITS; ++b) {
        if (b < bits) {                                      // uniform
            const int set = (int)(digit << (31 - b)) >> 31;  // all ones, or none
            const uint64_t bal = __ballot(set != 0);
            lo = __builtin_amdgcn_bitop3_b32(lo, (uint32_t)bal, (uint32_t)set, 0x90);    // lo & ~(bal ^ set)
            hi = __builtin_amdgcn_bitop3_b32(hi, (uint32_t)(bal >> 32), (uint32_t)set, 0x90);
        }
    }
    const uint32_t lower = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0u));
    return lower | (uint32_t)(__popc(lo) + __popc(hi)) << 16;
}

// The place of a key among its wave's keys of its digit: those that the wave counted before, then the lower lanes'.  `mine`: the
// wave's own counts in LDS, which it reads and writes in its own order.
__device__ __forceinline__ uint32_t count_digit(uint16_t *mine, uint32_t digit, uint32_t rank, bool in)
{
    const uint32_t before = in ? mine[digit] : 0u;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (in && (rank & 0xffffu) == 0) mine[digit] = (uint16_t)(before + (rank >> 16));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return before + (rank & 0xffffu);
}

// Places of the keys of a workgroup of TS_WG threads, R per thread, whose wave w owns R * 64 neighbouring ones, by digit, then by
// (wave, round, lane): place[r] = start of the key's digit + its place there.  before_me: of thread t, keys of digit t that are not this
// workgroup's and come first; all_keys: all keys of digit t (0, 0 where there is one workgroup).  cnt: [wave][digit], wsum: [wave].
template <int R>
__device__ __forceinline__ void places(const uint32_t (&digit)[R], const bool (&in)[R], int bits, bool one, uint32_t all_keys, uint32_t before_me,
                                       uint16_t *cnt, uint32_t *start, uint32_t *wsum, uint32_t (&place)[R])
{
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    uint16_t *mine = cnt + w * TS_BINS;
#pragma unroll
    for (int q = 0; q < TS_BINS / WAVE / 2; ++q) reinterpret_cast<uint32_t *>(mine)[q * WAVE + lane] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int r = 0; r < R; ++r) place[r] = rank_digit(digit[r], bits, in[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) place[r] = count_digit(mine, digit[r], place[r], in[r]);
    __syncthreads();
    uint32_t c[TS_WAVES], own = 0;
#pragma unroll
    for (int q = 0; q < TS_WAVES; ++q) {
        c[q] = cnt[q * TS_BINS + t];
        own += c[q];
    }
    const uint32_t all = one ? own : all_keys;
    uint32_t inc = all;
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) {
        const uint32_t o = __shfl_up(inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == WAVE - 1) wsum[w] = inc;
    uint32_t run = 0;
#pragma unroll
    for (int q = 0; q < TS_WAVES; ++q) {
        cnt[q * TS_BINS + t] = (uint16_t)run;
        run += c[q];
    }
    __syncthreads();
    uint32_t first = inc - all + before_me;
    for (int q = 0; q < w; ++q) first += wsum[q];
    start[t] = first;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) place[r] += start[digit[r]] + mine[digit[r]];
}

template <bool SCANNED>
__global__ __launch_bounds__(TS_WG) void token_scatter_kernel(const SortPass s)
{
    __shared__ uint32_t start[TS_BINS], wsum[TS_WAVES];
    __shared__ __align__(16) uint16_t cnt[TS_WAVES * TS_BINS];
    const int t = threadIdx.x;
    const int64_t base = (int64_t)blockIdx.x * TS_TILE + (t >> 6) * (TS_SUB * WAVE) + (t & 63);
    uint32_t key[TS_SUB], pos[TS_SUB], digit[TS_SUB], place[TS_SUB];
    bool in[TS_SUB];
#pragma unroll
    for (int q = 0; q < TS_SUB; ++q) {
        const int64_t i = base + q * WAVE;
        in[q] = i < s.n;
        key[q] = in[q] ? sort_key(s, i) : 0u;
        pos[q] = in[q] && !s.tokens ? s.vin[i] : (uint32_t)i;
        digit[q] = (key[q] >> s.shift) & ((1u << s.bits) - 1u);
        if (s.named && in[q] && key[q] < (uint32_t)s.num_rows) s.named[key[q]] = 1;
    }
    uint32_t all = 0, before = 0;
    if constexpr (SCANNED) {
        all = s.total[t];
        before = s.hist[(int64_t)blockIdx.x * TS_BINS + t];
    } else {
        for (int b0 = 0; b0 < s.tiles; b0 += 16) {
            uint32_t c[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) c[q] = s.hist[min(b0 + q, s.tiles - 1) * TS_BINS + t];
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                all += b0 + q < s.tiles ? c[q] : 0u;
                before += b0 + q < (int)blockIdx.x ? c[q] : 0u;
            }
        }
    }
    places<TS_SUB>(digit, in, s.bits, false, all, before, cnt, start, wsum, place);
#pragma unroll
    for (int q = 0; q < TS_SUB; ++q) {
        if (!in[q]) continue;
        s.kout[place[q]] = key[q];
        s.vout[place[q]] = pos[q];
    }
}

// Few tokens: the whole sort in one workgroup, in LDS.  One launch instead of two per digit: 13 us for 4,093 tokens of 50,001 rows, where
// four launches take 24; 37 us for 16,384 (an earlier form), where they take 22.
constexpr int TO_MOST = 8 * TS_WG;

static inline size_t sort_one_lds(int R) { return (size_t)R * TS_WG * 6 + (size_t)TS_WAVES * TS_BINS * 2 + TS_BINS * 4 + TS_WAVES * 4; }

template <int R>
__global__ __launch_bounds__(TS_WG) void token_sort_one_kernel(const SortPass s, int passes)
{
    extern __shared__ uint32_t lds_u32[];
    uint32_t *keys = lds_u32, *start = keys + R * TS_WG, *wsum = start + TS_BINS;
    uint16_t *cnt = (uint16_t *)(wsum + TS_WAVES), *poss = cnt + TS_WAVES * TS_BINS;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = (int)s.n;
    if (s.blank) blank_named(s);                             // (before the marks behind the next barrier)
    uint32_t key[R], pos[R], digit[R], place[R];
    bool in[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = (w * R + r) * WAVE + lane;
        in[r] = i < n;                                       // (the places behind stay where they are)
        key[r] = in[r] ? sort_key(s, i) : 0u;
        pos[r] = (uint32_t)i;
    }
    for (int pass = 0; pass < passes; ++pass) {
#pragma unroll
        for (int r = 0; r < R; ++r) digit[r] = (key[r] >> (pass * s.bits)) & ((1u << s.bits) - 1u);
        places<R>(digit, in, s.bits, true, 0u, 0u, cnt, start, wsum, place);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!in[r]) continue;
            keys[place[r]] = key[r];
            poss[place[r]] = (uint16_t)pos[r];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = (w * R + r) * WAVE + lane;
            key[r] = keys[i];
            pos[r] = poss[i];
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (!in[r]) continue;
        const int i = (w * R + r) * WAVE + lane;
        s.kout[i] = key[r];
        s.vout[i] = pos[r];
        if (s.named && key[r] < (uint32_t)s.num_rows) s.named[key[r]] = 1;
    }
}

// ---- gradient -------------------------------------------------------------------------------------------------------

constexpr int TG_LEAST_LG = 2;                               // lanes per tile (log), at least
constexpr int TG_MOST = 2048;                                // entries of a workgroup, at most

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
        Vec8<O> x = fetch8<WHOLE>(p, n, a.N);
        settle8<WHOLE>(x, n, a.N);
        widen8(x, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = fmaf(sum[j], a.factor, y[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = sum[j] * a.factor;
    }
    put8<WHOLE>(p, n, y);
}

// Rows that no token names are zero.  A byte per row says which are named (bytes, since any number of tokens can set one without an
// atomic).  A workgroup clears TZ_SWEEPS neighbouring parts of WG * 32 bytes, and is done.  The stores' order decides: clearing
// 2 GB in the order of the addresses, 16 bytes a thread and nothing else, runs at 6.85 TB/s; with a byte to be looked at first, parts
// per workgroup 1 / 2 / 4 / 8: 5.3 / 5.6 / 6.4 / 5.5 TB/s.
constexpr int TZ_SWEEPS = 4;

__global__ __launch_bounds__(WG) void token_blank_kernel(const SortPass s) { blank_named(s); }

struct ClearArgs {
    const uint8_t *named;
    uint32_t parts, chunks;      // parts of WG * 32 bytes; of a row (or rows side by side in one part)
    int lg;                      // threads along a row (log)
};

// TZ_SWEEPS parts of the table, the rows but those that named(row) names
template <typename O, typename F>
__device__ __forceinline__ void clear_rows(const ClearArgs &k, O *table, int64_t ld, uint32_t num_rows, int N, uint32_t b, F named)
{
    constexpr int E = 32 / sizeof(O);
    struct __attribute__((packed, aligned(sizeof(O)))) Piece { O v[E]; };
    uint32_t row[TZ_SWEEPS];
    int c[TZ_SWEEPS];
    bool absent[TZ_SWEEPS];
#pragma unroll
    for (int q = 0; q < TZ_SWEEPS; ++q) {
        const uint32_t part = b * TZ_SWEEPS + q, g = part / k.chunks;
        row[q] = g * (WG >> k.lg) + (threadIdx.x >> k.lg);
        c[q] = E * ((int)(part - g * k.chunks) * (1 << k.lg) + (threadIdx.x & ((1 << k.lg) - 1)));
        absent[q] = part < k.parts && row[q] < num_rows && c[q] < N;
        absent[q] = absent[q] && !named(absent[q] ? row[q] : 0u);
    }
#pragma unroll
    for (int q = 0; q < TZ_SWEEPS; ++q) {
        if (!absent[q]) continue;
        O *p = table + row_at(row[q], ld) + c[q];
        const int n = N - c[q];
        if (n >= E) {
            *reinterpret_cast<Piece *>(p) = Piece{};
        } else {
            for (int j = 0; j < n; ++j) p[j] = (O)0.f;
        }
    }
}

// A tile of sorted entries for tx lanes, each with a vector of columns.  A run of equal tokens that lies inside the tile is
// applied here; the part of a run that goes on in the next tile is left in part[tile][1], the part of one that began in an
// earlier tile in part[tile][0].  The workgroups behind the tiles' clear the rows that no token names, in the same launch: few sums
// do not fill the device.
template <typename G, typename O, bool WHOLE>
__global__ __launch_bounds__(WG) void token_grad_kernel(const GradArgs a, int lg_tx, int chunks, uint32_t sum_blocks, const ClearArgs k)
{
    constexpr int NB = 8;
    __shared__ uint32_t keys[TG_MOST + 2], poss[TG_MOST + 2];
    if (blockIdx.x >= sum_blocks) {
        for (uint32_t b = blockIdx.x - sum_blocks; (uint64_t)b * TZ_SWEEPS < k.parts; b += gridDim.x - sum_blocks)     // (once, but for the largest tables)
            clear_rows(k, (O *)a.table, a.ld_table, (uint32_t)a.num_rows, a.N, b, [&](uint32_t row) { return k.named[row] != 0; });
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
        for (int q = 0; q < NB; ++q) x[q] = fetch8<WHOLE>((const G *)a.g + row_at(tp[min(e0 + q, cnt - 1)], a.ld_g) + 8 * v, n, a.N);
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
            settle8<WHOLE>(x[q], n, a.N);
            widen8(x[q], y);
            if (a.drop.state) drop8(a.drop, dk, (uint64_t)row_at(tp[e0 + q], a.nv) + (uint64_t)v, y);   // (a.factor has the dropout's)
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
        constexpr int NB = 8;
        for (int u0 = tile + 1 + gi; u0 < lo; u0 += NB * groups) {
            Vec8<float> x[NB];
#pragma unroll
            for (int q = 0; q < NB; ++q) x[q] = fetch8<true>(a.part + (int64_t)min(u0 + q * groups, lo - 1) * 2 * (8 * a.nv) + 8 * v, 8, 8);
#pragma unroll
            for (int q = 0; q < NB; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += u0 + q * groups < lo ? __uint_as_float(x[q].w[j]) : 0.f;
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

// Few tokens (or none): no sort.  A workgroup takes a position and up to WG vectors of columns; it ends if the position's token has
// an earlier one, else it lists the token's positions, which groups of 1 << lg_tx lanes add up side by side; the groups' sums are
// added in their order.  The workgroups behind clear the rows that no token names, after a look at all tokens.
constexpr int TF_MOST = 1024, TF_ROUNDS = TF_MOST / WG;

template <typename G, typename O, bool WHOLE>
__global__ __launch_bounds__(WG) void token_few_kernel(const GradArgs a, const void *tokens, int wide, int lg_tx, int chunks, uint32_t sum_blocks, const ClearArgs k)
{
    constexpr int NB = 8;
    __shared__ uint32_t list[TF_MOST], marks[TZ_SWEEPS * WG / 32];
    __shared__ uint64_t equal[TF_MOST / WAVE];
    __shared__ float lds[WG * 8];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, total = (int)a.n;
    const uint32_t none = (uint32_t)a.num_rows;
    uint32_t key[TF_ROUNDS];
#pragma unroll
    for (int q = 0; q < TF_ROUNDS; ++q) {
        const int i = q * WG + t;
        const int64_t x = i < total ? token_at(tokens, wide, i) : -1;
        key[q] = x >= 0 && x < a.num_rows ? (uint32_t)x : none;
    }
    if (blockIdx.x >= sum_blocks) {
        for (uint32_t b = blockIdx.x - sum_blocks; (uint64_t)b * TZ_SWEEPS < k.parts; b += gridDim.x - sum_blocks) {
            const uint32_t first = b * TZ_SWEEPS / k.chunks * (WG >> k.lg), rows = (TZ_SWEEPS - 1 + k.chunks) / k.chunks * (WG >> k.lg) + (WG >> k.lg);
            for (int i = t; i < TZ_SWEEPS * WG / 32; i += WG) marks[i] = 0;
            __syncthreads();
#pragma unroll
            for (int q = 0; q < TF_ROUNDS; ++q) {
                const uint32_t r = key[q] - first;
                if (key[q] != none && r < rows && r < TZ_SWEEPS * WG) atomicOr(&marks[r >> 5], 1u << (r & 31));
            }
            __syncthreads();
            clear_rows(k, (O *)a.table, a.ld_table, (uint32_t)a.num_rows, a.N, b, [&](uint32_t row) { return (marks[(row - first) >> 5] >> ((row - first) & 31)) & 1u; });
            __syncthreads();
        }
        return;
    }
    const int p = (int)(blockIdx.x / (unsigned)chunks);
    const int64_t mine_ = token_at(tokens, wide, p);
    if (mine_ < 0 || mine_ >= a.num_rows) return;
    const uint32_t mine = (uint32_t)mine_;
    uint64_t bal[TF_ROUNDS];
#pragma unroll
    for (int q = 0; q < TF_ROUNDS; ++q) {
        bal[q] = __ballot(key[q] == mine);
        if (lane == 0) equal[q * NWAVE + w] = bal[q];
    }
    __syncthreads();
    int cnt = 0;
    bool earlier = false;
    int before[TF_ROUNDS];                                   // positions of the token in earlier words than this wave's
    for (int x = 0; x < TF_MOST / WAVE; ++x) {
        const uint64_t m = equal[x];
#pragma unroll
        for (int q = 0; q < TF_ROUNDS; ++q)
            if (x == q * NWAVE + w) before[q] = cnt;
        cnt += __popcll(m);
        earlier |= x < p / WAVE ? m != 0 : x == p / WAVE && (m & ((1ull << (p & 63)) - 1ull)) != 0;
    }
    if (earlier) return;
#pragma unroll
    for (int q = 0; q < TF_ROUNDS; ++q)
        if (key[q] == mine) list[before[q] + __popcll(bal[q] & lanemask_lt())] = (uint32_t)(q * WG + t);
    __syncthreads();
    const int tx = 1 << lg_tx, groups = WG >> lg_tx, gi = t >> lg_tx, v = (int)(blockIdx.x % (unsigned)chunks) * tx + (t & (tx - 1));
    const int vc = min(v, a.nv - 1), n = a.N - 8 * vc;
    const DropKey dk = drop_key(a.drop);
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int e0 = gi; e0 < cnt; e0 += NB * groups) {
        Vec8<G> x[NB];
#pragma unroll
        for (int q = 0; q < NB; ++q) x[q] = fetch8<WHOLE>((const G *)a.g + row_at(list[min(e0 + q * groups, cnt - 1)], a.ld_g) + 8 * vc, n, a.N);
#pragma unroll
        for (int q = 0; q < NB; ++q) {
            const int e = e0 + q * groups;
            if (e >= cnt) break;
            float y[8];
            settle8<WHOLE>(x[q], n, a.N);
            widen8(x[q], y);
            if (a.drop.state) drop8(a.drop, dk, (uint64_t)row_at(list[e], a.nv) + (uint64_t)vc, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += y[j];
        }
    }
    if (groups > 1 && cnt > 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[j * WG + t] = sum[j];
        __syncthreads();
        const int with = min(groups, cnt);
        if (gi == 0)
            for (int q = 1; q < with; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += lds[j * WG + q * tx + t];
    }
    if (gi == 0 && v < a.nv) apply_row<O, WHOLE>(a, mine, v, sum);
}

}  // namespace tt
