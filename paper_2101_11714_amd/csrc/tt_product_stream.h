// Products of 16-bit operands that are whole 16-byte chunks: operands straight from memory into LDS, two steps' worth.
#pragma once

#include "tt_product.h"

namespace tt {

constexpr uint32_t PS_RECORDS = 0x7ffffff0u, PS_NOWHERE = 0x80000000u;       // a buffer's bytes; an offset behind them: zeros are loaded
constexpr int64_t PS_MOST_STRIDE = 1 << 22;                  // of rows, so that offsets in a tile stay below PS_RECORDS

constexpr int PS_K = 64, PS_SLOTS = 5;                       // values of k in a step; tiles of operands that LDS holds

template <bool WIDE>
struct StreamShape {
    static constexpr int TILE = WIDE ? 256 : 128, THREADS = WIDE ? 512 : 256, WAVES = THREADS / WAVE;
    static constexpr int BM = TILE / 2 / BLOCK;              // a wave's blocks along m; along n they are four
    static constexpr int SLOT = TILE * 128, LDS = PS_SLOTS * SLOT;
};

// What a wave loads of an operand's tile: PIECES times 64 chunks, one per lane, which go to 1 KB of LDS in the lanes' order.
template <typename T, bool KDENSE, bool WIDE>
struct Stream {
    typedef StreamShape<WIDE> S;
    typedef OperandTile<T, KDENSE, S::TILE> Tile;
    static constexpr int PIECES = Tile::CHUNKS / S::THREADS, CH = Tile::CH;
    const char *base;            // of the step's values
    int64_t step;                // bytes to the next one's
    uint32_t at[PIECES];         // the lane's offsets
    int k[PIECES];               // where in the step their values of k begin
    int wave;

    __device__ __forceinline__ Stream(const void *data, int64_t ld, int64_t row0, int64_t rows, int64_t k0, int w, int lane) : wave(w)
    {
        base = (const char *)data + (KDENSE ? row0 * ld + k0 : k0 * ld + row0) * (int64_t)sizeof(T);
        step = (KDENSE ? PS_K : PS_K * ld) * (int64_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int s = (i * S::WAVES + wave) * WAVE + lane, line = s / Tile::LINE, chunk = (s % Tile::LINE) ^ Tile::swizzle(line);
            if (KDENSE) {
                const int64_t left = rows - row0 - 1;
                at[i] = (uint32_t)((line < left ? line : (int)left) * ld + chunk * CH) * (uint32_t)sizeof(T);
                k[i] = chunk * CH;
            } else {
                at[i] = row0 + chunk * CH < rows ? (uint32_t)(line * ld + chunk * CH) * (uint32_t)sizeof(T) : PS_NOWHERE;
                k[i] = line;
            }
        }
    }
    // The next step's tile; `left`: its values of k that exist.  Behind the last ones zeros are loaded, so that the number of loads does not depend on
    // it.  In assembly, since the compiler takes every read of LDS for one of what is still on its way and waits for it; nothing but LDS and M0 is
    // written, which nothing else here uses, and the waits are landed()'s.  A load into LDS reads M0 a wait state after it is written at the earliest, which
    // the compiler sees to around its own instructions and not in here: the s_nop.
    __device__ __forceinline__ void load(char *lds, int left)
    {
        typedef uint32_t Words __attribute__((ext_vector_type(4)));
        const uint64_t from = (uint64_t)base;
        const Words r = {(uint32_t)from, (uint32_t)(from >> 32), PS_RECORDS, 0x00020000u};
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + wave * 1024;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const uint32_t o = k[i] < left ? at[i] : PS_NOWHERE;
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to + i * S::WAVES * 1024), "v"(o), "s"(r) : "memory");
        }
        base += step;
    }
    template <int N>
    static __device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
};

// Steps of 64 values of k.  LDS holds five tiles of operands, both of the step that is read and of the next one, and a fifth that makes room for
// one operand's step after that, so that one tile is asked for in every half of a step (both in its first half: products of 8,192^3 zeros at 1,390 instead of 1,600
// TFLOP/s, since what misses an L2 holds up what follows it).
// WIDE: tiles of 256 x 256 by eight waves of 128 x 64 in two groups of four, one of each group on every SIMD.  A half is first read from LDS into
// registers and then multiplied; the second group is one phase behind, so that a SIMD's matrix core works for one wave while the other one
// reads.  A barrier ends every phase.
// Else: tiles of 128 x 128 by four waves of 64 x 64, two workgroups on a compute unit, which find their turns by themselves.
template <typename T, typename O, bool AK, bool BK, bool WIDE>
__device__ __forceinline__ void stream_tile(const ProductArgs &p, const EpilogueArgs &e, int id, char *lds)
{
    typedef StreamShape<WIDE> S;
    typedef Stream<T, AK, WIDE> SA;
    typedef Stream<T, BK, WIDE> SB;
    constexpr int BM = S::BM, BN = 4;
    int tm, tn, part;
    tile_of(id, p, tm, tn, part);
    const int64_t m0 = (int64_t)tm * S::TILE, n0 = (int64_t)tn * S::TILE, k0 = part * p.k_part;
    const int64_t k_end = k0 + p.k_part < p.K ? k0 + p.k_part : p.K;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave >> (WIDE ? 2 : 1);
    const int wm = group * (S::TILE / 2), wn = (wave & (WIDE ? 3 : 1)) * 64;
    SA a(p.a, p.lda, m0, p.M, k0, wave, lane);
    SB b(p.b, p.ldb, n0, p.N, k0, wave, lane);

    mfma_acc_t acc[BM][BN];
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j) acc[i][j] = mfma_acc_t{0.f, 0.f, 0.f, 0.f};
    uint4 fa[BM], fb[BN];
    auto read = [&](const char *ta, const char *tb, int h) {
#pragma unroll
        for (int j = 0; j < BN; ++j) fb[j] = SB::Tile::fragment(tb, wn, j, h, lane);
#pragma unroll
        for (int i = 0; i < BM; ++i) fa[i] = SA::Tile::fragment(ta, wm, i, h, lane);
    };
    auto left = [&](int64_t k) { return (int)(k_end - k < PS_K ? k_end - k : PS_K); };
    auto slot = [&](int first, int n) { return lds + (first + n >= PS_SLOTS ? first + n - PS_SLOTS : first + n) * S::SLOT; };
    auto multiply = [&] {
        __builtin_amdgcn_s_setprio(1);
        block_products<T>(fb, fa, acc);
        __builtin_amdgcn_s_setprio(0);
    };
    auto phase = [] {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

    auto have_read = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };

    // step t's tiles are in slots 2 t and 2 t + 1, modulo their number
    a.load(slot(0, 0), left(k0));
    b.load(slot(0, 1), left(k0));
    a.load(slot(0, 2), left(k0 + PS_K));
    SA::template landed<SA::PIECES>();
    phase();
    int first = 0;
    if (WIDE && group) phase();
    for (int64_t k = k0; k < k_end; k += PS_K) {
        read(slot(first, 0), slot(first, 1), 0);
        b.load(slot(first, 3), left(k + PS_K));              // where the first operand's step before this one was
        if (WIDE) {
            have_read();
            phase();
        }
        multiply();
        if (WIDE) phase();
        read(slot(first, 0), slot(first, 1), 1);
        a.load(slot(first, 4), left(k + 2 * PS_K));
        if (WIDE) {
            have_read();                                     // (what is read now may be written over from the next phase but one on)
            if (group) SA::template landed<SA::PIECES>();
            phase();
        }
        multiply();
        if (!WIDE || !group) SA::template landed<SA::PIECES>();
        phase();
        first = first + 2 >= PS_SLOTS ? first + 2 - PS_SLOTS : first + 2;
    }
    if (WIDE && !group) phase();
    SA::template landed<0>();
    phase();
    leave_tile<T, O, BM, 4, AK && BK>(p, e, part, m0 + wm, n0 + wn, lane, lds + wave * 4 * LEAVE_BLOCK, acc);
}

template <typename T, typename O, bool WIDE>
__global__ __launch_bounds__(StreamShape<WIDE>::THREADS, 2) void product_stream_kernel(ProductArgs p, EpilogueArgs e)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    if (workgroup() < (int64_t)p.tiles_m * p.tiles_n * p.parts) stream_tile<T, O, true, true, WIDE>(p, e, (int)workgroup(), lds);
}

template <typename T, typename W, bool WIDE>
__global__ __launch_bounds__(StreamShape<WIDE>::THREADS, 2) void pair_stream_kernel(PairArgs g)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    int64_t id = workgroup();
    const int which = which_of(g, id);
    if (which == 0) stream_tile<T, T, true, false, WIDE>(g.p[0], g.e[0], (int)id, lds);
    else if (which == 1) stream_tile<T, W, false, false, WIDE>(g.p[1], g.e[1], (int)id, lds);
}

}  // namespace tt
