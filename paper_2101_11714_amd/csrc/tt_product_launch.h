// Which kernel computes a product, and its launches.  The kernels of each type are compiled in a file of their own (tt_product_*.hip).
#pragma once

#include "tt_product_few.h"
#include "tt_product_stream.h"
#include "tt_rows_args.h"

namespace tt {

// which operands' rows are dense in k: x W^T, dz W, dz^T x
enum Layout { DENSE_DENSE, DENSE_STRIDED, STRIDED_STRIDED };

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
inline int64_t parts_of(int64_t tiles, int64_t steps)
{
    int64_t parts = tiles < 256 ? MOST_TILES / (tiles > 0 ? tiles : 1) : 1;
    if (parts > steps / 4) parts = steps / 4;
    return parts < 1 ? 1 : parts;
}

inline Plan plan_of(int64_t M, int64_t N, int64_t K, int32_t type, bool dense, bool whole)
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
inline size_t product_bytes(int64_t M, int64_t N, int64_t K, int32_t type)
{
    if (M <= 0 || N <= 0) return 0;
    const int64_t most = ceil_div(K, 128 / element_bytes(type)) / 4, wide = ceil_div(N, 256);
    if (wide >= 256 || most < 2) return 0;
    const int64_t rows = M * (most < MOST_TILES ? most : MOST_TILES), tiled = MOST_TILES * 256 / wide;
    return (size_t)(rows < tiled ? rows : tiled) * (size_t)(8 * ceil_div(N, 8)) * sizeof(float);
}

inline bool whole_chunks(const void *p, int64_t ld, int64_t columns, int32_t type)
{
    return type != TT_F32 && columns % 8 == 0 && ld % 8 == 0 && (uintptr_t)p % 16 == 0 && ld <= PS_MOST_STRIDE;
}

// C = A B^T, of M x N with sums over K, by the kernels of type T; out_type: T or 32 bits.
template <typename T>
int product_of(Layout layout, int32_t out_type, const void *a, int64_t lda, const void *b, int64_t ldb, int64_t M, int64_t N, int64_t K, const EpilogueArgs &e,
               void *workspace, hipStream_t st);
extern template int product_of<float>(Layout, int32_t, const void *, int64_t, const void *, int64_t, int64_t, int64_t, int64_t, const EpilogueArgs &, void *, hipStream_t);
extern template int product_of<bf16_t>(Layout, int32_t, const void *, int64_t, const void *, int64_t, int64_t, int64_t, int64_t, const EpilogueArgs &, void *, hipStream_t);
extern template int product_of<f16_t>(Layout, int32_t, const void *, int64_t, const void *, int64_t, int64_t, int64_t, int64_t, const EpilogueArgs &, void *, hipStream_t);

template <typename... A>
int product(int32_t type, A... args)
{
    return type == TT_F32 ? product_of<float>(args...) : type == TT_BF16 ? product_of<bf16_t>(args...) : product_of<f16_t>(args...);
}

}  // namespace tt
