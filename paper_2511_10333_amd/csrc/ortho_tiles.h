// Which tiles of a symmetric output are made, and in which order.  (Compiles for the host alone, for the test of it.)
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define ORTHO_BOTH __host__ __device__
#else
#define ORTHO_BOTH
#endif

namespace edgc {

// Tiles of an output of `tiles_m` rows of tiles, R times as high as wide, on and below the diagonal: R (i + 1) in row i, but of the last row no more than the
// `tiles_n` columns of tiles that there are.
template <uint32_t R>
ORTHO_BOTH inline uint32_t ortho_rows(uint32_t rows) { return R * (rows * (rows + 1) / 2); }
template <uint32_t R>
ORTHO_BOTH inline uint32_t ortho_tiles(uint32_t tiles_m, uint32_t tiles_n) { return ortho_rows<R>(tiles_m) - (R * tiles_m - tiles_n); }

// Tile `id` of them: in bands of eight rows, column by column, each XCD's (those of equal id modulo 8) neighbours of each other.  The tiles that are not made would be
// the last.
template <uint32_t R>
ORTHO_BOTH inline void ortho_tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn)
{
    constexpr uint32_t B = 8;
    const uint32_t total = ortho_tiles<R>(tiles_m, tiles_n), per = total / 8, left = total % 8, xcd = id % 8, at = id / 8;
    id = xcd * per + (xcd < left ? xcd : left) + at;
    uint32_t band = 0;
    while ((band + 1) * B < tiles_m && ortho_rows<R>((band + 1) * B) <= id) ++band;
    const uint32_t rows = tiles_m - band * B < B ? tiles_m - band * B : B;
    uint32_t in = id - ortho_rows<R>(band * B);
    if (in < rows * B * R * band) {         // left of the band's diagonal
        tm = band * B + in % rows;
        tn = in / rows;
        return;
    }
    in -= rows * B * R * band;
    uint32_t c = 0;                         // R columns at a time, of ever fewer rows
    while (in >= R * (rows - c)) in -= R * (rows - c++);
    tm = band * B + c + in % (rows - c);
    tn = R * (band * B + c) + in / (rows - c);
}

}  // namespace edgc
