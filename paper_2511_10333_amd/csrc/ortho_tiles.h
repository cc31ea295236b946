// Which tiles of a symmetric output are made, and in which order.  (Compiles for the host alone, for the test of it.)
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define ORTHO_BOTH __host__ __device__
#else
#define ORTHO_BOTH
#endif

namespace edgc {

// Tiles of an output of `tiles` rows of tiles, on and below the diagonal: i + 1 in row i
ORTHO_BOTH inline uint32_t ortho_tiles(uint32_t tiles) { return tiles * (tiles + 1) / 2; }

// Tile `id` of them: in bands of eight rows, column by column, each XCD's (those of equal id modulo 8) neighbours of each other
ORTHO_BOTH inline void ortho_tile_of(uint32_t id, uint32_t tiles, uint32_t& tm, uint32_t& tn)
{
    constexpr uint32_t B = 8;
    const uint32_t total = ortho_tiles(tiles), per = total / 8, left = total % 8, xcd = id % 8, at = id / 8;
    id = xcd * per + (xcd < left ? xcd : left) + at;
    uint32_t band = 0;
    while ((band + 1) * B < tiles && ortho_tiles((band + 1) * B) <= id) ++band;
    const uint32_t rows = tiles - band * B < B ? tiles - band * B : B;
    uint32_t in = id - ortho_tiles(band * B);
    if (in < rows * B * band) {             // left of the band's diagonal
        tm = band * B + in % rows;
        tn = in / rows;
        return;
    }
    in -= rows * B * band;
    uint32_t c = 0;                         // a column at a time, of ever fewer rows
    while (in >= rows - c) in -= rows - c++;
    tm = band * B + c + in;
    tn = band * B + c;
}

}  // namespace edgc
