// The way of a workgroup of linear8.hip over its tiles, and the stages that it asks for.
// A host test compiles it too: who includes it brings __device__.
//
// The stages go on over the tiles' borders, and past the last tile, where their buffers
// hold nothing.  A load's range is checked as (lane's offset) against (the buffer's bytes
// less what all lanes' offsets are moved by), and that difference must not be below 0: a
// stage that is not there begins at 0.
#pragma once

#include <cstdint>

namespace rocket {

struct Tile {
    int64_t t;   // rows t times a tile's and on
    int m;       // channels
};

struct Steps {
    int64_t t;
    int m, tiles;   // tiles along the channels
    __device__ Tile after(Tile x) const {
        x.t += t, x.m += m;
        if (x.m >= tiles) x.m -= tiles, x.t++;
        return x;
    }
};

// Bytes of `most` lines of `columns` from line `first` on, of those that there are.
__device__ inline int64_t bytes_of_lines(int64_t lines, int64_t first, int most, int64_t columns) {
    const int64_t left = lines - first;
    return left <= 0 ? 0 : (left < most ? left : most) * columns;
}

// The stages of the tiles in their order.  `stages` of a tile, the first of them stage0.
struct Asked {
    Tile tile;
    int stage;     // the next one's number in the tile
    bool there;    // whether the tile is

    // Whether the next stage is another tile's, which is then the current one.
    __device__ bool crosses(int stages, const Steps &steps) {
        if (stage < stages) return false;
        tile = steps.after(tile), stage = 0;
        return true;
    }
    // Where the next stage's columns begin in a line, bytes; goes on to the one after.
    __device__ uint32_t next(int stage0, int columns) {
        const uint32_t at = (uint32_t)((stage0 + stage) * columns);
        stage++;
        return there ? at : 0;
    }
};

}  // namespace rocket
