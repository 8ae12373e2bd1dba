// How the keys of a cache's sequences are shared out over waves (cache_attention.hip, cache_lanes.hip).
//
// A sequence's keys make tiles of 32.  All sequences' tiles in a row are cut into equal parts, one a wave, and once so for
// every unit (a key head and up to 32 query heads that read it): waves of neighbouring numbers take the same keys for
// different heads, which lie beside one another in memory.  A cut inside a sequence of few tiles moves to its start, so that
// only long ones have several waves' sums to join.
#pragma once

#include <stdint.h>

#ifdef __HIP__
#define SUREL_BOTH __host__ __device__ __forceinline__
#else
#define SUREL_BOTH inline
#endif

namespace surel {

constexpr int kCacheTile = 32;      // keys
constexpr int kLeastTiles = 4;      // of a wave's part, where there are as many
constexpr int kWholeTiles = 16;     // sequences of up to these many are not cut, and caches of no longer ones need no join: 8 of up to
                                    // 300 keys 20.8 us by parts of 4, 16.1 whole; 500 and 4,000 of up to 700 as long either way
constexpr int kLookup = 4096;       // entries that a wave looks through, 64 lanes twice

// Parts of `tiles` tiles for up to `waves` waves, and where the n-th begins (before it moves).
SUREL_BOTH int64_t parts_of(int64_t tiles, int64_t waves) {
    const int64_t most = (tiles + kLeastTiles - 1) / kLeastTiles;
    return most < waves ? most : waves;
}
SUREL_BOTH int64_t part_begin(int64_t tiles, int64_t parts, int64_t n) {
    // n tiles / parts without passing 64 bits: tiles = a parts + b
    const int64_t a = tiles / parts, b = tiles % parts;
    return n * a + n * b / parts;
}
// The part that a tile is of, before cuts move: the last that begins at it or before.
SUREL_BOTH int64_t part_with(int64_t tiles, int64_t parts, int64_t tile) { return ((tile + 1) * parts - 1) / tiles; }
// A cut t tiles behind the start of a sequence of n: how far back it moves.
SUREL_BOTH int64_t moves_back(int64_t t, int64_t n) { return n <= kWholeTiles ? t : 0; }
SUREL_BOTH bool may_be_cut(int64_t most_tiles) { return most_tiles > kWholeTiles; }

// Sequences of one entry of the list that is looked through first: 1, or 64 and more.
SUREL_BOTH int64_t seqs_of_an_entry(int64_t n_seqs) {
    if (n_seqs <= kLookup) return 1;
    const int64_t each = (n_seqs + kLookup - 1) / kLookup;
    return (each + 63) / 64 * 64;
}

}  // namespace surel
