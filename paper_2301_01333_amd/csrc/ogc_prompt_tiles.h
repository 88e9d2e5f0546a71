// How the tiles of prompt attention are sorted by how far they reach, as plain arithmetic: used by the kernels (ogc_prompt.hip), and by a test on
// the host that compares it with a count and looks for overflows.
#ifndef OGC_PROMPT_TILES_H
#define OGC_PROMPT_TILES_H

#include <stdint.h>

#ifdef __HIP__
#define PROMPT_FN static __host__ __device__ __forceinline__
#else
#define PROMPT_FN static inline
#endif

constexpr int PROMPT_LEVELS = 64;

// Keys of a level.  The announced longest sequence may be longer than all keys together.
PROMPT_FN int prompt_level_keys(int max_k, int k_rows) { return (max_k < k_rows ? max_k : k_rows) / PROMPT_LEVELS + 1; }

// Tiles of `tile_rows` rows (n queries times `group`) that reach key level * level_keys or further (level 0: all of them).  Causal: query i reaches
// key i + off, otherwise all reach the last of m.
PROMPT_FN int prompt_tiles_from(int n, int m, int off, int group, int causal, int level, int level_keys, int tile_rows) {
    const int rows = n * group, tiles = (rows + tile_rows - 1) / tile_rows;
    if (level <= 0) return tiles;
    if (level >= PROMPT_LEVELS) return 0;
    const int x = level * level_keys;
    if (!causal) return m > x ? tiles : 0;
    if (x <= off) return tiles;
    const uint32_t i = (uint32_t)x - (uint32_t)off;  // the first query that does (with more queries than keys it may be beyond 2^31)
    return i >= (uint32_t)n ? 0 : tiles - (int)i * group / tile_rows;
}

#endif
