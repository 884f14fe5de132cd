// Attention over the cache: which rows a workgroup has, which keys they see, and where the table names those keys' blocks.  All of it is
// arithmetic on lengths, starts and table entries that may hold anything, so it runs on the host too, where its tests are.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lffn {

#define LFFN_TILE __host__ __device__ __forceinline__

struct AttendArgs {
    const void *q;
    void *y;
    const uint8_t *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    const int *table, *starts, *lengths;
    bool join_each;       // the join takes several rows to a workgroup
    float *part;          // [chunk][token * heads][dim]: sums of a chunk of keys, of tiles whose keys take several; null where none does
    float *part_ml;       // [chunk][token * heads][2]: its maximum (in powers of two) and its sum of probabilities
    long long q_token, q_head, y_token, y_head, table_stride;
    int n_tokens, requests, heads, kv_heads, group;
    unsigned group_inverse;   // floor(2^32 / group), for group > 1
    int width, n_blocks, block_log;
    int causal, window;
    int max_keys;         // of a request: what the caller says, and what a row of the table holds
    int max_queries;      // tokens of a request that the grid (and the few-row kernel's LDS) has room for
    int chunk, chunks;    // keys of a chunk, chunks of the grid
    int row_tiles;        // tiles of rows of a request and key head, of the grid
    int tile_rows;        // rows of a tile
    float scale;          // log2(e) / sqrt(dim)
};

// The rows that a workgroup has and the keys they see.
struct RowTile {
    int r, h;                 // request, key head
    int first, fresh, past;   // the request's first token and its tokens; the position of the first
    int row0, rows;           // first row of the tile; rows of the request
    int lo, hi;               // keys that some row sees: lo .. hi - 1
};

// the query that a row belongs to: row / group (the product falls short of it by one at most)
LFFN_TILE int query_of(const AttendArgs &a, int row)
{
    if (a.group == 1) return row;
    const unsigned q = (unsigned)(((uint64_t)(unsigned)row * a.group_inverse) >> 32);
    return (int)(q + ((unsigned)row - q * (unsigned)a.group >= (unsigned)a.group));
}

// A length may be any int, and with it the position of the first token, so no key is worked out from it that is not held against `hi` first:
// hi is at most max_keys (2^30 at most), and lo at most hi, so that the keys of chunks and steps, and what they look up ahead, stay ints.
LFFN_TILE RowTile row_tile(const AttendArgs &a, int combo, int tile, int tile_rows)
{
    RowTile t;
    t.r = combo / a.kv_heads;
    t.h = combo - t.r * a.kv_heads;
    t.first = min(max(a.starts[t.r], 0), a.n_tokens);
    t.fresh = min(max(a.starts[t.r + 1], t.first), a.n_tokens) - t.first;
    const int whole = max(a.lengths[t.r], 0), length = min(whole, a.max_keys);
    t.past = whole - t.fresh;
    t.rows = min(t.fresh, a.max_queries) * a.group;
    t.row0 = tile * tile_rows;
    const int last = max(min(t.row0 + tile_rows, t.rows) - 1, 0);
    const int p0 = t.past + query_of(a, min(t.row0, last)), p1 = t.past + query_of(a, last);   // positions of the first and the last row
    t.hi = a.causal && p1 < length ? max(p1, -1) + 1 : length;
    t.lo = a.window ? max(p0 - a.window + 1, 0) : 0;
    t.lo = min(t.lo, t.hi) & ~63;   // chunks and steps begin at multiples of 64 keys
    return t;
}

// the tile's keys that are in a chunk: c0 .. c1 - 1
LFFN_TILE void chunk_keys(const AttendArgs &a, const RowTile &t, int chunk, int &c0, int &c1)
{
    c0 = t.lo + chunk * a.chunk;   // (the chunks before the last are fewer keys than max_keys, so up to 2^31 - 1)
    c1 = t.hi - c0 > a.chunk ? c0 + a.chunk : t.hi;
}

// the keys lo .. hi - 1 that row `row` of the tile's request sees
LFFN_TILE void row_keys(const AttendArgs &a, const RowTile &t, int row, int &lo, int &hi)
{
    const int i = query_of(a, row);
    hi = a.causal ? min(t.hi, t.past + i + 1) : t.hi;
    lo = a.window ? max(t.past + i - a.window + 1, 0) : 0;
}

// The block that holds a request's keys from `key` on, in two steps so that the first's load can be long on its way before the second:
// what the table says (of keys that are not negative), and that or -1 where the table, or the keys before `end`, or the cache have no such block.
LFFN_TILE int table_column(const AttendArgs &a, int key) { return min(key >> a.block_log, a.width - 1); }
LFFN_TILE int table_entry(const AttendArgs &a, const int *row, int key) { return row[table_column(a, key)]; }
LFFN_TILE int block_of(const AttendArgs &a, int entry, int key, int end)
{
    return key < end && (key >> a.block_log) < a.width && entry >= 0 && entry < a.n_blocks ? entry : -1;
}

#undef LFFN_TILE

}  // namespace lffn
