// The arithmetic of attention's tiles on the host (attend_tile.hpp), with lengths, starts and windows of any kind: every key that a kernel works
// out stays an int, every column of the table that it looks up is one, and what it finds is what the definition says.
#include "attend_tile.hpp"

#include <stdio.h>
#include <stdlib.h>

#include <algorithm>

using namespace lffn;

static long long cases = 0;

static void fail(const char *what, const AttendArgs &a, long long x)
{
    printf("%s: %lld (length %d, starts %d %d, window %d, causal %d, max_keys %d, chunk %d of %d, width %d)\n", what, x, a.lengths[0],
           a.starts[0], a.starts[1], a.window, a.causal, a.max_keys, a.chunk, a.chunks, a.width);
    exit(1);
}

static void look_up(const AttendArgs &a, long long key)
{
    if (key < 0 || key > INT32_MAX) fail("a key that is no key of a request", a, key);
    const int column = table_column(a, (int)key);
    if (column < 0 || column >= a.width) fail("a column outside the table", a, column);
}

// the keys that the kernels work out of a tile, in the order they do
static void few(const AttendArgs &a, const RowTile &t, int chunk)
{
    int c0, c1;
    chunk_keys(a, t, chunk, c0, c1);
    if (c0 >= c1 && chunk > 0) return;
    for (int wave = 0; wave < 4; ++wave) {
        int key0 = c0 + 64 * wave;
        for (int g = 0; g < 4 && a.width; ++g) look_up(a, key0 + 16 * g);
        if (key0 < c1) look_up(a, (long long)key0 + 256 + 48);
        // the first and the last steps (between them nothing but multiples of 256 are added)
        for (int i = 0; key0 < c1; ++i) {
            look_up(a, (long long)key0 + 512 + 48);
            if (i == 2 && c1 - key0 > 2048) key0 += (c1 - key0 - 1024) / 256 * 256;
            if (c1 - key0 <= 256) break;
            key0 += 256;
        }
    }
}
static void many(const AttendArgs &a, const RowTile &t, int chunk)
{
    int c0, c1;
    chunk_keys(a, t, chunk, c0, c1);
    if (c0 >= c1 && chunk > 0) return;
    const int steps = c0 < c1 ? (c1 - c0 + 63) / 64 : 0;
    for (int i : {0, 1, 2, 3, 4 * steps, 4 * steps + 3})
        if (a.width) look_up(a, (long long)c0 + 16 * i);
}

static void one(AttendArgs a, int start, int end, int length, int tile_rows)
{
    const int starts[2] = {start, end}, lengths[1] = {length};
    a.starts = starts;
    a.lengths = lengths;
    const int rows = a.group * a.max_queries;
    for (int tile : {0, 1, (rows - 1) / tile_rows}) {
        if (tile * (long long)tile_rows >= rows) continue;
        const RowTile t = row_tile(a, 0, tile, tile_rows);
        ++cases;
        if (t.row0 + (long long)tile_rows + 128 > INT32_MAX) fail("a row past the tile", a, t.row0);   // (waves and the join count on past the last)
        if (t.row0 >= t.rows) continue;
        if (t.lo < 0 || t.lo > t.hi || t.hi > a.max_keys || t.lo % 64) fail("the tile's keys", a, t.lo);
        // the definition, in 64 bits
        const long long fresh = t.fresh, whole = std::max(length, 0), past = whole - fresh;
        const long long held = std::min({whole, (long long)a.max_keys, (long long)a.width << a.block_log});
        const long long last = std::min<long long>(t.row0 + tile_rows, t.rows) - 1;
        long long some_lo = INT64_MAX, some_hi = 0;
        for (long long row : {(long long)t.row0, (t.row0 + last) / 2, last}) {
            const long long i = row / a.group, hi = a.causal ? std::min(held, past + i + 1) : held;
            const long long lo = a.window ? std::max(past + i - a.window + 1, 0LL) : 0;
            int klo, khi;
            row_keys(a, t, (int)row, klo, khi);
            if (lo < hi ? klo != lo || khi != hi : klo < khi) fail("a row's keys", a, row);
            if (lo < hi) some_lo = std::min(some_lo, lo), some_hi = std::max(some_hi, hi);
        }
        if (some_lo < some_hi && (t.lo > some_lo || t.hi < some_hi)) fail("keys that a row sees are not the tile's", a, t.lo);
        for (int chunk : {0, 1, 2, a.chunks / 2, a.chunks - 1})
            if (chunk < a.chunks) {
                few(a, t, chunk);
                many(a, t, chunk);
            }
    }
}

int main()
{
    const int top = INT32_MAX, big = 1 << 30;
    AttendArgs a{};
    a.kv_heads = 1;
    a.requests = 1;
    for (int group : {1, 2, 3, 8})
        for (int n : {1, 5, 300, big / group, (int)std::min<long long>(big, ((1LL << 31) - 256) / group)})
            for (int window : {0, 1, 2, 63, 64, 190, 2000, 100000, big})
                for (int causal : {0, 1})
                    for (int max_keys : {0, 1, 64, 1000, 131072, big})
                        for (int chunk : {256, 512, 4096, 8192, big})
                            for (int block_log : {4, 7})
                                for (int width : {0, 1, 17, (max_keys >> block_log) + 1, 1 << 28}) {
                                    a.group = group;
                                    a.heads = group;
                                    a.group_inverse = group > 1 ? (unsigned)(((uint64_t)1 << 32) / (unsigned)group) : 0;
                                    a.n_tokens = a.max_queries = n;
                                    a.window = window;
                                    a.causal = causal;
                                    a.max_keys = (int)std::min<long long>(max_keys, (long long)width << block_log);   // as attend() does
                                    a.block_log = block_log;
                                    a.width = width;
                                    a.n_blocks = 10;
                                    a.chunk = chunk;
                                    long long span = std::max(max_keys, 1);
                                    if (window) span = std::min<long long>(span, (long long)window + n + 64 + 128);
                                    span = (span + 63) / 64 * 64;
                                    a.chunks = (int)((span + chunk - 1) / chunk);
                                    for (int tile_rows : {16, 128})
                                        for (int length : {-top - 1, -1, 0, 1, n - 1, n, 700, big, big + 1, top - 2000, top - 190, top - 63, top - 1, top}) {
                                            one(a, 0, n, length, tile_rows);
                                            if (chunk != 512) continue;
                                            for (int start : {-top - 1, n - 1, n, top}) one(a, start, n, length, tile_rows);
                                            for (int end : {-top - 1, 0, top}) one(a, 0, end, length, tile_rows);
                                        }
                                }
    printf("%lld tiles ran clean\n", cases);
    return 0;
}
