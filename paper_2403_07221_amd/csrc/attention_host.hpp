// Host side of the entry points beside the layer (plan_cache, rotate, rotate_append, attend): argument checks, launch shapes and
// launches.  Part 0 of lookupffn.hip includes this in its anonymous namespace; the kernels are in parts 15 .. 18.

bool block_ok(int block) { return block == 16 || block == 32 || block == 64 || block == 128; }
int log2_of(int block) { return __builtin_ctz((unsigned)block); }
constexpr int64_t kMaxStepTokens = int64_t(1) << 30;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 256;   // tokens * heads: a tile's rows past the last one are ints too
constexpr int kMaxHeads = 4096;

// ---------------------------------------------------------------- plan

int plan_cache(const int32_t *past, const int32_t *fresh, const int32_t *free_blocks, int32_t *table, int32_t *starts, int32_t *lengths,
               int32_t *slots, int32_t *positions, int32_t *counts, int n_requests, int64_t n_free, int table_width, int64_t table_stride,
               int64_t n_tokens, int block, hipStream_t s)
{
    if (n_requests < 0 || n_free < 0 || table_width < 0 || table_stride < table_width || n_tokens < 0 || n_tokens > kMaxStepTokens)
        return LFFN_E_SIZE;
    if (!block_ok(block) || n_requests > kMaxRequests) return LFFN_E_UNSUPPORTED;
    if (!starts || !counts || (n_requests && (!past || !fresh || !lengths || (table_width && !table))) || (n_free && !free_blocks) ||
        (n_tokens && (!slots || !positions)))
        return LFFN_E_NULL;
    for (const void *p : {(const void *)past, (const void *)fresh, (const void *)free_blocks, (const void *)table, (const void *)starts,
                          (const void *)lengths, (const void *)slots, (const void *)positions, (const void *)counts})
        if (!aligned(p, 4)) return LFFN_E_ALIGN;
    PlanArgs a{};
    a.past = past;
    a.fresh = fresh;
    a.free_blocks = free_blocks;
    a.table = table;
    a.starts = starts;
    a.lengths = lengths;
    a.slots = slots;
    a.positions = positions;
    a.counts = counts;
    a.n_free = n_free;
    a.table_stride = table_stride;
    a.requests = n_requests;
    a.width = table_width;
    a.n_tokens = (int)n_tokens;
    a.block_log = log2_of(block);
    // past a workgroup to a compute unit the scans that each makes for itself would only be repeated
    const int threads = n_requests <= 512 && n_tokens <= 512 ? 256 : 1024;
    const int64_t groups = std::min<int64_t>(std::max<int64_t>((n_tokens + threads - 1) / threads, 1), 256);
    return lffn_host::plan_cache_part(threads, a, dim3((unsigned)groups), (size_t)(2 * n_requests + 2) * 4, s);
}

// ---------------------------------------------------------------- rotate, rotate_append

struct RowsIn {
    const void *in;
    void *out;
    const float *weight;
    int heads;
    int64_t st[4];   // in: token, head; out: token, head (elements)
};

int check_rows(const RowsIn &r, int elem)
{
    if (!r.in) return LFFN_E_NULL;
    if (!aligned(r.in, elem) || !aligned(r.out, elem) || !aligned(r.weight, 4)) return LFFN_E_ALIGN;
    for (int64_t s : r.st)
        if (s < 0) return LFFN_E_SIZE;
    return LFFN_OK;
}
// rows whose every piece of sixteen bytes can be taken as one
bool vector_rows(const RowsIn &r, int elem)
{
    bool ok = aligned(r.in, 16) && aligned(r.out, 16);
    for (int64_t s : r.st) ok = ok && (s * elem) % 16 == 0;
    return ok;
}
Rows rows_of(const RowsIn &r)
{
    Rows o{};
    o.in = r.in;
    o.out = r.out;
    o.in_token = r.st[0];
    o.in_head = r.st[1];
    o.out_token = r.st[2];
    o.out_head = r.st[3];
    o.weight = r.weight;
    o.heads = r.heads;
    return o;
}

int check_rotation(const float *angles, const int32_t *positions, int64_t n_tokens, int heads, int kv_heads, int dim, int rot,
                   int64_t n_positions, float eps, int dtype)
{
    if (n_tokens < 0 || n_tokens > kMaxStepTokens || heads < 1 || kv_heads < 1 || dim < 1 || rot < 0 || rot > dim || rot % 2 ||
        n_positions < 0 || n_positions > INT32_MAX || !(eps >= 0.0f))
        return LFFN_E_SIZE;
    if (heads > kMaxHeads || kv_heads > kMaxHeads) return LFFN_E_UNSUPPORTED;
    if (!dtype_ok(dtype)) return LFFN_E_DTYPE;
    if (dim % 16 || dim > kMaxHeadDim) return LFFN_E_UNSUPPORTED;
    if (rot && n_tokens) {
        if (!angles || !positions) return LFFN_E_NULL;
        if (n_positions < 1) return LFFN_E_SIZE;
        if (!aligned(angles, 4) || !aligned(positions, 4)) return LFFN_E_ALIGN;
    }
    return LFFN_OK;
}

// heads of a token that a lane group takes together: several once that leaves four workgroups to a compute unit
int rows_together(int64_t rows, int per) { return rows / per >= (int64_t)kRowsTogether * 1024 ? kRowsTogether : 1; }

int rotate(RowsIn q, RowsIn k, const float *angles, const int32_t *positions, int64_t n_tokens, int dim, int rot, int64_t n_positions,
           float eps, int interleaved, int dtype, hipStream_t s)
{
    int rc = check_rotation(angles, positions, n_tokens, q.heads, k.heads, dim, rot, n_positions, eps, dtype);
    if (rc != LFFN_OK || n_tokens == 0) return rc;
    if (!q.out || !k.out) return LFFN_E_NULL;
    const int elem = dtype == LFFN_F32 ? 4 : 2;
    if ((rc = check_rows(q, elem)) != LFFN_OK || (rc = check_rows(k, elem)) != LFFN_OK) return rc;
    RotateArgs a{};
    a.q = rows_of(q);
    a.k = rows_of(k);
    a.angles = rot ? angles : nullptr;
    a.positions = positions;
    a.n_tokens = (int)n_tokens;
    a.dim = dim;
    a.rot = rot;
    a.n_positions = (int)n_positions;
    a.eps = eps;
    const bool vec = vector_rows(q, elem) && vector_rows(k, elem) && (interleaved || rot % 16 == 0);
    const int per = 256 / row_lanes(dim), together = rows_together(n_tokens * (q.heads + k.heads), per);
    const int64_t units = (q.heads + together - 1) / together + (k.heads + together - 1) / together;
    return lffn_host::rotate_part(dtype, vec, interleaved != 0, together, a, grid_of((n_tokens * units + per - 1) / per), s);
}

int rotate_append(RowsIn q, RowsIn k, RowsIn v, const float *angles, const int32_t *positions, const int32_t *slots, void *k_cache,
                  void *v_cache, float *k_scale, float *v_scale, int64_t n_tokens, int dim, int rot, int64_t n_positions, int64_t n_blocks,
                  int block, float eps, int interleaved, int dtype, hipStream_t s)
{
    int rc = check_rotation(angles, positions, n_tokens, q.heads, k.heads, dim, rot, n_positions, eps, dtype);
    if (rc != LFFN_OK) return rc;
    if (n_blocks < 0 || n_blocks > INT32_MAX) return LFFN_E_SIZE;
    if (dim > kMaxCacheDim || !block_ok(block)) return LFFN_E_UNSUPPORTED;
    if (n_tokens == 0) return LFFN_OK;
    if (!q.out || !slots || !k_cache || !v_cache || !k_scale || !v_scale) return LFFN_E_NULL;
    const int elem = dtype == LFFN_F32 ? 4 : 2;
    for (const RowsIn *r : {&q, &k, &v})
        if ((rc = check_rows(*r, elem)) != LFFN_OK) return rc;
    if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned(slots, 4))
        return LFFN_E_ALIGN;
    AppendArgs a{};
    a.rows.q = rows_of(q);
    a.rows.k = rows_of(k);
    a.rows.angles = rot ? angles : nullptr;
    a.rows.positions = positions;
    a.rows.n_tokens = (int)n_tokens;
    a.rows.dim = dim;
    a.rows.rot = rot;
    a.rows.n_positions = (int)n_positions;
    a.rows.eps = eps;
    a.v = v.in;
    a.v_token = v.st[0];
    a.v_head = v.st[1];
    a.slots = slots;
    a.k_cache = static_cast<uint8_t *>(k_cache);
    a.v_cache = static_cast<uint8_t *>(v_cache);
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.block_log = log2_of(block);
    a.n_slots = n_blocks << a.block_log;
    a.kv_heads = k.heads;
    const bool vec = vector_rows(q, elem) && vector_rows(k, elem) && vector_rows(v, elem) && (interleaved || rot % 16 == 0);
    // Few tokens are single ones of many requests, each a run of its own: a workgroup to a token; many are prompts, a run a block.  Tiles of a
    // token and of a block, 32 + 8 + 8 heads of 128 in bf16, blocks of 16 and of 128, us: 64 single tokens 7 / 43 and 16 / 430, 512 of them 29 / 51
    // and 88 / 889; one prompt of 512 14 / 7 and 29 / 14, 1632 tokens of eight 36 / 15 and 78 / 25, 14763 of twelve 293 / 91 and 676 / 93.  The rule
    // counts tokens, not runs: 1000 single tokens take the block's tile, 53 / 65 and 166 / 847.
    a.tile = n_tokens * k.heads * 2 <= 8192 ? 1 : block;
    a.append_groups = (n_tokens + a.tile - 1) / a.tile * 2 * k.heads;
    // half the lanes where a block's keys are a sixteenth each for them
    const int pieces = block * row_lanes(dim), threads = pieces <= 128 ? 128 : 256;
    const int per = threads / row_lanes(dim);
    a.rows_together = rows_together(n_tokens * q.heads, 256 / row_lanes(dim));
    const int64_t q_units = (q.heads + a.rows_together - 1) / a.rows_together;
    const size_t lds = (size_t)dim * (block / 4 + 1) * 4;
    return lffn_host::append_part(dtype, vec, interleaved != 0, threads, pieces <= 512, a,
                                  grid_of(a.append_groups + (n_tokens * q_units + per - 1) / per), lds, s);
}

// ---------------------------------------------------------------- attend

constexpr int kAttendCus = 256;   // the size queries plan without a device

struct AttendPlan {
    bool many = false;   // attend_many_kernel
    int tile_rows = 16, row_tiles = 1;
    int chunk = 0, chunks = 1;
    int64_t bytes = 0, ml_at = 0;
};

int64_t attend_group_rows(int heads, int kv_heads, int64_t max_queries) { return heads / kv_heads * max_queries; }

AttendPlan plan_attend(int64_t n_tokens, int n_requests, int heads, int kv_heads, int dim, int64_t max_queries, int64_t max_keys, int causal,
                       int window, int dtype)
{
    AttendPlan p;
    const int64_t rows = attend_group_rows(heads, kv_heads, max_queries);
    // Tiles of sixteen rows read the keys once more each, from L2.  24 requests of 1000 .. 4000 keys, 16 / 32 / 64 rows a key head, few-row
    // kernel and many-row kernel, us: dim 64 32 / - / 61 and 56 / - / 72; dim 128 37 / 54 / 91 and 60 / 64 / 78; dim 256 25 / 43 / 64 and
    // 46 / 47 / 51.
    p.many = rows > (dim == 64 ? 64 : 32);
    p.tile_rows = !p.many ? 16 : rows > 64 ? 128 : 64;
    p.row_tiles = (int)std::max<int64_t>((rows + p.tile_rows - 1) / p.tile_rows, 1);
    // keys that a tile of rows can see, from a multiple of 64 on; where rows see what follows them, to the end of the request, which may bring
    // more tokens than max_queries (the rows inside that bound see the others' keys)
    int64_t span = std::max<int64_t>(max_keys, 1);
    if (window) span = std::min<int64_t>(span, (int64_t)window + (causal ? p.tile_rows : std::max<int64_t>(n_tokens, p.tile_rows)) + 64);
    span = (span + 63) / 64 * 64;
    const int64_t units = std::max<int64_t>((int64_t)n_requests * kv_heads * p.row_tiles, 1);
    // Chunks until the grid has 8 workgroups to a compute unit (many-row kernel: one and a half times what fits, as long as there are no
    // more; each chunk's sums cost a trip to memory, and a causal prompt's first tiles end early by themselves: 8 prompts of 447 to 895
    // tokens after 134 to 404, whole and in two or three chunks, us: 8 heads of 64 33 / 41, 8 on 2 of 128 42 / 61, 6 on 2 of 256 76 / 100; but
    // one of 3000 tokens whole and in chunks of 1024: 58 / 35, 74 / 50, 121 / 79).  Of 512 keys at least, and of 1024 from dim 192 on where
    // a workgroup has few rows and a compute unit to itself, so that its beginning and end weigh more (the steps above with dim 256, 512 and
    // 1024 keys, us: 16 rows 32 / 25, 64 rows 61 / 52; dim 128 32 / 34, 76 / 79), but of 256 where even chunks of 512 do not reach every
    // compute unit, in the many-row kernel and from dim 192 on (5 requests of 1 to 30 tokens after 600 to 1900, 256 and 512 keys: 6 heads on
    // 2 of 256 25 / 34, 8 on 2 of 128 18 / 24; one row of 384 keys, dim 64, in one and two chunks 6.2 / 8.5).  Of 4096 keys at most where one
    // tile has all rows (two contexts of 100000 and 131071: 103 us, 2048 keys 115), of what the many-row kernel's LDS has room for.
    const int64_t fit = dim == 64 ? 3 : dim == 128 ? 2 : 1;
    const int64_t want = std::max<int64_t>(p.many ? 3 * fit * kAttendCus / (2 * units) : (8 * kAttendCus + units - 1) / units, 1);
    int64_t chunk = ((span + want - 1) / want + 255) / 256 * 256;
    const int64_t least = (p.many || dim >= 192) && units * ((span + 511) / 512) < kAttendCus ? 256 : dim >= 192 && p.tile_rows <= 64 ? 1024 : 512;
    chunk = std::max<int64_t>(chunk, least);
    if (p.many) chunk = std::min<int64_t>(chunk, kManyChunk);
    if (!p.many && p.row_tiles == 1) chunk = std::min<int64_t>(chunk, 4096);
    p.chunk = (int)chunk;
    p.chunks = (int)((span + chunk - 1) / chunk);
    if (p.chunks > 1) {
        p.ml_at = sat_bytes((u128)p.chunks * (u128)n_tokens * (u128)heads * (u128)dim * 4);
        p.bytes = sat_add(p.ml_at, sat_bytes((u128)p.chunks * (u128)n_tokens * (u128)heads * 8));
    }
    return p;
}

bool attend_dim_ok(int dim) { return dim == 64 || dim == 128 || dim == 192 || dim == 256; }

int check_attend_sizes(int64_t n_tokens, int n_requests, int heads, int kv_heads, int dim, int64_t max_queries, int64_t max_keys, int window,
                       int dtype)
{
    if (n_tokens < 0 || n_requests < 0 || heads < 1 || kv_heads < 1 || dim < 1 || max_queries < 0 || max_keys < 0 || max_keys > kMaxStepTokens ||
        window < 0 || window > kMaxStepTokens)
        return LFFN_E_SIZE;
    if (heads % kv_heads) return LFFN_E_SIZE;
    if (heads > kMaxHeads || !attend_dim_ok(dim)) return LFFN_E_UNSUPPORTED;
    if (n_tokens > kMaxStepTokens || n_tokens * heads > kMaxRows || (int64_t)n_requests * kv_heads > kMaxRows) return LFFN_E_SIZE;
    if (!dtype_ok(dtype)) return LFFN_E_DTYPE;
    return LFFN_OK;
}

int64_t attend_workspace_bytes(int64_t n_tokens, int n_requests, int heads, int kv_heads, int dim, int64_t max_queries, int64_t max_keys,
                               int window, int dtype)
{
    if (check_attend_sizes(n_tokens, n_requests, heads, kv_heads, dim, max_queries, max_keys, window, dtype) != LFFN_OK) return 0;
    max_queries = std::min(max_queries, n_tokens);   // enough for either, causal or not
    return std::max(plan_attend(n_tokens, n_requests, heads, kv_heads, dim, max_queries, max_keys, 1, window, dtype).bytes,
                    plan_attend(n_tokens, n_requests, heads, kv_heads, dim, max_queries, max_keys, 0, window, dtype).bytes);
}

int attend(const void *q, const void *k_cache, const void *v_cache, const float *k_scale, const float *v_scale, const int32_t *table,
           const int32_t *starts, const int32_t *lengths, void *y, int64_t n_tokens, int n_requests, int heads, int kv_heads, int dim,
           int64_t n_blocks, int block, int table_width, int64_t table_stride, const int64_t *st, int64_t max_queries, int64_t max_keys,
           int causal, int window, int dtype, void *workspace, int64_t workspace_bytes, hipStream_t s)
{
    int rc = check_attend_sizes(n_tokens, n_requests, heads, kv_heads, dim, max_queries, max_keys, window, dtype);
    if (rc != LFFN_OK) return rc;
    if (n_blocks < 1 || n_blocks > INT32_MAX || table_width < 0 || table_stride < table_width) return LFFN_E_SIZE;
    if (!block_ok(block)) return LFFN_E_UNSUPPORTED;
    if ((int64_t)block * dim * kv_heads > INT32_MAX) return LFFN_E_UNSUPPORTED;   // the kernels' offsets inside a block
    const int64_t strides[4] = {st ? st[0] : (int64_t)heads * dim, st ? st[1] : dim, st ? st[2] : (int64_t)heads * dim, st ? st[3] : dim};
    for (int64_t v : strides)
        if (v < 0) return LFFN_E_SIZE;
    max_queries = std::min(max_queries, n_tokens);
    if (n_tokens == 0 || n_requests == 0 || max_queries == 0) return LFFN_OK;
    if (!q || !k_cache || !v_cache || !k_scale || !v_scale || (table_width && !table) || !starts || !lengths || !y) return LFFN_E_NULL;
    const int elem = dtype == LFFN_F32 ? 4 : 2;
    if (!aligned(q, elem) || !aligned(y, elem) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(k_scale, 4) ||
        !aligned(v_scale, 4) || !aligned(table, 4) || !aligned(starts, 4) || !aligned(lengths, 4))
        return LFFN_E_ALIGN;
    const AttendPlan p = plan_attend(n_tokens, n_requests, heads, kv_heads, dim, max_queries, max_keys, causal, window, dtype);
    Scratch sc;
    rc = get_scratch(workspace, workspace_bytes, p.bytes, &sc);
    if (rc != LFFN_OK) return rc;
    AttendArgs a{};
    a.q = q;
    a.y = y;
    a.k_cache = static_cast<const uint8_t *>(k_cache);
    a.v_cache = static_cast<const uint8_t *>(v_cache);
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.table = table;
    a.starts = starts;
    a.lengths = lengths;
    if (p.chunks > 1) {
        a.part = reinterpret_cast<float *>(sc.base);
        a.part_ml = reinterpret_cast<float *>(sc.base + p.ml_at);
    }
    a.q_token = strides[0];
    a.q_head = strides[1];
    a.y_token = strides[2];
    a.y_head = strides[3];
    a.table_stride = table_stride;
    a.n_tokens = (int)n_tokens;
    a.requests = n_requests;
    a.heads = heads;
    a.kv_heads = kv_heads;
    a.group = heads / kv_heads;
    a.group_inverse = a.group > 1 ? (unsigned)(((uint64_t)1 << 32) / (unsigned)a.group) : 0;
    a.width = table_width;
    a.n_blocks = (int)n_blocks;
    a.block_log = log2_of(block);
    a.causal = causal != 0;
    a.window = window;
    a.max_keys = (int)std::min<int64_t>(max_keys, (int64_t)table_width * block);
    a.max_queries = (int)max_queries;
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.row_tiles = p.row_tiles;
    a.tile_rows = p.tile_rows;
    a.scale = (float)(1.4426950408889634 / std::sqrt((double)dim));
    const int64_t combos = (int64_t)n_requests * kv_heads;
    // up to 4096 rows a workgroup of the join to a row (they take 5 us to start), so that many chunks of few rows are read together
    a.join_each = n_tokens * heads > 4096;
    const int join_rows = a.join_each ? 256 / (dim / 4) : 1;
    const u128 groups = (u128)combos * (u128)p.row_tiles * (u128)p.chunks;
    const u128 joins = (u128)combos * (u128)p.row_tiles * (u128)((p.tile_rows + join_rows - 1) / join_rows);
    if (groups > (u128)INT32_MAX || joins > (u128)INT32_MAX) return LFFN_E_SIZE;
    const int64_t rows = std::min<int64_t>(p.tile_rows, attend_group_rows(heads, kv_heads, max_queries));
    rc = p.many ? lffn_host::attend_many_part(dtype, dim, a, grid_of((int64_t)groups), s)
                : lffn_host::attend_few_part(dtype, dim, a, grid_of((int64_t)groups), (size_t)(4 * rows * (dim + 4) * 4), s);
    if (rc != LFFN_OK || p.chunks == 1) return rc;
    return lffn_host::attend_join_part(dtype, dim, a, grid_of((int64_t)joins), s);
}
