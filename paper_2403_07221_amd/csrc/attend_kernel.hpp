// Attention over the 8-bit cache (keys [block][kv head][token][dim], values [block][kv head][dim][token], e4m3, a scale for each
// block and head; a request's blocks in its row of the table):
//
//   y[row] = sum_j p_j v_j / sum_j p_j,   p_j = exp(q[row] . k_j / sqrt(dim) - max),   j over the keys that the row sees:
//   those of its request, up to its own position where causal, the last `window` of those where there is a window.
// A row that sees no key is zero.
//
// Rows and precision.  The query heads that share a key head are rows of one matrix: row = query * group + head in the group.  e4m3 is
// exact in bf16 and in half, so the bytes go into the matrix cores unscaled, and a block's scale multiplies the fp32 score (keys) or
// the fp32 probability (values).  A number with more bits than the matrix cores' type is a sum of pieces, each the rounded rest of
// those before it: fp32 queries are three bf16 pieces (24 bits); probabilities times their value's scale two (16 bits, a relative
// 2^-17 each), with fp32 rows three.  Running maximum, sum and products are fp32; y is rounded once.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attend_tile.hpp"
#include "elem16.hpp"

namespace lffn {

typedef float fv4 __attribute__((ext_vector_type(4)));
typedef unsigned uv4 __attribute__((ext_vector_type(4)));
typedef unsigned uv2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 hf8 __attribute__((ext_vector_type(8)));
typedef _Float16 hf2 __attribute__((ext_vector_type(2)));

// eight e4m3 bytes as bf16 or half (exact)
__device__ __forceinline__ bf8 widen8_bf16(unsigned lo, unsigned hi)
{
    const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const bf2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return bf8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ hf8 widen8_half(unsigned lo, unsigned hi)
{
    const hf2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const hf2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return hf8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <int KIND>
struct QueryPieces;
template <>
struct QueryPieces<kElemF32> { static constexpr int N = 3; };
template <>
struct QueryPieces<kElemBF16> { static constexpr int N = 1; };
template <>
struct QueryPieces<kElemF16> { static constexpr int N = 1; };

// the matrix cores' operands of the scores: half for half rows (their 11 bits fit), bf16 else
template <int KIND>
struct ScoreOperand {
    using V = bf8;
    static __device__ __forceinline__ V widen(unsigned lo, unsigned hi) { return widen8_bf16(lo, hi); }
    static __device__ __forceinline__ fv4 mma(V a, V b, fv4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct ScoreOperand<kElemF16> {
    using V = hf8;
    static __device__ __forceinline__ V widen(unsigned lo, unsigned hi) { return widen8_half(lo, hi); }
    static __device__ __forceinline__ fv4 mma(V a, V b, fv4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// eight queries' columns as pieces
template <int KIND>
__device__ __forceinline__ void load_query8(const void *q, long long at, bool aligned, typename ScoreOperand<KIND>::V out[])
{
    if constexpr (KIND == kElemF32) {
        float v[8];
        const float *p = static_cast<const float *>(q) + at;
        if (aligned) {
            const fv4 a = reinterpret_cast<const fv4 *>(p)[0], b = reinterpret_cast<const fv4 *>(p)[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = a[i];
                v[i + 4] = b[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __bf16 a = (__bf16)v[i];
            // (an infinity or NaN has no rest)
            const bool finite = fabsf(v[i]) < __uint_as_float(0x7F800000u);
            const float ra = finite ? v[i] - (float)a : 0.0f;
            const __bf16 b = (__bf16)ra;
            out[0][i] = a;
            out[1][i] = b;
            out[2][i] = (__bf16)(ra - (float)b);
        }
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(q) + at;
        uv4 w;
        if (aligned) {
            w = *reinterpret_cast<const uv4 *>(p);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = p[2 * i] | ((unsigned)p[2 * i + 1] << 16);
        }
        out[0] = __builtin_bit_cast(typename ScoreOperand<KIND>::V, w);
    }
}

// 1 / total of a row, or zero where the row sees no key
__device__ __forceinline__ float inverse_of(float total) { return total == 0.0f ? 0.0f : 1.0f / total; }

// four columns of an output row: sums times inverse_of the sum of probabilities, rounded once to nearest even
template <int KIND>
__device__ __forceinline__ void store_row4(const AttendArgs &a, int token, int head, int column, fv4 sum, float inverse)
{
    const long long at = token * a.y_token + head * a.y_head + column;
    constexpr int E = KIND == kElemF32 ? 4 : 2;
    using T = std::conditional_t<KIND == kElemF32, float, std::conditional_t<KIND == kElemBF16, __bf16, _Float16>>;
    typedef T T4 __attribute__((ext_vector_type(4)));
    const T4 v = {(T)(sum[0] * inverse), (T)(sum[1] * inverse), (T)(sum[2] * inverse), (T)(sum[3] * inverse)};
    T *to = static_cast<T *>(a.y) + at;
    if (((reinterpret_cast<uintptr_t>(a.y) | (a.y_token * E) | (a.y_head * E)) & (4 * E - 1)) == 0) {
        *reinterpret_cast<T4 *>(to) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = v[i];
    }
}

// A larger maximum rescales a row's sums, DIM products, and of a wave's 32 rows some row finds one in most steps (at 31 steps of random
// scores still in two of three); probabilities up to 2^6 cost nothing instead: half holds 2^(8 + 6).
constexpr float kSlack = 6.0f;

// 0x80 in every byte of w that is an e4m3 NaN
__device__ __forceinline__ unsigned nan_bytes(unsigned w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// Few rows: decode steps and drafted tokens.  A workgroup has 16 rows of one request and key head and a chunk of keys; its four waves
// take steps of 64 keys in turn, each with a softmax of its own, and are joined in LDS at the end.
//
// What bounds it: the cache's bytes.  They go from memory straight into the operand registers: no LDS, no barrier in the loop.  Scores
// are S^T = K Q^T in tiles of 16 keys x 16 rows, so that a row's probabilities lie along one lane column.  The key that row m of tile t
// stands for is 16 (m / 4) + 4 t + m % 4 of the step: lane group g then ends up with the probabilities of keys 16 g .. 16 g + 15, which
// is what it holds of the values' operand with one 16-byte load for each column (a block has at least 16 tokens), and all of whose keys
// lie in one block: one scale.  A lane group takes the columns 64 j + 16 g .. + 15 of a key, so its loads are 16 bytes too.
// Measured with the join: 64 contexts of 500 to 8191, 32 heads on 8 of 128, 100 us, 4.3 TB/s; two of 100000 and 131071 100 us, 5.0 TB/s.
template <int KIND, int DIM>
__global__ __launch_bounds__(256, DIM <= 128 ? 2 : 1) void attend_few_kernel(AttendArgs a)
{
    using Op = ScoreOperand<KIND>;
    using V = typename Op::V;
    constexpr int J = DIM / 64, D = DIM / 16, NQ = QueryPieces<KIND>::N, NP = KIND == kElemF32 ? 3 : 2, ROWS = 16, PITCH = DIM + 4;
    constexpr float kNone = -__builtin_huge_valf();
    extern __shared__ float attend_lds[];   // [wave][row][PITCH] of the rows that there are
    __shared__ float wave_m[4][ROWS], wave_l[4][ROWS];
    const unsigned wg = blockIdx.y * gridDim.x + blockIdx.x, combos = (unsigned)(a.requests * a.kv_heads), rest = wg / combos;
    const int combo = (int)(wg - rest * combos), chunk = (int)(rest / (unsigned)a.row_tiles), tile = (int)rest - chunk * a.row_tiles;
    if (chunk >= a.chunks) return;
    const RowTile t = row_tile(a, combo, tile, ROWS);
    if (t.row0 >= t.rows) return;
    int c0, c1;
    chunk_keys(a, t, chunk, c0, c1);
    if (c0 >= c1 && chunk > 0) return;
    // one chunk has all the tile's keys (or there are none, or the grid, for requests that bring more than max_queries): y is written here
    const bool whole = t.hi - t.lo <= a.chunk || a.chunks == 1;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, g = lane >> 4;
    const int n_rows = min(ROWS, t.rows - t.row0);

    // the rows' queries, as the right operand: column lr, k of step (j, half) = columns 64 j + 16 g + 8 half ..
    constexpr int E = KIND == kElemF32 ? 4 : 2;
    const bool q_aligned = (((reinterpret_cast<uintptr_t>(a.q) | (a.q_token * E) | (a.q_head * E)) & 15) == 0);
    V q[J][2][NQ];
    int key_lo, key_hi;
    {
        const int row = min(t.row0 + lr, t.rows - 1), i = query_of(a, row), head = t.h * a.group + (row - i * a.group);
        row_keys(a, t, row, key_lo, key_hi);
        const long long at = (long long)(t.first + i) * a.q_token + head * a.q_head;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int half = 0; half < 2; ++half) load_query8<KIND>(a.q, at + 64 * j + 16 * g + 8 * half, q_aligned, q[j][half]);
    }
    // keys that every row of the tile sees: steps inside need no mask
    int all_lo, all_hi;
    {
        int x, y;
        row_keys(a, t, t.row0, x, y);
        all_hi = y;
        row_keys(a, t, t.row0 + n_rows - 1, x, y);
        all_lo = x;
    }

    fv4 o[D];
    float m = kNone, l = 0.0f;
#pragma unroll
    for (int d = 0; d < D; ++d) o[d] = fv4{0.0f, 0.0f, 0.0f, 0.0f};
    const int *table = a.table + t.r * a.table_stride;
    const int in_block = (1 << a.block_log) - 1, sk = lr >> 2;
    const long long head_bytes = (long long)DIM << a.block_log;

    // A step's keys leave their registers with its scores and its values with its sums, so the next step's are on their way while
    // this one's softmax and sums go on; the blocks of the step after that are looked up meanwhile.
    uv4 kr[4][J], vr[D];
    int entry_k, entry_v;      // the table's entries of the step to fetch next
    float ks_next, vs_next;
    auto look_up = [&](int key0) {
        entry_k = table_entry(a, table, key0 + 16 * sk);
        entry_v = table_entry(a, table, key0 + 16 * g);
    };
    auto fetch_keys = [&](int key0, int id_k, int id_v) {
        const uint8_t *kp = a.k_cache + ((long long)max(id_k, 0) * a.kv_heads + t.h) * head_bytes +
                            (long long)(((key0 + 16 * sk) & in_block) + (lr & 3)) * DIM + 16 * g;
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int j = 0; j < J; ++j) kr[tt][j] = *reinterpret_cast<const uv4 *>(kp + 4 * tt * DIM + 64 * j);
        const long long at = (long long)max(id_v, 0) * a.kv_heads + t.h;
        ks_next = a.k_scale[at];
        vs_next = a.v_scale[at];
    };
    auto fetch_values = [&](int key0, int id_v) {
        const uint8_t *vp = a.v_cache + ((long long)max(id_v, 0) * a.kv_heads + t.h) * head_bytes + ((long long)lr << a.block_log) +
                            ((key0 + 16 * g) & in_block);
#pragma unroll
        for (int d = 0; d < D; ++d) vr[d] = *reinterpret_cast<const uv4 *>(vp + ((long long)(16 * d) << a.block_log));
    };
    int key0 = c0 + 64 * w;
    bool valid = false;
    entry_k = entry_v = -1;
    if (a.width) look_up(key0);
    // (the queries and these, once: where the compiler cannot tell how many loads are under way, it waits for all in every step)
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    if (key0 < c1) {
        const int id_k = block_of(a, entry_k, key0 + 16 * sk, c1), id_v = block_of(a, entry_v, key0 + 16 * g, c1);
        look_up(key0 + 256);
        valid = id_v >= 0;
        fetch_keys(key0, id_k, id_v);
        fetch_values(key0, id_v);
    }
    // (all steps but the last fetch another: without a branch around its loads the waits count them one by one)
    auto step = [&](auto fetches) {
        constexpr bool more = decltype(fetches)::value;
        const float ks = ks_next * a.scale, vs = vs_next;
        const int next_k = block_of(a, entry_k, key0 + 256 + 16 * sk, c1), next_v = block_of(a, entry_v, key0 + 256 + 16 * g, c1);
        const bool masked = key0 < all_lo || key0 + 64 > min(all_hi, c1) || __any(!valid);

        fv4 s[4];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) s[tt] = fv4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const V k8 = Op::widen(kr[tt][j][2 * half], kr[tt][j][2 * half + 1]);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) s[tt] = Op::mma(k8, q[j][half][n], s[tt]);
                }

        if constexpr (more) {
            look_up(key0 + 512);
            fetch_keys(key0 + 256, next_k, next_v);
        }

        bf8 p[2][NP];   // the probabilities' pieces: [32 keys of 16 g ..: halves of 8]
        float x[16], top = kNone;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = s[e >> 2][e & 3] * ks;
            if (masked) {
                const int key = key0 + 16 * g + e;
                x[e] = valid && key >= key_lo && key < min(key_hi, c1) ? x[e] : kNone;
            }
            top = fmaxf(top, x[e]);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        // The maximum that the powers are taken from follows the rows' own only where one has left it kSlack behind.
        if (__any(top > m + kSlack)) {
            const float now = fmaxf(m, top), f = now == m ? 1.0f : __builtin_amdgcn_exp2f(m - now);
            l *= f;
#pragma unroll
            for (int d = 0; d < D; ++d) o[d] *= f;
            m = now;
        }
        const float base = m == kNone ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float pe = __builtin_amdgcn_exp2f(x[e] - base);
            sum += pe;
            float rest = pe * vs;
            if (masked) rest = x[e] == kNone ? 0.0f : rest;   // (the scale of a block that is not there may be anything)
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                const __bf16 piece = (__bf16)rest;
                p[e >> 3][n][e & 7] = piece;
                rest -= (float)piece;
            }
        }
        l += sum;
        // A masked key's probability is zero, but zero times a NaN byte is not: in masked steps such bytes become zeros, and
        // the rows that do see one get their NaN from a product with ones in its place.  (A seen key whose probability is too small for
        // bf16 takes the smallest in such a step.)
        bool nans = false;
        if (masked) {
            unsigned any = 0;
#pragma unroll
            for (int d = 0; d < D; ++d) any |= nan_bytes(vr[d][0]) | nan_bytes(vr[d][1]) | nan_bytes(vr[d][2]) | nan_bytes(vr[d][3]);
            nans = __any(any != 0);
        }
        if (__builtin_expect(nans, false)) {
            // (bit e: whether the row sees key 16 g + e of the step; anew, or the masks of all sixteen scores are kept until here)
            const int at = key0 + 16 * g, from = min(max(key_lo - at, 0), 16), to = valid ? min(max(min(key_hi, c1) - at, 0), 16) : 0;
            const unsigned seen = ((1u << to) - 1) & (~0u << from);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uv4 words = __builtin_bit_cast(uv4, p[u][0]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned shift = 16 * (e & 1), small = (words[e >> 1] >> shift & 0x7F80u) == 0;
                    words[e >> 1] |= (seen >> (8 * u + e) & small) << (7 + shift);   // 2^-126
                }
                p[u][0] = __builtin_bit_cast(bf8, words);
            }
#pragma unroll
            for (int d = 0; d < D; ++d) {
                uv4 ones;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned b = nan_bytes(vr[d][i]) >> 7;
                    vr[d][i] &= ~(b * 0xFFu);
                    ones[i] = b * 0x38u;   // 1.0
                }
                fv4 hit = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8_bf16(ones[2 * u], ones[2 * u + 1]), p[u][0], hit, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (hit[i] != 0.0f) o[d][i] = __uint_as_float(0x7FC00000u);
            }
        }
#pragma unroll
        for (int d = 0; d < D; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf8 v8 = widen8_bf16(vr[d][2 * u], vr[d][2 * u + 1]);
#pragma unroll
                for (int n = 0; n < NP; ++n) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, p[u][n], o[d], 0, 0, 0);
            }
        if constexpr (more) fetch_values(key0 + 256, next_v);
        valid = next_v >= 0;
    };
    for (; key0 + 256 < c1; key0 += 256) step(std::true_type{});
    if (key0 < c1) step(std::false_type{});

    // the four waves' sums: a lane column's sum over its groups, then the waves' through LDS
    float *mine = attend_lds + (long long)w * n_rows * PITCH;
    {
        float sum = l;
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (g == 0) {
            wave_m[w][lr] = m;
            wave_l[w][lr] = sum;
        }
        if (lr < n_rows) {
#pragma unroll
            for (int d = 0; d < D; ++d) *reinterpret_cast<fv4 *>(mine + lr * PITCH + 16 * d + 4 * g) = o[d];
        }
    }
    __syncthreads();
    for (int at = tid; at < n_rows * (DIM / 4); at += 256) {
        const int row = at / (DIM / 4), column = (at % (DIM / 4)) * 4;
        float top = kNone, total = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, wave_m[i][row]);
        const float base = top == kNone ? 0.0f : top;
        fv4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = __builtin_amdgcn_exp2f(wave_m[i][row] - base);
            total += wave_l[i][row] * f;
            sum += *reinterpret_cast<const fv4 *>(attend_lds + ((long long)i * n_rows + row) * PITCH + column) * f;
        }
        const int i = query_of(a, t.row0 + row), head = t.h * a.group + (t.row0 + row) - i * a.group, token = t.first + i;
        if (!whole) {
            const long long to = ((long long)chunk * a.n_tokens + token) * a.heads + head;
            *reinterpret_cast<fv4 *>(a.part + to * DIM + column) = sum;
            if (column == 0) {
                a.part_ml[to * 2] = top;
                a.part_ml[to * 2 + 1] = total;
            }
        } else {
            store_row4<KIND>(a, token, head, column, sum, inverse_of(total));
        }
    }
}

// Many rows: prompts and encodings.  A workgroup has 128 rows of one request and key head, a wave 32 (KS = 2: 64, and of a step's two tiles
// of 32 keys each wave has one; two waves join at the end); its keys go through LDS in steps of 64, widened to the matrix cores' type once
// for all four waves.  Measured: 4 prompts of 3500 to 4096 tokens, 32 heads on 8 of 128, 594 to 611 us, 800 to 820 TFLOP/s; 64 encodings of 300 to 512,
// 12 heads of 64, 77 us, 460 TFLOP/s; 24 requests with 3 to 8 drafted tokens, 16 heads on 2 of 256 (KS = 2), 46 us, 1.2 TB/s.
//
// What bounds it: the matrix cores, and beside them the softmax's vector instructions.  Scores are S^T = K Q^T in tiles of 32 keys x 32
// rows, so a row's probabilities lie along a lane column, and as they stand they are the right operand of y^T = V^T P^T: a lane half h
// holds keys 16 u + 8 h .. + 7 of the tile's step u because row m of the tile stands for key m with its bits 2 and 3 exchanged.
//
// Scales cost no instruction for each score: they are powers of two as rotate_append writes them, so the widening multiplies by the
// block's scale relative to the largest of the chunk.  That is exact down to 2^-15 (the smallest byte is 2^-9, half's smallest number
// 2^-24), and is done down to 2^-kSpread.  Probabilities of 16-bit rows are half there (11 bits, off by a relative 2^-11 at most, as fine as
// the finest 16-bit output) times 2^8, so that those of 2^-22 still have all their bits and smaller ones are off by 2^-33 at most; fp32 rows
// keep three bf16 pieces (24 bits).
//
// A chunk with a scale that is no power of two, or with scales further apart, is `exact`: its bytes stay as they are, a block's scale
// multiplies its fp32 scores or its fp32 probabilities, and those are two bf16 pieces (16-bit rows), as in the few-row kernel.  So no block's
// scale costs the bits of another's bytes, and nothing of a block reaches a row that does not see it.  All of its steps cost what that takes:
// the prompts above 1012 to 1022 us, the encodings 153, the drafted tokens 58.
constexpr int kManyKeys = 64;
constexpr float kProbUp = 8.0f;   // probabilities times 2^8
// Scales of a chunk lie at most 2^8 apart: 8192 probabilities off by 2^-33 each, of values 2^8 times the row's others, are then no more than
// the rounding of one probability.
constexpr int kSpread = 8;

constexpr int kManyChunk = 8192;  // the most keys of a chunk: its segments lie in LDS
constexpr int kManySegments = kManyChunk / 16 + 16;   // and some past the last

template <int KIND, int DIM>
struct ManyShape {
    static constexpr int KP = DIM + 8, VP = kManyKeys + 8;   // pitches of a key's columns and a column's keys: no bank is read twice
    static constexpr int BUFFER = kManyKeys * KP + DIM * VP;   // 16-bit words
    static constexpr size_t LDS = 2 * BUFFER * 2;
};

typedef float fv16 __attribute__((ext_vector_type(16)));

template <bool HALF>
struct Operand {   // of the 32 x 32 x 16 products
    using V = bf8;
    static __device__ __forceinline__ V widen(unsigned lo, unsigned hi, float f)
    {
        const bf2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, true);
        const bf2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, true);
        return V{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ fv16 mma(V a, V b, fv16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Operand<true> {
    using V = hf8;
    static __device__ __forceinline__ V widen(unsigned lo, unsigned hi, float f)
    {
        const hf2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, f, true);
        const hf2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, f, true);
        return V{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    static __device__ __forceinline__ fv16 mma(V a, V b, fv16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((unsigned)(min(max(e, -126), 127) + 127) << 23); }
__device__ __forceinline__ bool power_of_two(float s)   // 2^-126 .. 2^127
{
    const unsigned u = __float_as_uint(s);
    return (u & 0x807FFFFFu) == 0 && u >= 0x00800000u && u < 0x7F800000u;
}
__device__ __forceinline__ int exponent_of(float s) { return (int)((__float_as_uint(s) >> 23) & 255u) - 127; }
typedef short sv2 __attribute__((ext_vector_type(2)));

#define LFFN_INLINE __attribute__((always_inline))   // (a lambda that both kinds of chunks call would keep its sums in memory)

__device__ __forceinline__ float lane_of(float x, int lane)
{
    return __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane));
}

template <int KIND, int DIM, int KS>
__global__ __launch_bounds__(256, KIND == kElemF32 || DIM > 128 ? 1 : DIM == 64 ? 3 : 2) void attend_many_kernel(AttendArgs a)
{
    using Shape = ManyShape<KIND, DIM>;
    using KO = Operand<KIND == kElemF16>;     // keys and queries
    using VO = Operand<KIND != kElemF32>;     // values and probabilities
    using XO = Operand<false>;                // those of an exact chunk
    constexpr int NQ = QueryPieces<KIND>::N, NP = KIND == kElemF32 ? 3 : 1, XP = KIND == kElemF32 ? 3 : 2;   // pieces
    constexpr int ROWS = 128 / KS, KP = Shape::KP, VP = Shape::VP;
    constexpr int T = 2 / KS;                 // tiles of 32 keys that a wave has of a step
    constexpr int PIECES = DIM / 64;          // 16-byte pieces of keys, and of values, that a thread stages
    // LDS reads ahead of the products.  Of 256 columns more than two leave too few registers, and the compiler drops the order: 8 prompts of 447 to
    // 895 tokens after 134 to 404, 6 heads on 2 of 256, 72 us, with eight 79; 24 requests with 3 to 8 drafted tokens, 16 heads on 2, 46 and 47.
    constexpr int FIRST = DIM == 64 ? 4 : DIM == 256 ? 2 : 8;
    constexpr float kNone = -__builtin_huge_valf();
    extern __shared__ uint16_t many_lds[];
    __shared__ uint64_t nan_keys[2][DIM];   // of a step that some row sees in part: the keys whose value is NaN in a column
    __shared__ uint32_t nans[2][4];        // whether a wave has staged any
    __shared__ uv2 segments[kManySegments];       // block or -1; the upper halves of the keys' and the values' relative scale
    __shared__ int tops[4][3];   // of a wave's segments: the largest exponents, the smallest negated, whether some scale is no power of two
    const unsigned wg = blockIdx.y * gridDim.x + blockIdx.x, combos = (unsigned)(a.requests * a.kv_heads), rest = wg / combos;
    const int combo = (int)(wg - rest * combos), chunk = (int)(rest / (unsigned)a.row_tiles);
    if (chunk >= a.chunks) return;
    // the last rows see the most keys: they go first
    const int tile = a.row_tiles - 1 - ((int)rest - chunk * a.row_tiles);
    const RowTile t = row_tile(a, combo, tile, ROWS);
    if (t.row0 >= t.rows) return;
    int c0, c1;
    chunk_keys(a, t, chunk, c0, c1);
    if (c0 >= c1 && chunk > 0) return;
    // one chunk has all the tile's keys (or there are none, or the grid, for requests that bring more than max_queries): y is written here
    const bool whole = t.hi - t.lo <= a.chunk || a.chunks == 1;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 31, h = lane >> 5;
    const int wave_row0 = t.row0 + (w % (4 / KS)) * 32, tile0 = KS == 1 ? 0 : w >> 1;   // tile0: the wave's first tile of a step

    constexpr int E = KIND == kElemF32 ? 4 : 2;
    const bool q_aligned = (((reinterpret_cast<uintptr_t>(a.q) | (a.q_token * E) | (a.q_head * E)) & 15) == 0);
    typename KO::V q[DIM / 16][NQ];
    int key_lo, key_hi;
    {
        const int row = min(wave_row0 + lr, t.rows - 1), i = query_of(a, row), head = t.h * a.group + (row - i * a.group);
        row_keys(a, t, row, key_lo, key_hi);
        const long long at = (long long)(t.first + i) * a.q_token + head * a.q_head;
#pragma unroll
        for (int c = 0; c < DIM / 16; ++c) load_query8<KIND>(a.q, at + 16 * c + 8 * h, q_aligned, q[c]);
    }
    // the keys that some, and that all, of this wave's rows see, and that all of the workgroup's do
    int some_lo, some_hi, all_lo, all_hi, tile_lo, tile_hi;
    {
        const int first = min(wave_row0, t.rows - 1), last = min(wave_row0 + 31, t.rows - 1);
        int x;
        row_keys(a, t, first, some_lo, all_hi);
        row_keys(a, t, last, all_lo, some_hi);
        if (wave_row0 >= t.rows) some_hi = 0;
        some_hi = min(some_hi, c1);
        all_hi = min(all_hi, c1);
        row_keys(a, t, t.row0, x, tile_hi);
        row_keys(a, t, min(t.row0 + ROWS, t.rows) - 1, tile_lo, x);
        tile_hi = min(tile_hi, c1);
    }
    auto edge = [&](int key0) { return key0 < tile_lo || key0 + kManyKeys > tile_hi; };
    auto visible = [&](int key0) { return key0 < some_hi && key0 + kManyKeys > some_lo; };

    fv16 o[DIM / 32];
    float m = kNone, l = 0.0f;
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d) o[d] = fv16{};
    const int *table = a.table + t.r * a.table_stride;
    const int in_block = (1 << a.block_log) - 1;
    const long long head_bytes = (long long)DIM << a.block_log;

    const int steps = c0 < c1 ? (c1 - c0 + kManyKeys - 1) / kManyKeys : 0;
    // The chunk's segments of 16 keys, all looked up before the first step: their blocks, and their scales relative to the largest
    // (as they are, in an exact chunk).
    float k_unit = 1.0f, v_unit = 1.0f;   // what the largest are
    bool exact;
    {
        sv2 top = {-300, -300}, low = top;   // exponents of keys' and values' scales, and those negated
        bool odd = false;
        for (int i = tid; i < 4 * (steps + 1); i += 256) {
            const int key = c0 + 16 * i, id = a.width ? block_of(a, table_entry(a, table, key), key, c1) : -1;
            const long long at = (long long)max(id, 0) * a.kv_heads + t.h;
            const float ks = id >= 0 ? a.k_scale[at] : 1.0f, vs = id >= 0 ? a.v_scale[at] : 1.0f;
            const int ek = exponent_of(ks), ev = exponent_of(vs);
            segments[i] = uv2{(unsigned)id, (unsigned)(ek + 256) << 16 | (unsigned)(ev + 256)};
            odd |= !power_of_two(ks) || !power_of_two(vs);
            if (id >= 0) {
                top = __builtin_elementwise_max(top, sv2{(short)ek, (short)ev});
                low = __builtin_elementwise_max(low, sv2{(short)-ek, (short)-ev});
            }
        }
        for (int d = 1; d < 64; d <<= 1) {
            top = __builtin_elementwise_max(top, __builtin_bit_cast(sv2, __shfl_xor(__builtin_bit_cast(int, top), d)));
            low = __builtin_elementwise_max(low, __builtin_bit_cast(sv2, __shfl_xor(__builtin_bit_cast(int, low), d)));
        }
        const int any = __any(odd);
        if (lane == 0) {
            tops[w][0] = __builtin_bit_cast(int, top);
            tops[w][1] = __builtin_bit_cast(int, low);
            tops[w][2] = any;
        }
        __syncthreads();
        int any_odd = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top = __builtin_elementwise_max(top, __builtin_bit_cast(sv2, tops[i][0]));
            low = __builtin_elementwise_max(low, __builtin_bit_cast(sv2, tops[i][1]));
            any_odd |= tops[i][2];
        }
        const int k_top = __builtin_amdgcn_readfirstlane(top[0]), v_top = __builtin_amdgcn_readfirstlane(top[1]);
        exact = __builtin_amdgcn_readfirstlane(any_odd != 0 || k_top + low[0] > kSpread || v_top + low[1] > kSpread) != 0;
        if (!exact) {
            k_unit = pow2f(k_top);
            v_unit = pow2f(v_top);
        }
        for (int i = tid; i < 4 * (steps + 1); i += 256) {
            const uv2 e = segments[i];
            const unsigned rel = __float_as_uint(pow2f((int)(e[1] >> 16) - 256 - k_top)) | __float_as_uint(pow2f((int)(e[1] & 0xFFFFu) - 256 - v_top)) >> 16;
            // (bytes that stand in for a block that is not there become zeros, or all but)
            segments[i][1] = (int)e[0] < 0 ? 0u : exact ? 0x3F803F80u : rel;
        }
        __syncthreads();
    }

    uv4 kr[PIECES], vr[PIECES];
    const int seg16 = 16 * (lane & 3);
    // A wave stages the keys of segment w, whose sixteen rows lie together in their block, and of the values the segment of each lane.
    const int v_column = tid >> 2;      // the first of this lane's columns, 64 apart
    // (32 bits hold a block's bytes over all heads, and the scales' indices: checked before the launch)
    const unsigned block_bytes = (unsigned)(a.kv_heads * head_bytes);
    const uint8_t *k_head = a.k_cache + t.h * head_bytes, *v_head = a.v_cache + t.h * head_bytes + ((long long)v_column << a.block_log);
    auto segment = [&](int step) { return segments[4 * step + (lane & 3)]; };   // of this lane
    auto fetch = [&](int step, const uv2 &e) LFFN_INLINE {
        const int key0 = c0 + step * kManyKeys, id = max((int)e[0], 0);
        const uint8_t *kp = k_head + (unsigned long long)(unsigned)__builtin_amdgcn_readlane(id, w) * block_bytes + ((key0 + 16 * w) & in_block) * DIM;
        const uint8_t *vp = v_head + (unsigned long long)(unsigned)id * block_bytes + ((key0 + seg16) & in_block);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            kr[p] = *reinterpret_cast<const uv4 *>(kp + 16 * (lane + 64 * p));
            vr[p] = *reinterpret_cast<const uv4 *>(vp + (64 * p << a.block_log));
        }
    };
    auto stage = [&](auto exactly, int buffer, int step, const uv2 &e) LFFN_INLINE {   // e: segment(step), as it was fetched
        const bool there = (int)e[0] >= 0;
        // Steps that some row sees in part: a masked key's probability is zero, but zero times a NaN byte is not.  Such bytes become
        // zeros, and their places go to the rows that do see them.
        if (edge(c0 + step * kManyKeys) || __any(!there)) {
            bool any = false;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                unsigned bits = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned b = nan_bytes(vr[p][i]) >> 7;
                    vr[p][i] &= ~(b * 0xFFu);
                    bits |= ((b * 0x10204080u) >> 28) << (4 * i);   // a bit for each byte
                }
                bits = there ? bits : 0;
                any |= bits != 0;
                reinterpret_cast<uint16_t *>(&nan_keys[buffer][v_column + 64 * p])[lane & 3] = (uint16_t)bits;
            }
            const unsigned some = __any(any);
            if (lane == 0) nans[buffer][w] = some;
        }
        const float fk = lane_of(__uint_as_float(e[1] & 0xFFFF0000u), w), fv = __uint_as_float(e[1] << 16);
        uint16_t *kb = many_lds + buffer * Shape::BUFFER, *vb = kb + kManyKeys * KP;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int piece = lane + 64 * p, key = 16 * w + piece / (DIM / 16), column = (piece % (DIM / 16)) * 16;
            typename KO::V *to = reinterpret_cast<typename KO::V *>(kb + key * KP + column);
            to[0] = KO::widen(kr[p][0], kr[p][1], fk);
            to[1] = KO::widen(kr[p][2], kr[p][3], fk);
            using O = std::conditional_t<decltype(exactly)::value, XO, VO>;
            typename O::V *tv = reinterpret_cast<typename O::V *>(vb + (v_column + 64 * p) * VP + seg16);
            tv[0] = O::widen(vr[p][0], vr[p][1], fv);
            tv[1] = O::widen(vr[p][2], vr[p][3], fv);
        }
    };

    const int key_of = (lr & 19) | ((lr & 4) << 1) | ((lr & 8) >> 1);   // bits 2 and 3 exchanged
    // (bits of a step's four segments: whether they are there)
    auto there_of = [&](int step) { return (unsigned)__ballot((int)segment(step)[0] >= 0) & 15u; };
    auto masked = [&](int key0, unsigned there) { return key0 < all_lo || key0 + kManyKeys > all_hi || there != 15u; };
    // the keys of a step that a row sees, a bit each
    auto seen_keys = [&](int key0, unsigned there) LFFN_INLINE {
        int lo = key_lo, hi = key_hi;
        asm volatile("" : "+v"(lo), "+v"(hi));   // (not to be worked out in the steps without a mask)
        const int from = min(max(lo - key0, 0), 64), to = min(max(min(hi, c1) - key0, 0), 64);
        const uint64_t below = to == 64 ? ~0ull : (1ull << to) - 1;
        const uint64_t in = (there & 1u ? 0xFFFFull : 0) | (there & 2u ? 0xFFFFull << 16 : 0) | (there & 4u ? 0xFFFFull << 32 : 0) |
                            (there & 8u ? 0xFFFFull << 48 : 0);
        return from == 64 ? 0 : below & (~0ull << from) & in;
    };
    fv16 s[T];
    auto scores = [&](int buffer) LFFN_INLINE {
        const uint16_t *kb = many_lds + buffer * Shape::BUFFER;
#pragma unroll
        for (int tt = 0; tt < T; ++tt) s[tt] = fv16{};
#pragma unroll
        for (int c = 0; c < DIM / 16; ++c)
#pragma unroll
            for (int tt = 0; tt < T; ++tt) {
                const typename KO::V k8 = *reinterpret_cast<const typename KO::V *>(kb + (32 * (tile0 + tt) + key_of) * KP + 16 * c + 8 * h);
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[tt] = KO::mma(k8, q[c][n], s[tt]);
            }
    };
    const float unit = k_unit * a.scale;
    // the scale of the block of segment u of the wave's tiles
    auto scale_of_segment = [&](const float *scale, int step, int u) {
        const int id = (int)segments[4 * step + 2 * tile0 + u][0];
        return id >= 0 ? scale[(long long)id * a.kv_heads + t.h] : 1.0f;
    };
    auto softmax = [&](auto exactly, int step, auto &p) LFFN_INLINE {   // p: pieces of the probabilities, of 16 keys of the wave's tiles each
        constexpr bool EXACT = decltype(exactly)::value;
        const int key0 = c0 + step * kManyKeys;
        const unsigned there = there_of(step);
        if constexpr (EXACT) {
#pragma unroll
            for (int u = 0; u < 2 * T; ++u) {
                const float ks = scale_of_segment(a.k_scale, step, u);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[u >> 1][8 * (u & 1) + e] *= ks;
            }
        }
        const bool partly = masked(key0, there);
        unsigned words[T];   // bit 16 (e / 8) + e % 8 of word tt: whether the row sees the key of s[tt][e]
        if (partly) {
            const uint64_t seen = seen_keys(key0, there);
#pragma unroll
            for (int tt = 0; tt < T; ++tt) {
                words[tt] = (unsigned)(seen >> (32 * (tile0 + tt))) >> (8 * h);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!(words[tt] & (1u << (16 * (e >> 3) + (e & 7))))) s[tt][e] = kNone;
            }
        }
        float top = kNone;
#pragma unroll
        for (int tt = 0; tt < T; ++tt)
#pragma unroll
            for (int e = 0; e < 16; ++e) top = fmaxf(top, s[tt][e]);
        top = fmaxf(top, __shfl_xor(top, 32)) * unit;
        // The maximum that the powers are taken from follows the rows' own only where one has left it kSlack behind.
        if (__any(top > m + kSlack)) {
            const float now = fmaxf(m, top), down = now == m ? 1.0f : __builtin_amdgcn_exp2f(m - now);
            l *= down;
#pragma unroll
            for (int d = 0; d < DIM / 32; ++d) o[d] *= down;
            m = now;
        }
        const float base = (m == kNone ? 0.0f : m) - (EXACT ? 0.0f : kProbUp);
#pragma unroll
        for (int tt = 0; tt < T; ++tt)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[tt][e] = __builtin_amdgcn_exp2f(fmaf(s[tt][e], unit, -base));
#pragma unroll
        for (int u = 0; u < 2 * T; ++u) {
            float vs = 1.0f;
            if constexpr (EXACT) vs = scale_of_segment(a.v_scale, step, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float rest = s[u >> 1][8 * (u & 1) + e];
                if constexpr (EXACT) {
                    rest *= vs;
                    if (partly) rest = words[u >> 1] & (1u << (16 * (u & 1) + e)) ? rest : 0.0f;   // (a scale that the row does not see may be anything)
                }
                constexpr int N = EXACT ? XP : NP;
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    p[u][n][e] = rest;
                    if (n + 1 < N) rest -= (float)p[u][n][e];
                }
            }
        }
        // (the sum is of the probabilities as they are, not as they were rounded)
#pragma unroll
        for (int tt = 0; tt < T; ++tt)
#pragma unroll
            for (int e = 0; e < 16; ++e) l += s[tt][e];
    };
    auto sums = [&](auto exactly, int buffer, const auto &p) LFFN_INLINE {
        using O = std::conditional_t<decltype(exactly)::value, XO, VO>;
        constexpr int N = decltype(exactly)::value ? XP : NP;
        const uint16_t *vb = many_lds + buffer * Shape::BUFFER + kManyKeys * KP;
#pragma unroll
        for (int d2 = 0; d2 < DIM / 32; d2 += 2)   // (two sums in turn)
#pragma unroll
            for (int u = 0; u < 2 * T; ++u)
#pragma unroll
                for (int d = d2; d < d2 + 2; ++d) {
                    const typename O::V v8 = *reinterpret_cast<const typename O::V *>(vb + (32 * d + lr) * VP + 32 * tile0 + 16 * u + 8 * h);
#pragma unroll
                    for (int n = 0; n < N; ++n) o[d] = O::mma(v8, p[u][n], o[d]);
                }
    };
    // the sums of rows that see a NaN value, of the steps whose NaN bytes stage() has cleared: also for waves whose rows see all of the step
    auto nan_rows = [&](int buffer, int step) LFFN_INLINE {
        const int key0 = c0 + step * kManyKeys;
        const unsigned there = there_of(step);
        if (!edge(key0) && there == 15u) return;
        unsigned some_nan = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) some_nan |= nans[buffer][i];
        if (some_nan) {
            const uint64_t mine = KS == 1 ? ~0ull : 0xFFFFFFFFull << (32 * tile0), seen = seen_keys(key0, there) & mine;
#pragma unroll
            for (int d = 0; d < DIM / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint64_t bad = nan_keys[buffer][32 * d + 8 * (i >> 2) + 4 * h + (i & 3)];
                    o[d][i] = (bad & seen) != 0 ? __uint_as_float(0x7FC00000u) : o[d][i];
                }
        }
    };
    // Reads from LDS ahead of the products that take them, `first` of them and then one with each product: left alone, a product waits for
    // the two reads before it.
    auto reads_ahead = [](auto first, auto products) {
        constexpr int F = decltype(first)::value, N = decltype(products)::value;
        __builtin_amdgcn_sched_group_barrier(0x100, F, 0);   // LDS reads
#pragma unroll
        for (int i = 0; i < N - F; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);   // a product
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, F, 0);
    };

    auto run = [&](auto exactly) LFFN_INLINE {
        constexpr bool EXACT = decltype(exactly)::value;
        uv2 ahead = {};         // the segment of the step whose bytes are on their way
        if (steps > 0) {
            ahead = segment(0);
            fetch(0, ahead);
            stage(exactly, 0, 0, ahead);
        }
        __syncthreads();
        for (int i = 0; i < steps; ++i) {
            // (past the last step too, of block 0: with a branch around its loads, the waits in a step are for all of them)
            ahead = segment(i + 1);
            fetch(i + 1, ahead);
            if (visible(c0 + i * kManyKeys)) {
                typename std::conditional_t<EXACT, XO, VO>::V p[2 * T][EXACT ? XP : NP];
                scores(i & 1);
                if constexpr (KIND != kElemF32) reads_ahead(std::integral_constant<int, FIRST>{}, std::integral_constant<int, DIM / 16 * T>{});
                softmax(exactly, i, p);
                __builtin_amdgcn_sched_barrier(0);
                sums(exactly, i & 1, p);
                if constexpr (KIND != kElemF32 && !EXACT) reads_ahead(std::integral_constant<int, FIRST>{}, std::integral_constant<int, DIM / 16 * T>{});
                nan_rows(i & 1, i);
            }
            stage(exactly, ~i & 1, i + 1, ahead);
            __syncthreads();
        }
    };
    if (__builtin_expect(exact, false))
        run(std::true_type{});
    else
        run(std::false_type{});

    // (probabilities as they are from here on: chunks of both kinds are joined)
    const float lift = exact ? 1.0f : __builtin_amdgcn_exp2f(-kProbUp), up = v_unit * lift;
    float total = (l + __shfl_xor(l, 32)) * lift;
    if constexpr (KS > 1) {
        // the two waves of a row block: the later's sums go through LDS (whose steps are over) to the earlier
        float *from = reinterpret_cast<float *>(many_lds) + (w & 1) * (DIM / 2 + 2) * 64;
        if (tile0) {
#pragma unroll
            for (int d = 0; d < DIM / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) from[(16 * d + i) * 64 + lane] = o[d][i];
            from[DIM / 2 * 64 + lane] = m;
            from[(DIM / 2 + 1) * 64 + lane] = total;
        }
        __syncthreads();
        if (tile0) return;
        const float other = from[DIM / 2 * 64 + lane], top = fmaxf(m, other), base = top == kNone ? 0.0f : top;
        const float f = __builtin_amdgcn_exp2f(m - base), g = __builtin_amdgcn_exp2f(other - base);
        total = total * f + from[(DIM / 2 + 1) * 64 + lane] * g;
        m = top;
#pragma unroll
        for (int d = 0; d < DIM / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * f + from[(16 * d + i) * 64 + lane] * g;
    }
    const int row = wave_row0 + lr;
    if (row >= t.rows) return;
    const int i = query_of(a, row), head = t.h * a.group + row - i * a.group, token = t.first + i;
    const long long to = ((long long)chunk * a.n_tokens + token) * a.heads + head;
    const float inverse = inverse_of(total) * up;
    if (!whole && h == 0) {
        a.part_ml[to * 2] = m;
        a.part_ml[to * 2 + 1] = total;
    }
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int column = 32 * d + 8 * e + 4 * h;
            const fv4 sum = fv4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
            if (!whole)
                *reinterpret_cast<fv4 *>(a.part + to * DIM + column) = sum * up;
            else
                store_row4<KIND>(a, token, head, column, sum, inverse);
        }
}

// Joins the chunks of a row, its columns by four to a lane; sums in a fixed order.  Few rows (EACH false): a workgroup to a row, the chunks
// in turn over what is left of its lanes.  Many (EACH): a row to as many lanes as it has columns by four, so that a row does not cost a
// workgroup's start, 1.1 ns (4 prompts of 3000 tokens, 8 heads of 64, two chunks, attention and join: 178 us with a workgroup to a row, 83
// so).  What bounds it: latency (7 us of a decode step's 100), bytes of many rows.
template <int KIND, int DIM, bool EACH>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a)
{
    constexpr int C4 = DIM / 4, SETS = 256 / C4;
    constexpr float kNone = -__builtin_huge_valf();
    const unsigned wg = blockIdx.y * gridDim.x + blockIdx.x, combos = (unsigned)(a.requests * a.kv_heads), rest = wg / combos;
    const int set = threadIdx.x / C4, column = (threadIdx.x - set * C4) * 4;
    const int per_tile = EACH ? (a.tile_rows + SETS - 1) / SETS : a.tile_rows;   // workgroups
    const int tile = (int)(rest / (unsigned)per_tile), in_tile = ((int)rest - tile * per_tile) * (EACH ? SETS : 1) + (EACH ? set : 0);
    if (tile >= a.row_tiles) return;
    const RowTile t = row_tile(a, (int)(wg - rest * combos), tile, a.tile_rows);
    const int row = t.row0 + in_tile;
    if (row >= t.rows) return;
    const int i = query_of(a, row), head = t.h * a.group + row - i * a.group, token = t.first + i;
    const int chunks = t.hi > t.lo ? min((t.hi - t.lo + a.chunk - 1) / a.chunk, a.chunks) : 0;
    if (chunks <= 1) return;   // y is written
    const long long at = (long long)token * a.heads + head, per_chunk = (long long)a.n_tokens * a.heads;
    float top = kNone;
    if constexpr (EACH) {
        if (set >= SETS || in_tile >= a.tile_rows) return;
        for (int c = 0; c < chunks; ++c) top = fmaxf(top, a.part_ml[(c * per_chunk + at) * 2]);
    } else {   // every wave finds the maximum for itself, a chunk to a lane
        for (int c = threadIdx.x & 63; c < chunks; c += 64) top = fmaxf(top, a.part_ml[(c * per_chunk + at) * 2]);
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    }
    const float base = top == kNone ? 0.0f : top;
    fv4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    float total = 0.0f;
    if (set < SETS) {
#pragma unroll 4
        for (int c = EACH ? 0 : set; c < chunks; c += EACH ? 1 : SETS) {
            const float *ml = a.part_ml + (c * per_chunk + at) * 2;
            const float f = __builtin_amdgcn_exp2f(ml[0] - base);
            total += ml[1] * f;
            sum += *reinterpret_cast<const fv4 *>(a.part + (c * per_chunk + at) * DIM + column) * f;
        }
    }
    if constexpr (!EACH) {
        __shared__ fv4 sums[SETS][C4];
        __shared__ float totals[SETS];
        if (set < SETS) {
            sums[set][column / 4] = sum;
            if (column == 0) totals[set] = total;
        }
        __syncthreads();
        if (set != 0) return;
        for (int k = 1; k < SETS; ++k) {
            sum += sums[k][column / 4];
            total += totals[k];
        }
    }
    store_row4<KIND>(a, token, head, column, sum, inverse_of(total));
}

}  // namespace lffn
