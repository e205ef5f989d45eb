// Attention of single tokens over the 4-bit cache.
//
//   x_j  = sum_g a_jg (q_g . c_jg)                        seven times the score, groups of 64 channels
//   w_j  = the exponential of x_j against the row's maximum (steps 1-5 of the softmax)
//   u_jg = (w_j a'_jg + 64) >> 7,   o_d = floor(2^54 / sum w_j) * sum_j u_jg c'_jd >> 39
//
// Bound by the bytes of the cache (head_dim / 2 + 1 or 2 per key, twice).  The exponentials need the row's maximum
// before the first of them, so there are two phases, keys and then values, with the scores kept
// between them: as 16-bit differences from the largest score of their 64-key tile and column, saturated (a score
// that far below the maximum has weight 0 either way).
//
// Columns are the queries that share a kv head: e = token * group + head of the group, 16 of them to the narrow
// side of v_mfma_i32_16x16x64_i8.  Keys go by tiles of 64, in blocks of 16 that never cross a page.  Scores are
// transposed, keys x columns: lane (column l % 16, p = l / 16) gets rows 4 p + r of each of a tile's four products, which
// read their keys in the order kappa(s, 4 p + r) = 16 p + 4 s + r, so that its 16 scores are the keys
// 16 p .. 16 p + 15 of the tile, one block, and its 16 weights the right operand of the second product
// without leaving the lane.  The values' layout in the cache gives the left operand the same way: 16 tokens of a
// channel pair are one 16-byte load.
//
// Codes go into the products as 16 c, the nibble in the byte's upper half: no sign extension; the factor 16 leaves
// with the score's shift and, of the values' sums, by a division without remainder.
#pragma once

#include "block.h"

namespace iptq {

constexpr int kTile = 64;             // keys
constexpr int kSplitWaves = 4;        // wavefronts of a workgroup where the keys are split over workgroups

struct CacheAttentionArgs {
    const int8_t *q;
    int8_t *out;
    int64_t q_stride, out_stride;
    const int32_t *pages, *lengths;
    int32_t max_pages, q_tokens, group, columns;          // columns = group * q_tokens
    DivDev by_group, by_kv_heads, by_chunks, by_splits;   // column -> token; workgroup -> kv head, columns, split, sequence
    int32_t split_keys, splits;                           // keys of a workgroup (a multiple of 256), workgroups a sequence
    // between the phases: in LDS where one workgroup has all keys of a sequence, else here
    int16_t *deltas;                                      // [sequence, kv head][tile, p][column][16]
    int32_t *refs;                                        // [sequence, kv head][tile][column]
    int32_t *tops;                                        // [sequence, kv head][split][column]
    int32_t *partial;                                     // [sequence, kv head][split][column][head_dim]
    uint32_t *sums;                                       // [sequence, kv head][split][column]
    CacheDev C;
    AttentionDev P;
};

typedef i32x4 __attribute__((aligned(1))) i32x4_any;

IPTQ_DEV i32x4 upper_nibbles(u32x2_t v)               // 16 codes: the even channels of 8, the odd ones, of the next 8
{
    return (i32x4){(int32_t)(v.x << 4 & 0xf0f0f0f0u), (int32_t)(v.x & 0xf0f0f0f0u), (int32_t)(v.y << 4 & 0xf0f0f0f0u),
                   (int32_t)(v.y & 0xf0f0f0f0u)};
}
IPTQ_DEV i32x4 in_nibble_order(i32x4 v)               // 16 channels of a query in that order
{
    return (i32x4){(int32_t)__builtin_amdgcn_perm((uint32_t)v.y, (uint32_t)v.x, 0x06040200u),
                   (int32_t)__builtin_amdgcn_perm((uint32_t)v.y, (uint32_t)v.x, 0x07050301u),
                   (int32_t)__builtin_amdgcn_perm((uint32_t)v.w, (uint32_t)v.z, 0x06040200u),
                   (int32_t)__builtin_amdgcn_perm((uint32_t)v.w, (uint32_t)v.z, 0x07050301u)};
}
IPTQ_DEV int32_t byte_of(const u32x4 *v, int i) { return (int32_t)(v[i >> 4][i >> 2 & 3] >> (8 * (i & 3)) & 255u); }

// PHASES 3: both, scores in LDS; 1: keys only; 2: values only.
// CT: column tiles of a workgroup.
template <int D, int VARIANT, int CT, int PHASES>
struct CacheAttention {
    static constexpr int G = (D + kGroup - 1) / kGroup, PAIRS = D / 2, BLOCKS = D / 32;    // blocks of 16 channel pairs
    static constexpr int ACC = BLOCKS * 2 * 4 * 64;       // sums of one column tile

    struct Keys { u32x2_t codes[4][G]; u32x4 steps[G]; int32_t page; };
    struct Values { u32x4 codes[BLOCKS]; u32x4 steps[G]; };

    const CacheAttentionArgs &A;
    const int lane, col, p;
    uint32_t kvh, seq, e0;
    int32_t length, from, to;                             // keys [from, to) of the workgroup
    const int32_t *table;
    i32x4 q[CT][G];
    int32_t limit[CT], least;                             // keys that a column sees, that all of them see
    uint32_t e[CT];

    IPTQ_DEV CacheAttention(const CacheAttentionArgs &a, uint32_t kvh_, uint32_t seq_, uint32_t chunk, uint32_t split)
        : A(a), lane(threadIdx.x & 63), col(lane & 15), p(lane >> 4), kvh(kvh_), seq(seq_), e0(chunk * 16 * CT)
    {
        length = min(max(A.lengths[seq], 0), A.max_pages << A.C.page_log);
        from = (int32_t)split * A.split_keys;
        to = min(length, from + A.split_keys);
        table = A.pages + (int64_t)seq * A.max_pages;
        least = A.P.causal ? length - (A.q_tokens - 1) : length;
    }
    IPTQ_DEV int64_t q_row(uint32_t token) const { return (int64_t)seq * A.q_tokens + token; }
    IPTQ_DEV void load_queries()
    {
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            e[c] = min(e0 + 16 * c + col, (uint32_t)A.columns - 1);       // columns past the last repeat it
            const uint32_t token = div_by(e[c], A.by_group), head = kvh * (uint32_t)A.group + (e[c] - token * (uint32_t)A.group);
            limit[c] = A.P.causal ? length - (A.q_tokens - 1 - (int32_t)token) : length;
            const int8_t *src = A.q + q_row(token) * A.q_stride + head * D + 16 * p;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                q[c][g] = (i32x4){0, 0, 0, 0};
                if (kGroup * g + 16 * p < D) q[c][g] = in_nibble_order(*reinterpret_cast<const i32x4_any *>(src + kGroup * g));
            }
        }
    }
    IPTQ_DEV int32_t page_of(int32_t key) const { return page_of_key(table, A.C.page_log, A.C.n_pages, key, length); }

    // Keys [at, at + 64): a page that is not there reads the cache's first one, and is masked.
    IPTQ_DEV Keys load_keys(int32_t at) const
    {
        Keys k;
        const CacheDev &C = A.C;
        const int32_t mine = at + 16 * p, theirs = at + 16 * (col >> 2);   // the block of the lane's scores; of the keys it loads
        const int32_t key_page = page_of(theirs);
        k.page = page_of(mine);
        const int64_t key_row = ((int64_t)max(key_page, 0) * C.kv_heads + kvh) * C.page_tokens + (theirs & (C.page_tokens - 1)) + (col & 3);
        const int64_t step_row = ((int64_t)max(k.page, 0) * C.kv_heads + kvh) * C.page_tokens + (mine & (C.page_tokens - 1));
        const uint8_t *src = C.k_codes + key_row * PAIRS + 8 * p;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                k.codes[s][g] = (u32x2_t){0, 0};
                if (kGroup * g + 16 * p < D) k.codes[s][g] = *reinterpret_cast<const u32x2_t *>(src + 4 * s * PAIRS + kGroup / 2 * g);
            }
#pragma unroll
        for (int g = 0; g < G; ++g) k.steps[g] = *reinterpret_cast<const u32x4 *>(C.k_steps + step_row * G + 16 * g);
        return k;
    }
    IPTQ_DEV Values load_values(int32_t at) const
    {
        Values v;
        const CacheDev &C = A.C;
        const int32_t mine = at + 16 * p, pos = mine & (C.page_tokens - 1);
        const int64_t head_at = (int64_t)max(page_of(mine), 0) * C.kv_heads + kvh;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
            v.codes[b] = *reinterpret_cast<const u32x4 *>(C.v_codes + (head_at * PAIRS + 16 * b + col) * C.page_tokens + pos);
#pragma unroll
        for (int g = 0; g < G; ++g) v.steps[g] = *reinterpret_cast<const u32x4 *>(C.v_steps + (head_at * C.page_tokens + pos) * G + 16 * g);
        return v;
    }
    // Scores of a tile -> 16-bit differences from the tile's largest of the column (packed pairs), and that largest.
    IPTQ_DEV void score(const Keys &k, int32_t at, int c, uint32_t (&d)[8], int32_t *ref) const
    {
        int32_t x[16];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const i32x4 y = __builtin_amdgcn_mfma_i32_16x16x64_i8(upper_nibbles(k.codes[s][g]), q[c][g], (i32x4){0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int32_t t = __mul24(byte_of(k.steps, (4 * s + r) * G + g), y[r]);
                    x[4 * s + r] = g ? x[4 * s + r] + t : t;
                }
            }
        }
        // scores are 16 times their value: a shift of four more
        const int32_t shift = A.P.shift + 4, rounding = A.P.shift > 0 ? 1 << (shift - 1) : 0;
        const int32_t seen = k.page >= 0 ? limit[c] - (at + 16 * p) : 0;      // of the lane's 16 keys
        const bool whole = __all(seen >= 16);
        int32_t top = kI32Min;
        if (whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(top, x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) top = i < seen ? max(top, x[i]) : top;
        }
        top = max(top, __shfl_xor(top, 16));
        top = max(top, __shfl_xor(top, 32));
        *ref = top == kI32Min ? kI32Min : (top + rounding) >> shift;
        const int32_t base = top == kI32Min ? 0 : rounding - (*ref << shift);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = (x[i] + base) >> shift;
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = i < seen ? x[i] : -32768;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pk_i16(x[2 * i], x[2 * i + 1]));
    }
    // One tile's share of the weighted values of a column tile.
    IPTQ_DEV void accumulate(const Values &v, const uint32_t (&d)[8], int32_t ref, int32_t top, i32x4 (&acc)[BLOCKS][2][2], uint32_t *sum) const
    {
        const short off = (short)(ref == kI32Min ? -32768 : max(ref - top, -32768));
        const i16x2 least_d = {(short)-A.P.d_clamp, (short)-A.P.d_clamp}, offs = {off, off};
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const i16x2 t = __builtin_elementwise_max(__builtin_elementwise_add_sat(__builtin_bit_cast(i16x2, d[i]), offs), least_d);
            w[i] = weights_of_pair<VARIANT>(t, A.P);
            *sum = __builtin_amdgcn_udot2(__builtin_bit_cast(u16x2_t, w[i]), (u16x2_t){1, 1}, *sum, false);
        }
        i32x4 hi[G], lo[G];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t u[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t ww = w[2 * i + j];
                    const uint32_t a = __umul24(ww & 0xffff, (uint32_t)byte_of(v.steps, (4 * i + 2 * j) * G + g)) + 64;
                    const uint32_t b = __umul24(ww >> 16, (uint32_t)byte_of(v.steps, (4 * i + 2 * j + 1) * G + g)) + 64;
                    u[j] = a >> 7 | b >> 7 << 16;
                }
                uint32_t h, l;
                split_weights(u[0], u[1], &h, &l);
                hi[g][i] = (int32_t)h;
                lo[g][i] = (int32_t)l;
            }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const int g = 32 * b / kGroup;
            const i32x4 even = __builtin_bit_cast(i32x4, v.codes[b] << 4 & 0xf0f0f0f0u), odd = __builtin_bit_cast(i32x4, v.codes[b] & 0xf0f0f0f0u);
            acc[b][0][0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(even, hi[g], acc[b][0][0], 0, 0, 0);
            acc[b][0][1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(even, lo[g], acc[b][0][1], 0, 0, 0);
            acc[b][1][0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(odd, hi[g], acc[b][1][0], 0, 0, 0);
            acc[b][1][1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(odd, lo[g], acc[b][1][1], 0, 0, 0);
        }
    }
};

// 8 sums of a channel pair block -> 8 output bytes
IPTQ_DEV void store_means(int8_t *out, uint64_t f, const int64_t (&acc)[8], const DyadicDev &post)
{
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)(mean_byte(f, acc[i], 39, post) & 255) << (8 * (i & 3));
    typedef u32x2_t __attribute__((aligned(1))) u32x2_any;
    *reinterpret_cast<u32x2_any *>(out) = (u32x2_t){w[0], w[1]};
}

// LDS: [tops 16 CT][sums 16 CT] then the sums [CT][ACC], and (PHASES 3) deltas [tiles * 4][16 CT][16] and
// refs [tiles][16 CT].
template <int D, int VARIANT, int CT, int PHASES>
IPTQ_DEV void cache_attention_body(const CacheAttentionArgs &A, uint32_t kvh, uint32_t seq, uint32_t chunk, uint32_t split)
{
    typedef CacheAttention<D, VARIANT, CT, PHASES> T;
    extern __shared__ __attribute__((aligned(16))) int32_t lds[];
    int32_t *lds_top = lds, *lds_acc = lds + 32 * CT;
    uint32_t *lds_sum = reinterpret_cast<uint32_t *>(lds + 16 * CT);
    T t(A, kvh, seq, chunk, split);
    const int waves = blockDim.x >> 6, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = t.lane, col = t.col, p = t.p;
    if (PHASES != 3 && t.from >= t.to) return;            // no key in this split
    t.load_queries();
    const int64_t pair = (int64_t)seq * A.C.kv_heads + kvh;
    const int32_t tiles = (A.split_keys * A.splits) / kTile;               // of a sequence's share of the workspace
    const int columns = PHASES == 3 ? 16 * CT : A.columns;
    int16_t *deltas = PHASES == 3 ? reinterpret_cast<int16_t *>(lds_acc + CT * T::ACC) : A.deltas + pair * tiles * 4 * columns * 16;
    int32_t *refs = PHASES == 3 ? lds_acc + CT * T::ACC + tiles * 4 * 16 * CT * 8 : A.refs + pair * tiles * columns;
    const int e0 = PHASES == 3 ? 0 : (int)t.e0;
    bool mine[CT];                                        // whether the column is one of the workspace's
#pragma unroll
    for (int c = 0; c < CT; ++c) mine[c] = PHASES == 3 || e0 + 16 * c + col < columns;

    const int32_t first = t.from + kTile * wave, step = kTile * waves;
    int32_t top[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) top[c] = kI32Min;
    if (threadIdx.x < 16 * CT) lds_top[threadIdx.x] = kI32Min;
    if (PHASES & 2)
        for (int i = threadIdx.x; i < 16 * CT + CT * T::ACC; i += blockDim.x) lds[16 * CT + i] = 0;       // sums
    __syncthreads();
    if (PHASES & 1) {
        if (first < t.to) {
            typename T::Keys now = t.load_keys(first);
            for (int32_t at = first; at < t.to; at += step) {
                const typename T::Keys next = t.load_keys(min(at + step, t.to - 1) & ~(kTile - 1));
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    uint32_t d[8];
                    int32_t ref;
                    t.score(now, at, c, d, &ref);
                    top[c] = max(top[c], ref);
                    const int32_t tile = at / kTile;
                    if (mine[c]) {
                        u32x4 *o = reinterpret_cast<u32x4 *>(deltas + ((int64_t)(tile * 4 + p) * columns + e0 + 16 * c + col) * 16);
                        o[0] = (u32x4){d[0], d[1], d[2], d[3]};
                        o[1] = (u32x4){d[4], d[5], d[6], d[7]};
                        if (p == 0) refs[tile * columns + e0 + 16 * c + col] = ref;
                    }
                }
                now = next;
            }
#pragma unroll
            for (int c = 0; c < CT; ++c)
                if (p == 0) atomicMax(lds_top + 16 * c + col, top[c]);
        }
        __syncthreads();
        if (PHASES == 1) {
            const int i = threadIdx.x;
            if (i < 16 * CT && e0 + i < columns) A.tops[(pair * A.splits + split) * columns + e0 + i] = lds_top[i];
            return;
        }
    }
    if (PHASES == 2) {                                    // the largest score of all splits that have keys
        const int32_t live = (t.length + A.split_keys - 1) / A.split_keys;
        for (int i = threadIdx.x; i < live * 16 * CT; i += blockDim.x) {
            const int c = i % (16 * CT);
            if (e0 + c < columns) atomicMax(lds_top + c, A.tops[(pair * A.splits + i / (16 * CT)) * columns + e0 + c]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) top[c] = lds_top[16 * c + col];

    if (first < t.to) {
        i32x4 acc[CT][T::BLOCKS][2][2];
        uint32_t sum[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            sum[c] = 0;
#pragma unroll
            for (int b = 0; b < T::BLOCKS; ++b)
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[c][b][n >> 1][n & 1] = (i32x4){0, 0, 0, 0};
        }
        typename T::Values now = t.load_values(first);
        for (int32_t at = first; at < t.to; at += step) {
            const typename T::Values next = t.load_values(min(at + step, t.to - 1) & ~(kTile - 1));
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const int32_t tile = at / kTile, column = mine[c] ? e0 + 16 * c + col : columns - 1;
                const u32x4 *o = reinterpret_cast<const u32x4 *>(deltas + ((int64_t)(tile * 4 + p) * columns + column) * 16);
                const u32x4 a = o[0], b = o[1];
                const uint32_t d[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                t.accumulate(now, d, refs[tile * columns + column], top[c], acc[c], &sum[c]);
            }
            now = next;
        }
        // the wavefronts' sums: whole numbers, so the order in which they are added does not matter
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            sum[c] += (uint32_t)__shfl_xor((int32_t)sum[c], 16);
            sum[c] += (uint32_t)__shfl_xor((int32_t)sum[c], 32);
            if (p == 0) atomicAdd(lds_sum + 16 * c + col, sum[c]);
#pragma unroll
            for (int b = 0; b < T::BLOCKS; ++b)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        atomicAdd(lds_acc + c * T::ACC + ((b * 2 + n) * 4 + r) * 64 + lane, acc[c][b][n][0][r] * 16 + (acc[c][b][n][1][r] >> 4));
        }
    }
    __syncthreads();
    // a thread's block of 16 channel pairs and lane: rows 4 p + r are the pairs 16 b + 4 p + r, eight channels in a row
    for (int u = threadIdx.x; u < CT * T::BLOCKS * 64; u += blockDim.x) {
        const int c = u / (T::BLOCKS * 64), b = (u >> 6) % T::BLOCKS, l = u & 63;
        const uint32_t column = t.e0 + 16 * c + (l & 15);
        if (column >= (uint32_t)A.columns) continue;
        int64_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lds_acc[c * T::ACC + ((b * 2 + (i & 1)) * 4 + (i >> 1)) * 64 + l];
        const uint32_t s = lds_sum[16 * c + (l & 15)];
        const int channel = 32 * b + 8 * (l >> 4);
        if (PHASES == 3) {
            const uint32_t token = div_by(column, A.by_group), head = kvh * (uint32_t)A.group + (column - token * (uint32_t)A.group);
            store_means(A.out + t.q_row(token) * A.out_stride + head * D + channel, floor_div_u64((uint64_t)1 << 54, s), v, A.P.post);
        } else {
            const int64_t at = (pair * A.splits + split) * A.columns + column;
            i32x4 *o = reinterpret_cast<i32x4 *>(A.partial + at * D + channel);
            o[0] = (i32x4){(int32_t)v[0], (int32_t)v[1], (int32_t)v[2], (int32_t)v[3]};
            o[1] = (i32x4){(int32_t)v[4], (int32_t)v[5], (int32_t)v[6], (int32_t)v[7]};
            if (channel == 0) A.sums[at] = s;
        }
    }
}

template <int D, int VARIANT, int CT, int PHASES>
__global__ __launch_bounds__(PHASES == 3 ? 512 : 256) void attention_cache_i4_kernel(const CacheAttentionArgs A)
{
    const uint32_t r1 = div_by(blockIdx.x, A.by_kv_heads), kvh = blockIdx.x - r1 * A.by_kv_heads.d;
    const uint32_t r2 = div_by(r1, A.by_chunks), chunk = r1 - r2 * A.by_chunks.d;
    const uint32_t seq = div_by(r2, A.by_splits), split = r2 - seq * A.by_splits.d;
    cache_attention_body<D, VARIANT, CT, PHASES>(A, kvh, seq, chunk, split);
}

hipError_t attention_cache_i4_launch_32(const CacheAttentionArgs &a, int ct, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);
hipError_t attention_cache_i4_launch_64(const CacheAttentionArgs &a, int ct, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);
hipError_t attention_cache_i4_launch_96(const CacheAttentionArgs &a, int ct, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);
hipError_t attention_cache_i4_launch_128(const CacheAttentionArgs &a, int ct, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);

// One file per head dimension instantiates its kernels.
template <int D, int VARIANT>
hipError_t attention_cache_i4_launch_of(const CacheAttentionArgs &a, int ct, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream)
{
    auto kernel = phases == 3 ? (ct == 1 ? attention_cache_i4_kernel<D, VARIANT, 1, 3> : attention_cache_i4_kernel<D, VARIANT, 2, 3>)
                  : phases == 2 ? (ct == 1 ? attention_cache_i4_kernel<D, VARIANT, 1, 2> : attention_cache_i4_kernel<D, VARIANT, 2, 2>)
                  : ct == 1 ? attention_cache_i4_kernel<D, 0, 1, 1> : attention_cache_i4_kernel<D, 0, 2, 1>;
    launch_kernel(kernel, dim3(grid), dim3(block), lds, stream, a);
    return take_launch_status();
}
#define IPTQ_ATTENTION_CACHE_I4_OF(D)                                                                                         \
    hipError_t iptq::attention_cache_i4_launch_##D(const CacheAttentionArgs &a, int ct, int phases, uint32_t grid, uint32_t block, \
                                                   size_t lds, hipStream_t stream)                                            \
    {                                                                                                                         \
        return (a.P.variant == 0   ? attention_cache_i4_launch_of<D, 0>                                                       \
                : a.P.variant == 1 ? attention_cache_i4_launch_of<D, 1>                                                       \
                                   : attention_cache_i4_launch_of<D, 2>)(a, ct, phases, grid, block, lds, stream);            \
    }

}  // namespace iptq
