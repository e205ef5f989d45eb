// Attention of single tokens over the 4-bit cache.
//
//   x_j  = sum_g a_jg (q_g . c_jg)                        seven times the score, groups of 64 channels
//   w_j  = the exponential of x_j against the row's maximum (steps 1-5 of the softmax)
//   u_jg = (w_j a'_jg + 64) >> 7,   o_d = floor(2^54 / sum w_j) * sum_j u_jg c'_jd >> 39
//
// The bytes of the cache (head_dim / 2 + 1 or 2 per key, twice) bound it for one head to a kv head.  The exponentials need the row's maximum
// before the first of them, so there are two phases, keys and then values, with the scores kept
// between them: as 16-bit differences from the largest score of their 64-key tile and column, saturated (a score
// that far below the maximum has weight 0 either way).  Their 2 bytes per key and column, written and read, are as many as the cache's
// from 32 columns on, and the values' phase has 310 vector instructions per 64 keys and 16 columns (210 per 8).
// Measured: 64 sequences of 200 to 8192 tokens, 32 heads on 8 of 128, 63 us (3.0 TB/s of cache; 28 us keys, 31 values, 5 the sum of
// the splits); two of 131072, 32 columns, 136 us (2.0 TB/s of cache, 4.0 with the scores; 55, 80, 6); one of 700, 7 us with the call.
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

struct CacheAttentionArgs {
    const int8_t *q;
    int8_t *out;
    int64_t q_stride, out_stride;
    const int32_t *pages, *lengths;
    int32_t max_pages, q_tokens, group, columns;          // columns = group * q_tokens
    DivDev by_group, by_kv_heads, by_chunks, by_splits;   // column -> token; workgroup -> kv head, columns, split, sequence
    DivDev by_span, by_columns;                           // span: 64 keys of each wavefront that a sequence's keys are divided over
    int32_t key_waves;                                    // wavefronts of a workgroup, over the keys
    uint32_t all_columns;                                 // of all sequences and kv heads
    int32_t splits, tiles;                                // workgroups over a sequence; tiles of the workspace a sequence
    // between the phases, where one workgroup does not have all keys of a sequence
    int16_t *deltas;                                      // [sequence, kv head][tile, p][2][column][8]
    int32_t *refs;                                        // [sequence, kv head][tile][column]
    int32_t *tops;                                        // [sequence, kv head][split][column]
    int32_t *partial;                                     // [sequence, kv head][split][column][head_dim]
    uint32_t *sums;                                       // [sequence, kv head][split][column]
    CacheDev C;
    AttentionDev P;
};

// Keys of a wavefront: a sequence's keys are divided evenly, whatever its length, so that short sequences beside long
// ones leave no workgroup idle and the long ones none behind.
IPTQ_DEV int32_t wave_keys_of(const CacheAttentionArgs &A, int32_t length)
{
    return kTile * (int32_t)div_by((uint32_t)length + A.by_span.d - 1, A.by_span);
}
IPTQ_DEV int32_t length_of(const CacheAttentionArgs &A, uint32_t seq)
{
    return min(max(A.lengths[seq], 0), A.max_pages << A.C.page_log);
}

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

// PHASES 3: both, a tile a wavefront and its scores in registers; 1: keys only; 2: values only.
// HALVES 2: up to eight queries share a kv head.  The second product's sixteen columns are then the upper halves of
// eight queries' weights and the lower halves of the same: one product in place of two.  The two lanes of a query divide
// the scores and weights of a block's 16 keys, eight each, and hand each other the halves of weights that they do not multiply with.
// (One of 1000 tokens, 4 queries, 7.9 us, 64 of 4000 67, one of 131072 45; with all the keys in both lanes 8.9, 72 and 48, with a
// product for either half a few per cent more.)
// HALVES 1: sixteen queries, one product for either half.
template <int D, int VARIANT, int HALVES, int PHASES>
struct CacheAttention {
    static constexpr int G = (D + kGroup - 1) / kGroup, PAIRS = D / 2, BLOCKS = D / 32;    // blocks of 16 channel pairs
    static constexpr int QUERIES = 16 / HALVES, PRODUCTS = 3 - HALVES;
    static constexpr int ACC = BLOCKS * 2 * 4 * 64;       // sums of 16 columns
    static constexpr int OWN = 16 / HALVES;               // of a block's keys, the lane's

    // A tile's codes as the wavefront loads them, 16 bytes a lane in the order of the memory (a quarter of a
    // wavefront-wide load then meets whole lines; loaded in the products' order, every lane of a quad had a line of its own
    // and the L1 took four times the cycles).  They change places in LDS, in a buffer of the wavefront's own.
    struct Keys { u32x4 codes[BLOCKS]; u32x4 steps[G]; int32_t page; };
    struct Values { u32x4 codes[BLOCKS]; u32x4 steps[G]; };
    static constexpr int kValueBlock = 4 * 288;           // 16 pairs: four blocks of 256 bytes, 32 apart for the banks' sake
    static constexpr int STAGE = BLOCKS * kValueBlock > kTile * PAIRS + 256 ? BLOCKS * kValueBlock : kTile * PAIRS + 256;
    // Where a 16-key block of either starts in the buffer: shifted against each other so that a read's lanes meet all banks.
    static IPTQ_DEV int keys_at(int block)
    {
        return block * 16 * PAIRS + (BLOCKS >= 3 ? 16 * block : BLOCKS == 2 ? 16 * (block & 1) + 128 * (block >> 1) : 64 * block);
    }

    const CacheAttentionArgs &A;
    const int lane, col, p;
    int8_t *stage;
    uint32_t kvh, seq, e;
    int32_t length, limit;                                // keys of the sequence, keys that the lane's query sees
    int32_t from, to;                                     // the wavefront's keys, at most 1024
    int32_t page_of_block;                                // lane l: page of the wavefront's block l, or -1
    i32x4 q[G];

    // first: the wavefront's number among those that the sequence's keys are divided over
    IPTQ_DEV CacheAttention(const CacheAttentionArgs &a, uint32_t kvh_, uint32_t seq_, uint32_t e0, int32_t first, int8_t *stage_)
        : A(a), lane(threadIdx.x & 63), col(lane & 15), p(lane >> 4), stage(stage_), kvh(kvh_), seq(seq_)
    {
        length = length_of(A, seq);
        const int32_t keys = wave_keys_of(A, length);
        from = first * keys;
        to = min(length, from + keys);
        const int32_t key = from + 16 * lane;
        page_of_block = page_of_key(A.pages + (int64_t)seq * A.max_pages, A.C.page_log, A.C.n_pages, key, to);
        e = min(e0 + (col & (QUERIES - 1)), (uint32_t)A.columns - 1);     // columns past the last repeat it
    }
    IPTQ_DEV uint32_t token() const { return div_by(e, A.by_group); }
    IPTQ_DEV int64_t q_row(uint32_t token) const { return (int64_t)seq * A.q_tokens + token; }
    IPTQ_DEV void load_queries()
    {
        const uint32_t t = token(), head = kvh * (uint32_t)A.group + (e - t * (uint32_t)A.group);
        limit = A.P.causal ? length - (A.q_tokens - 1 - (int32_t)t) : length;
        const int8_t *src = A.q + q_row(t) * A.q_stride + head * D + 16 * p;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            q[g] = (i32x4){0, 0, 0, 0};
            if (kGroup * g + 16 * p < D) q[g] = in_nibble_order(*reinterpret_cast<const i32x4_any *>(src + kGroup * g));
        }
    }
    // Keys [at, at + 64): a page that is not there reads the cache's first one, and is masked.
    IPTQ_DEV Keys load_keys(int32_t at) const
    {
        Keys k;
        const CacheDev &C = A.C;
        const int first = (at - from) >> 4, mask = C.page_tokens - 1;
        if (C.page_log >= 6) {                            // a tile lies in one page: one address (64 of 1000 tokens 20.3 us, block by block 21.8)
            k.page = __builtin_amdgcn_readlane(page_of_block, first);
            const int64_t row = ((int64_t)max(k.page, 0) * C.kv_heads + kvh) * C.page_tokens + (at & mask);
            const uint8_t *codes = C.k_codes + row * PAIRS + 16 * lane, *steps = C.k_steps + (row + 16 * p) * G;
#pragma unroll
            for (int i = 0; i < BLOCKS; ++i) k.codes[i] = *reinterpret_cast<const u32x4 *>(codes + 1024 * i);
#pragma unroll
            for (int g = 0; g < G; ++g) k.steps[g] = *reinterpret_cast<const u32x4 *>(steps + 16 * g);
            return k;
        }
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {                // (a key's row is BLOCKS chunks of 16 bytes)
            const int chunk = 64 * i + lane, block = chunk / (16 * BLOCKS), in_block = chunk - block * 16 * BLOCKS;
            const int32_t page = max(__shfl(page_of_block, first + block), 0);
            const int64_t row = ((int64_t)page * C.kv_heads + kvh) * C.page_tokens + ((at + 16 * block) & mask);
            k.codes[i] = *reinterpret_cast<const u32x4 *>(C.k_codes + row * PAIRS + 16 * in_block);
        }
        k.page = __shfl(page_of_block, first + p);
        const int64_t step_row = ((int64_t)max(k.page, 0) * C.kv_heads + kvh) * C.page_tokens + ((at + 16 * p) & mask);
#pragma unroll
        for (int g = 0; g < G; ++g) k.steps[g] = *reinterpret_cast<const u32x4 *>(C.k_steps + step_row * G + 16 * g);
        return k;
    }
    IPTQ_DEV void stage_keys(const Keys &k) const
    {
#pragma unroll
        for (int i = 0; i < BLOCKS; ++i) {
            const int chunk = 64 * i + lane, block = chunk / (16 * BLOCKS), in_block = chunk - block * 16 * BLOCKS;
            *reinterpret_cast<u32x4 *>(stage + keys_at(block) + 16 * in_block) = k.codes[i];
        }
        wave_lds_fence();
    }
    // The block and the channel pair (of 16) whose tokens the lane loads: a page's tokens of a pair lie side by side, so
    // the lanes of a quad take blocks of the same page and then further pairs.
    IPTQ_DEV int value_block(int lane) const { return A.C.page_log >= 6 ? lane & 3 : A.C.page_log == 5 ? (lane & 1) | lane >> 5 << 1 : lane >> 4; }
    IPTQ_DEV int value_pair(int lane) const { return A.C.page_log >= 6 ? lane >> 2 : A.C.page_log == 5 ? lane >> 1 & 15 : lane & 15; }
    IPTQ_DEV Values load_values(int32_t at) const
    {
        Values v;
        const CacheDev &C = A.C;
        int l = lane;
        asm volatile("" : "+v"(l));                       // (made again each time: kept, it may spill)
        const int first = (at - from) >> 4, mask = C.page_tokens - 1, block = value_block(l);
        if (C.page_log >= 6) {
            const int64_t head = (int64_t)max(__builtin_amdgcn_readlane(page_of_block, first), 0) * C.kv_heads + kvh;
            const uint8_t *codes = C.v_codes + head * PAIRS * C.page_tokens + (at & mask) + (value_pair(l) * C.page_tokens + 16 * block);
            const uint8_t *steps = C.v_steps + (head * C.page_tokens + (at & mask) + 16 * p) * G;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) v.codes[b] = *reinterpret_cast<const u32x4 *>(codes + 16 * b * C.page_tokens);
#pragma unroll
            for (int g = 0; g < G; ++g) v.steps[g] = *reinterpret_cast<const u32x4 *>(steps + 16 * g);
            return v;
        }
        const int64_t head_at = (int64_t)max(__shfl(page_of_block, first + block), 0) * C.kv_heads + kvh;
        const uint8_t *src = C.v_codes + (head_at * PAIRS + value_pair(l)) * C.page_tokens + ((at + 16 * block) & mask);
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) v.codes[b] = *reinterpret_cast<const u32x4 *>(src + (int64_t)(16 * b) * C.page_tokens);
        const int64_t step_row = ((int64_t)max(__shfl(page_of_block, first + p), 0) * C.kv_heads + kvh) * C.page_tokens + ((at + 16 * p) & mask);
#pragma unroll
        for (int g = 0; g < G; ++g) v.steps[g] = *reinterpret_cast<const u32x4 *>(C.v_steps + step_row * G + 16 * g);
        return v;
    }
    IPTQ_DEV void stage_values(const Values &v) const
    {
        int l = lane;
        asm volatile("" : "+v"(l));
        const int at = value_block(l) * 288 + value_pair(l) * 16;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) *reinterpret_cast<u32x4 *>(stage + b * kValueBlock + at) = v.codes[b];
        wave_lds_fence();
    }
    IPTQ_DEV bool second() const { return HALVES == 2 && col >= 8; }      // the lane's keys are a block's last eight
    // The steps of the lane's own keys, OWN * G bytes.
    struct Steps { u32x4 v[OWN * G > 16 ? 2 : 1]; };
    IPTQ_DEV Steps own_steps(const u32x4 (&steps)[G]) const
    {
        Steps t;
        if (HALVES == 1) {
#pragma unroll
            for (int g = 0; g < G; ++g) t.v[g] = steps[g];
        } else if (G == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) t.v[0][i] = second() ? steps[G - 1][i] : steps[0][i];
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) t.v[0][i] = second() ? steps[0][2 + i] : steps[0][i];
        }
        return t;
    }
    static IPTQ_DEV int32_t other_half(int32_t v) { return __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true); }      // row_ror:8
    // Scores of a tile -> 16-bit differences from the tile's largest of the column (packed pairs), and that largest.
    IPTQ_DEV void score(const Keys &k, int32_t at, uint32_t (&d)[OWN / 2], int32_t *ref) const
    {
        int32_t x[OWN];
        stage_keys(k);
        const Steps steps = own_steps(k.steps);
        const int8_t *src = stage + keys_at(col >> 2) + (col & 3) * PAIRS + 8 * p;
#pragma unroll
        for (int s = 0; s < 4 / HALVES; ++s) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                i32x4 y;
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    // (where the last group is half a one, lanes 32 on take the others' codes, against zeros of the query)
                    const u32x2_t codes = *reinterpret_cast<const u32x2_t *>(src + (kGroup * g + 48 < D ? 0 : p >= 2 ? -16 : 0) + 4 * (s + 2 * h) * PAIRS +
                                                                             kGroup / 2 * g);
                    const i32x4 z = __builtin_amdgcn_mfma_i32_16x16x64_i8(upper_nibbles(codes), q[g], (i32x4){0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) y[r] = h == 0 || second() ? z[r] : y[r];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int32_t t = __mul24(byte_of(steps.v, (4 * s + r) * G + g), y[r]);
                    x[4 * s + r] = g ? x[4 * s + r] + t : t;
                }
            }
        }
        wave_lds_fence();                                 // the buffer may be written again
        // scores are 16 times their value: a shift of four more
        const int32_t shift = A.P.shift + 4, rounding = A.P.shift > 0 ? 1 << (shift - 1) : 0;
        const int32_t seen = k.page >= 0 ? limit - (at + 16 * p + (second() ? 8 : 0)) : 0;       // of the lane's keys
        const bool whole = __all(seen >= OWN);
        int32_t top = kI32Min;
        if (whole) {
#pragma unroll
            for (int i = 0; i < OWN; ++i) top = max(top, x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < OWN; ++i) top = i < seen ? max(top, x[i]) : top;
        }
        if (HALVES == 2) top = max(top, other_half(top));
        top = max(top, __shfl_xor(top, 16));
        top = max(top, __shfl_xor(top, 32));
        *ref = top == kI32Min ? kI32Min : (top + rounding) >> shift;
        const int32_t base = top == kI32Min ? 0 : rounding - (*ref << shift);
#pragma unroll
        for (int i = 0; i < OWN; ++i) x[i] = (x[i] + base) >> shift;
        if (!whole) {
#pragma unroll
            for (int i = 0; i < OWN; ++i) x[i] = i < seen ? x[i] : -32768;
        }
#pragma unroll
        for (int i = 0; i < OWN / 2; ++i) d[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pk_i16(x[2 * i], x[2 * i + 1]));
    }
    // One tile's share of the weighted values.
    IPTQ_DEV void accumulate(const Values &v, const uint32_t (&d)[OWN / 2], int32_t ref, int32_t top, i32x4 (&acc)[BLOCKS][2][PRODUCTS],
                             uint32_t *sum) const
    {
        stage_values(v);
        const short off = (short)(ref == kI32Min ? -32768 : max(ref - top, -32768));
        const i16x2 least = {(short)-A.P.d_clamp, (short)-A.P.d_clamp}, offs = {off, off};
        uint32_t w[OWN / 2];
#pragma unroll
        for (int i = 0; i < OWN / 2; ++i) {
            const i16x2 t = __builtin_elementwise_max(__builtin_elementwise_add_sat(__builtin_bit_cast(i16x2, d[i]), offs), least);
            w[i] = __builtin_bit_cast(uint32_t, t);
        }
#pragma unroll
        for (int i = 0; i < OWN / 8; ++i) weights_of_pairs<VARIANT, 4>(*reinterpret_cast<uint32_t (*)[4]>(w + 4 * i), A.P);
#pragma unroll
        for (int i = 0; i < OWN / 2; ++i) *sum = __builtin_amdgcn_udot2(__builtin_bit_cast(u16x2_t, w[i]), (u16x2_t){1, 1}, *sum, false);
        // u = (w a + 64) >> 7 is the upper part of t = 2 w a + 128, from bit 8 on; with 128 more of u in it, its upper byte
        // is the upper half of u and its lower byte the lower half with the sign turned
        const Steps steps = own_steps(v.steps);
        i32x4 hi[G], lo[G];                               // HALVES 2: hi is the half that the lane multiplies with
        const uint32_t select = second() ? 0x06040200u : 0x07050301u, turn = second() ? 0x80808080u : 0u;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < OWN / 4; ++i) {
                uint32_t u[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t w2 = __builtin_bit_cast(uint32_t, __builtin_bit_cast(u16x2_t, w[2 * i + j]) << (unsigned short)1);
                    const int at0 = (4 * i + 2 * j) * G + g;
                    uint32_t ta = __umul24(w2 & 0xffffu, (uint32_t)byte_of(steps.v, at0)), tb = __umul24(w2 >> 16, (uint32_t)byte_of(steps.v, at0 + G));
                    asm("" : "+v"(ta), "+v"(tb));         // (kept from the addition, the products take their operands' halves and bytes as they lie)
                    ta += 128u + 32768u;
                    tb += 128u + 32768u;
                    u[j] = __builtin_amdgcn_perm(tb, ta, 0x06050201u);
                }
                if (HALVES == 1) {
                    hi[g][i] = (int32_t)__builtin_amdgcn_perm(u[1], u[0], 0x07050301u);
                    lo[g][i] = (int32_t)(__builtin_amdgcn_perm(u[1], u[0], 0x06040200u) ^ 0x80808080u);
                } else {
                    const int32_t mine = (int32_t)(__builtin_amdgcn_perm(u[1], u[0], select) ^ turn);
                    const int32_t given = other_half((int32_t)__builtin_amdgcn_perm(u[1], u[0], select ^ 0x01010101u)) ^ (int32_t)turn;
                    hi[g][i & 1] = second() ? given : mine;
                    hi[g][2 + (i & 1)] = second() ? mine : given;
                }
            }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const int g = 32 * b / kGroup;
            const u32x4 codes = *reinterpret_cast<const u32x4 *>(stage + b * kValueBlock + p * 288 + col * 16);
            const i32x4 even = __builtin_bit_cast(i32x4, codes << 4 & 0xf0f0f0f0u), odd = __builtin_bit_cast(i32x4, codes & 0xf0f0f0f0u);
            acc[b][0][0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(even, hi[g], acc[b][0][0], 0, 0, 0);
            acc[b][1][0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(odd, hi[g], acc[b][1][0], 0, 0, 0);
            if (HALVES == 1) {
                acc[b][0][PRODUCTS - 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(even, lo[g], acc[b][0][PRODUCTS - 1], 0, 0, 0);
                acc[b][1][PRODUCTS - 1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(odd, lo[g], acc[b][1][PRODUCTS - 1], 0, 0, 0);
            }
        }
        wave_lds_fence();                                 // the buffer may be written again
    }
};

// 8 sums of a channel pair block -> 8 output bytes
IPTQ_DEV void store_means(int8_t *out, uint64_t f, const int64_t (&acc)[8], const AttentionDev &P)
{
    const int64_t a[4] = {acc[0], acc[1], acc[2], acc[3]}, b[4] = {acc[4], acc[5], acc[6], acc[7]};
    const uint32_t w[2] = {mean_bytes(f, a, 39, P.post_shift, P.post), mean_bytes(f, b, 39, P.post_shift, P.post)};
    typedef u32x2_t __attribute__((aligned(1))) u32x2_any;
    *reinterpret_cast<u32x2_any *>(out) = (u32x2_t){w[0], w[1]};
}

// A workgroup has up to 16 queries of a split's keys, which its wavefronts divide.  (32 queries of the same keys, two wavefronts side by
// side, took 5 to 9 % longer: the keys come from the L2 the second time.)
// LDS: a staging buffer per wavefront, [tops 16], [sums 16], [ACC].
template <int D, int VARIANT, int HALVES, int PHASES>
IPTQ_DEV void cache_attention_body(const CacheAttentionArgs &A, uint32_t kvh, uint32_t seq, uint32_t chunk, uint32_t split)
{
    typedef CacheAttention<D, VARIANT, HALVES, PHASES> T;
    extern __shared__ __attribute__((aligned(16))) int8_t lds_bytes[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t *lds_top = reinterpret_cast<int32_t *>(lds_bytes + A.key_waves * T::STAGE), *lds_acc = lds_top + 32;
    uint32_t *lds_sum = reinterpret_cast<uint32_t *>(lds_top + 16);
    const int e_wg = (int)chunk * T::QUERIES;                              // the workgroup's first query
    T t(A, kvh, seq, (uint32_t)e_wg, (int32_t)split * A.key_waves + wave, lds_bytes + wave * T::STAGE);
    const int lane = t.lane, col = t.col, p = t.p;
    const int32_t split_keys = wave_keys_of(A, t.length) * A.key_waves;
    if (PHASES != 3 && (int32_t)split * split_keys >= t.length) return;   // no key in this split
    t.load_queries();
    const int64_t pair = (int64_t)seq * A.C.kv_heads + kvh;
    const int32_t tiles = A.tiles;
    const int columns = A.columns, column = e_wg + (col & (T::QUERIES - 1));
    int16_t *deltas = A.deltas + pair * tiles * 4 * columns * 16;
    int32_t *refs = A.refs + pair * tiles * columns;
    const bool mine = column < columns;                                    // the lane writes its column's scores

    // (PHASES 3) the values are on their way while the keys are worked on
    typename T::Values only;
    uint32_t only_d[T::OWN / 2];
    int32_t only_ref = kI32Min;
    int32_t top = kI32Min;
    const int32_t last = (t.to - 1) & ~(kTile - 1);                        // the wavefront's last tile
    if (threadIdx.x < 16) lds_top[threadIdx.x] = kI32Min;
    if (PHASES & 2)
        for (int i = threadIdx.x; i < 16 + T::ACC; i += blockDim.x) lds_top[16 + i] = 0;       // sums
    if (PHASES & 1) {
        if (PHASES == 3 && t.from < t.to) {
            const typename T::Keys keys = t.load_keys(t.from);
            only = t.load_values(t.from);
            t.score(keys, t.from, only_d, &only_ref);
            top = only_ref;
        }
        if (PHASES == 1 && t.from < t.to) {
            auto step = [&](const typename T::Keys &keys, int32_t at) {
                uint32_t d[T::OWN / 2];
                int32_t ref;
                t.score(keys, at, d, &ref);
                top = max(top, ref);
                const int32_t tile = at / kTile;
                if (!mine) return;
                u32x4 *o = reinterpret_cast<u32x4 *>(deltas) + (int64_t)(tile * 4 + p) * 2 * columns + column;
                o[t.second() ? columns : 0] = (u32x4){d[0], d[1], d[2], d[3]};
                if (HALVES == 1) o[columns] = (u32x4){d[T::OWN / 2 - 4], d[T::OWN / 2 - 3], d[T::OWN / 2 - 2], d[T::OWN / 2 - 1]};
                if (p == 0) refs[tile * columns + column] = ref;
            };
            // (two tiles a trip: no copies from the next one's registers)
            typename T::Keys ka = t.load_keys(t.from), kb;
            for (int32_t at = t.from; at < t.to; at += 2 * kTile) {
                kb = t.load_keys(min(at + kTile, last));
                step(ka, at);
                if (at + kTile >= t.to) break;
                ka = t.load_keys(min(at + 2 * kTile, last));
                step(kb, at + kTile);
            }
        }
        __syncthreads();
        if (p == 0 && t.from < t.to) atomicMax(lds_top + col, top);
        __syncthreads();
        if (PHASES == 1) {
            const int i = threadIdx.x;
            if (i < T::QUERIES && e_wg + i < columns) A.tops[(pair * A.splits + split) * columns + e_wg + i] = lds_top[i];
            return;
        }
    } else {
        __syncthreads();
    }
    if (PHASES == 2) {                                    // the largest score of all splits that have keys
        for (int i = threadIdx.x & 15, s = threadIdx.x >> 4; s < A.splits && s * split_keys < t.length; s += blockDim.x >> 4) {
            const int x = e_wg + (i & (T::QUERIES - 1));
            if (x < columns) atomicMax(lds_top + i, A.tops[(pair * A.splits + s) * columns + x]);
        }
        __syncthreads();
    }
    top = lds_top[col];

    if (t.from < t.to) {
        i32x4 acc[T::BLOCKS][2][T::PRODUCTS];
        uint32_t sum = 0;
#pragma unroll
        for (int b = 0; b < T::BLOCKS; ++b)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int h = 0; h < T::PRODUCTS; ++h) acc[b][n][h] = (i32x4){0, 0, 0, 0};
        if (PHASES == 3) {
            t.accumulate(only, only_d, only_ref, top, acc, &sum);
        } else {
            const int from_column = min(column, columns - 1);
            struct Scores { u32x4 v[2 / HALVES]; int32_t ref; };
            auto load_scores = [&](int32_t at) {
                const u32x4 *o = reinterpret_cast<const u32x4 *>(deltas) + (int64_t)(at / kTile * 4 + p) * 2 * columns + from_column;
                Scores x;
                x.v[0] = o[t.second() ? columns : 0];
                if (HALVES == 1) x.v[2 / HALVES - 1] = o[columns];
                x.ref = refs[at / kTile * columns + from_column];
                return x;
            };
            typename T::Values va = t.load_values(t.from), vb;
            Scores sa = load_scores(t.from), sb;
            auto step = [&](const typename T::Values &v, const Scores &x) {
                uint32_t d[T::OWN / 2];
#pragma unroll
                for (int i = 0; i < T::OWN / 2; ++i) d[i] = x.v[i >> 2][i & 3];
                t.accumulate(v, d, x.ref, top, acc, &sum);
            };
            for (int32_t at = t.from; at < t.to; at += 2 * kTile) {
                vb = t.load_values(min(at + kTile, last));
                sb = load_scores(min(at + kTile, last));
                step(va, sa);
                if (at + kTile >= t.to) break;
                va = t.load_values(min(at + 2 * kTile, last));
                sa = load_scores(min(at + 2 * kTile, last));
                step(vb, sb);
            }
        }
        // the wavefronts' sums: whole numbers, so the order in which they are added does not matter
        if (HALVES == 2) sum += (uint32_t)T::other_half((int32_t)sum);
        sum += (uint32_t)__shfl_xor((int32_t)sum, 16);
        sum += (uint32_t)__shfl_xor((int32_t)sum, 32);
        if (p == 0) atomicAdd(lds_sum + col, sum);
        // 16 (256 hi + lo) of either half; HALVES 2: of the half that the lane's column is
        const int up = HALVES == 2 && col >= 8 ? 0 : 8;
#pragma unroll
        for (int b = 0; b < T::BLOCKS; ++b)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    int32_t v = HALVES == 2 ? acc[b][n][0][r] >> 4 << up : acc[b][n][0][r] * 16 + (acc[b][n][T::PRODUCTS - 1][r] >> 4);
                    atomicAdd(lds_acc + ((b * 2 + n) * 4 + r) * 64 + (HALVES == 2 ? lane & ~8 : lane), v);
                }
    }
    __syncthreads();
    // a thread's block of 16 channel pairs and lane: rows 4 p + r are the pairs 16 b + 4 p + r, eight channels in a row
    for (int u = threadIdx.x; u < T::BLOCKS * 64; u += blockDim.x) {
        const int b = u >> 6, l = u & 63, j = l & 15;
        const uint32_t x = (uint32_t)(e_wg + j);
        if (j >= T::QUERIES || x >= (uint32_t)A.columns) continue;
        int64_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lds_acc[((b * 2 + (i & 1)) * 4 + (i >> 1)) * 64 + l];
        const uint32_t s = lds_sum[j];
        const int channel = 32 * b + 8 * (l >> 4);
        if (PHASES == 3) {
            const uint32_t token = div_by(x, A.by_group), head = kvh * (uint32_t)A.group + (x - token * (uint32_t)A.group);
            store_means(A.out + t.q_row(token) * A.out_stride + head * D + channel, floor_div_scaled(1, 54, s), v, A.P);
        } else {
            const int64_t at = (pair * A.splits + split) * A.columns + x;
            i32x4 *o = reinterpret_cast<i32x4 *>(A.partial + at * D + channel);
            o[0] = (i32x4){(int32_t)v[0], (int32_t)v[1], (int32_t)v[2], (int32_t)v[3]};
            o[1] = (i32x4){(int32_t)v[4], (int32_t)v[5], (int32_t)v[6], (int32_t)v[7]};
            if (channel == 0) A.sums[at] = s;
        }
    }
}

template <int D, int VARIANT, int HALVES, int PHASES>
// (the bound on wavefronts per SIMD keeps the compiler from fetching further ahead than occupancy is worth: 208 registers otherwise)
__global__ __launch_bounds__(PHASES == 3 ? 1024 : 256, PHASES == 2 && HALVES == 1 ? 3 : 4) void attention_cache_i4_kernel(const CacheAttentionArgs A)
{
    const uint32_t r1 = div_by(blockIdx.x, A.by_kv_heads), kvh = blockIdx.x - r1 * A.by_kv_heads.d;
    const uint32_t r2 = div_by(r1, A.by_chunks), chunk = r1 - r2 * A.by_chunks.d;
    const uint32_t seq = div_by(r2, A.by_splits), split = r2 - seq * A.by_splits.d;
    cache_attention_body<D, VARIANT, HALVES, PHASES>(A, kvh, seq, chunk, split);
}

hipError_t attention_cache_i4_launch_32(const CacheAttentionArgs &a, int halves, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);
hipError_t attention_cache_i4_launch_64(const CacheAttentionArgs &a, int halves, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);
hipError_t attention_cache_i4_launch_96(const CacheAttentionArgs &a, int halves, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);
hipError_t attention_cache_i4_launch_128(const CacheAttentionArgs &a, int halves, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream);

// One file per head dimension instantiates its kernels.
template <int D, int VARIANT>
hipError_t attention_cache_i4_launch_of(const CacheAttentionArgs &a, int halves, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream)
{
    auto kernel = phases == 3 ? (halves == 1 ? attention_cache_i4_kernel<D, VARIANT, 1, 3> : attention_cache_i4_kernel<D, VARIANT, 2, 3>)
                  : phases == 2 ? (halves == 1 ? attention_cache_i4_kernel<D, VARIANT, 1, 2> : attention_cache_i4_kernel<D, VARIANT, 2, 2>)
                  : halves == 1 ? attention_cache_i4_kernel<D, 0, 1, 1> : attention_cache_i4_kernel<D, 0, 2, 1>;
    launch_kernel(kernel, dim3(grid), dim3(block), lds, stream, a);
    return take_launch_status();
}
#define IPTQ_ATTENTION_CACHE_I4_OF(D)                                                                                         \
    hipError_t iptq::attention_cache_i4_launch_##D(const CacheAttentionArgs &a, int halves, int phases, uint32_t grid, uint32_t block, \
                                                   size_t lds, hipStream_t stream)                                            \
    {                                                                                                                         \
        return (a.P.variant == 0   ? attention_cache_i4_launch_of<D, 0>                                                       \
                : a.P.variant == 1 ? attention_cache_i4_launch_of<D, 1>                                                       \
                                   : attention_cache_i4_launch_of<D, 2>)(a, halves, phases, grid, block, lds, stream);            \
    }

}  // namespace iptq
