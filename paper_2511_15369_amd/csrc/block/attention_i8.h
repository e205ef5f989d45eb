// Attention over packed prompts: int8 queries, keys and values -> int8, the softmax's bit-shifting
// exponentials between two integer matrix products.
//
//   x_j = q . k_j                                     (v_mfma_i32_32x32x32_i8)
//   w_j = the exponential of x_j against the row's maximum (steps 1-5 of the softmax), below 2^15 - 128
//   o   = floor(2^54 / sum w_j) * sum_j w_j v_j >> 46,    out = the output step of o
//
// The exponentials need the row's maximum before the first of them (their floors do not commute with
// a later rescaling), so the keys are run over twice: once for the maximum, once for weights and
// values.  The weights go into the second product as two 8-bit halves, w = 256 hi + lo.
//
// Bound by the issue of vector and matrix instructions: 16 products of 32 x 32 x 32 per 32 queries and 32 keys (4 for the maximum, 4
// for the scores, 8 for the values' two halves) and about 180 vector instructions, of two wavefronts per SIMD, which is as many as
// 256 registers allow.  One prompt of 8192 tokens, 32 heads on 8 of 128, causal: 620 to 640 us, 1.7 POP/s of products done, four fifths of
// what a large library product of int8 reaches; matrix units 34 % busy, vector units 55 %.  24 prompts of 17 to 1900 tokens: 190 us.
// Weights from a table in LDS in place of the arithmetic (half or none of the vector work) gave 3.5 and 5 % at 22 KB more LDS per
// workgroup; a third tile buffer, wavefront priorities, scores of all 128 queries by each wavefront for a quarter of the keys gave nothing.
//
// A wavefront owns 32 queries and computes transposed scores, keys x queries: in the accumulator's layout a lane
// then holds 16 scores of one query, and with the keys of a 32-key block read in the order
// pi(8 i + 4 h + c) = 16 h + 4 i + c these are keys 16 h .. 16 h + 15 (h the lane's half), which is what
// the second product wants of its right operand: weights stay in the lane that made them.
#pragma once

#include "block.h"

namespace iptq {

// The output step where the means are below 2^15 in magnitude, as those of int8 values with eight fractional bits are: products
// below 2^30 (from s = 31 on all of them round to 0).
struct NarrowPost {
    int32_t m, s, rnd;
};
inline NarrowPost narrow_post_of(int32_t m, int32_t s)
{
    if (s > 30) return {0, 0, 0};
    return {m, s, s > 0 ? 1 << (s - 1) : 0};
}

struct AttentionArgs {
    const int8_t *q, *k, *v;
    int8_t *out;
    int64_t q_stride, k_stride, v_stride, out_stride;
    const int32_t *q_offsets, *k_offsets;
    int32_t q_tokens, k_tokens, q_len, k_len, max_q;      // q_len, k_len: of every sequence where there are no offsets
    DivDev by_kv_heads, by_group, by_seq;                 // workgroup number -> kv head, heads of its group, sequence, tile
    int32_t together;                                     // log2 of the heads of a group that a workgroup takes
    uint32_t tiles;
    uint32_t first_wg;                                    // of this launch
    AttentionDev P;
    NarrowPost post;
};

constexpr int kWaves = 4;             // 32 queries each, of one head or of several that share a kv head
constexpr int kQueries = 32 * kWaves;
constexpr int kKeys = 64;             // keys per staged tile

// Position in LDS of key `key` of a 32-key block.
IPTQ_DEV int key_row(int key) { return (key & ~31) | ((key >> 2 & 3) << 3) | ((key >> 4 & 1) << 2) | (key & 3); }

typedef i32x4 __attribute__((aligned(1))) i32x4_a1;
typedef int32_t __attribute__((aligned(1))) i32_a1;

// 16 scores of a lane, brought to i0's scale and stabilised -> 16 weights as two 8-bit halves; adds them up.
template <int VARIANT>
IPTQ_DEV void weights_of_scores(const i32x16 &x, const AttentionDev &P, i32x4 *hi, i32x4 *lo, uint32_t *sum)
{
    const i16x2 least = {(short)-P.d_clamp, (short)-P.d_clamp};
#pragma unroll
    for (int g = 0; g < 2; ++g) {                         // eight scores at a time
        uint32_t w[4];
        int32_t t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = x[8 * g + i] >> P.shift;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, __builtin_amdgcn_cvt_pk_i16(t[2 * i], t[2 * i + 1])), least));
        weights_of_pairs<VARIANT, 4>(w, P);
        uint32_t part[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i & 1] = __builtin_amdgcn_udot2(__builtin_bit_cast(u16x2_t, w[i]), (u16x2_t){1, 1}, i < 2 ? (i ? 0u : *sum) : part[i & 1], false);
        *sum = part[0] + part[1];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t h, l;
            split_weights(w[2 * i], w[2 * i + 1], &h, &l);
            (*hi)[2 * g + i] = (int32_t)h;
            (*lo)[2 * g + i] = (int32_t)l;
        }
    }
}

// What a workgroup works on: a sequence's queries [q0, q0 + nq) and keys [k0, k0 + nk) among the tokens, the first query of its tile.
struct AttentionTile {
    uint32_t head, kvh;
    int32_t q0, nq, k0, nk, diag, first;
};
// false: nothing to do
IPTQ_DEV bool attention_tile(const AttentionArgs &A, uint32_t wg, int queries, AttentionTile *t)
{
    const uint32_t r1 = div_by(wg, A.by_kv_heads);
    t->kvh = wg - r1 * A.by_kv_heads.d;
    const uint32_t r2 = div_by(r1, A.by_group);
    t->head = (t->kvh * A.by_group.d + (r1 - r2 * A.by_group.d)) << A.together;
    // (sequences change places from tile to tile: workgroups go to the chip's parts in turn, and a long sequence in the same place every time
    // would keep meeting the same ones: 24 of 17 to 1900 tokens, 32 queries of four heads a workgroup, 404 us, so 190.)
    const uint32_t r3 = div_by(r2, A.by_seq), turned = r2 - r3 * A.by_seq.d + r3, seq = turned - div_by(turned, A.by_seq) * A.by_seq.d;
    t->first = (int32_t)(A.tiles - 1 - r3) * queries;     // the longest rows first
    if (A.q_offsets) {
        clamped_range(A.q_offsets[seq], A.q_offsets[seq + 1], A.q_tokens, &t->q0, &t->nq);
        clamped_range(A.k_offsets[seq], A.k_offsets[seq + 1], A.k_tokens, &t->k0, &t->nk);
        if (t->nk > IPTQ_KEYS_MAX) return false;          // not served: its rows are left as they were
    } else {
        t->nq = A.q_len; t->nk = A.k_len;
        t->q0 = (int32_t)seq * t->nq; t->k0 = (int32_t)seq * t->nk;
    }
    t->diag = t->nk - t->nq;                              // causal: query i sees keys 0 .. i + diag
    t->nq = min(t->nq, A.max_q);
    return t->first < t->nq;
}

// Where the sums of shifted scores start so that they come out stabilised: x' - max x' ==
// (x + rounding - (max x' << shift)) >> shift.
IPTQ_DEV int32_t score_start(int32_t top, int shift)
{
    const int32_t rounding = shift > 0 ? 1 << (shift - 1) : 0;
    return top == kI32Min ? 0 : rounding - (((top + rounding) >> shift) << shift);
}

// Rows of V in LDS, bytes: eight of them, 32 bytes of each, meet all banks once.
template <int D> struct ValueRow { static constexpr int bytes = D == 128 ? 160 : D == 64 ? 96 : D; };

typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
// Left operand of the second product, 32 channels x 32 keys, out of rows of keys: the transposing read gives a lane
// eight keys' bytes of one channel.  src: the lane's address for the block's first eight keys.
template <int ROW>
IPTQ_DEV i32x4 values_of_block(const int8_t *src)
{
    typedef __attribute__((address_space(3))) i32x2 *Lds;
    const i32x2 a = __builtin_amdgcn_ds_read_tr8_b64_v2i32((Lds)(uintptr_t)(src));
    const i32x2 b = __builtin_amdgcn_ds_read_tr8_b64_v2i32((Lds)(uintptr_t)(src + 8 * ROW));
    return (i32x4){a.x, a.y, b.x, b.y};
}

// floor(2^54 / sum) times four sums, 46 bits down, requantized.  NARROW: the sum of the weights is below 2^24, that of the weighted
// values below 2^31 then, and f = 2^32 fh + fl with a signed fl has two products in place of five.
template <bool NARROW, typename Sum>
IPTQ_DEV int32_t means_of(uint64_t f, const Sum (&acc)[4], const AttentionArgs &A)
{
    const int32_t fl = (int32_t)f, fh = (int32_t)((int64_t)(f - (uint64_t)(int64_t)fl) >> 32);
    int32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int32_t o = NARROW ? (fh * (int32_t)acc[i] + __mulhi(fl, (int32_t)acc[i])) >> 14 : mean_of(f, acc[i], 46);
        c[i] = clamp_i32(((__mul24(o, A.post.m) + A.post.rnd) >> A.post.s) + A.P.post.zp, A.P.post.qmin, A.P.post.qmax);
    }
    return (int32_t)four_bytes(c);
}
// 16 outputs of a 32-channel block
template <bool NARROW>
IPTQ_DEV void store_block(int8_t *out, uint64_t f, const i32x16 &hi, const i32x16 &lo, int half, const AttentionArgs &A)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int64_t acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = NARROW ? (hi[4 * i + j] << 8) + lo[4 * i + j] : (int64_t)hi[4 * i + j] * 256 + lo[4 * i + j];
        *reinterpret_cast<i32_a1 *>(out + 8 * i + 4 * half) = means_of<NARROW>(f, acc, A);
    }
}

template <int D, int VARIANT>
__global__ __launch_bounds__(64 * kWaves, 2) void attention_i8_kernel(const AttentionArgs A)
{
    constexpr int STEPS = D / 32;                     // 32-channel steps of the first product, blocks of the second
    constexpr int KROW = D + 16, VROW = ValueRow<D>::bytes;
    constexpr int CHUNKS = kKeys * D / 16, LOADS = (CHUNKS + 64 * kWaves - 1) / (64 * kWaves);
    __shared__ __attribute__((aligned(16))) int8_t lds_k[2][kKeys * KROW];
    __shared__ __attribute__((aligned(16))) int8_t lds_v[2][kKeys * VROW];

    AttentionTile T;
    const int queries = kQueries >> A.together;
    if (!attention_tile(A, A.first_wg + blockIdx.x, queries, &T)) return;
    const int32_t nq = T.nq, nk = T.nk;
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t first = T.first + (32 * wave & (queries - 1));      // the wavefront's first query
    const uint32_t head = T.head + (uint32_t)(wave >> (2 - A.together));
    const int32_t row = first + col;
    const int32_t limit = A.P.causal ? min(max(row + T.diag + 1, 0), nk) : nk;
    // keys that any / every row of the wavefront sees, and that any row of the workgroup sees
    const int32_t wave_most = first >= nq ? 0 : A.P.causal ? min(max(min(first + 32, nq) + T.diag, 0), nk) : nk;
    const int32_t wave_least = A.P.causal ? min(max(first + T.diag + 1, 0), nk) : nk;
    const int32_t most = A.P.causal ? min(max(min(T.first + queries, nq) + T.diag, 0), nk) : nk;

    i32x4 qf[STEPS];
    {
        const int8_t *p = A.q + (int64_t)(T.q0 + min(row, nq - 1)) * A.q_stride + head * D + 16 * half;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) qf[s] = *reinterpret_cast<const i32x4_a1 *>(p + 32 * s);
    }
    const int8_t *kp = A.k + (int64_t)T.k0 * A.k_stride + T.kvh * D, *vp = A.v + (int64_t)T.k0 * A.v_stride + T.kvh * D;

    // the thread's share of a tile: 16-byte chunks; keys past the last repeat it
    int chunk_key[LOADS], chunk_at[LOADS];
    bool chunk_mine[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int u = threadIdx.x + 64 * kWaves * i;
        chunk_mine[i] = CHUNKS % (64 * kWaves) == 0 || u < CHUNKS;
        chunk_key[i] = u / (D / 16);
        chunk_at[i] = 16 * (u - chunk_key[i] * (D / 16));
    }
    auto load = [&](const int8_t *base, int64_t stride, int32_t at, i32x4 (&t)[LOADS]) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (chunk_mine[i]) t[i] = *reinterpret_cast<const i32x4_a1 *>(base + (int64_t)min(at + chunk_key[i], nk - 1) * stride + chunk_at[i]);
    };
    auto stage_k = [&](int buffer, const i32x4 (&t)[LOADS]) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (chunk_mine[i]) *reinterpret_cast<i32x4 *>(lds_k[buffer] + key_row(chunk_key[i]) * KROW + chunk_at[i]) = t[i];
    };
    auto stage_v = [&](int buffer, const i32x4 (&t)[LOADS]) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if (chunk_mine[i]) *reinterpret_cast<i32x4 *>(lds_v[buffer] + chunk_key[i] * VROW + chunk_at[i]) = t[i];
    };
    // transposed scores of keys [32 b, 32 b + 32) of a staged tile
    auto scores = [&](int buffer, int b, const i32x16 &start) {
        const int8_t *src = lds_k[buffer] + (32 * b + col) * KROW + 16 * half;
        i32x16 x = start;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            x = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4 *>(src + 32 * s), qf[s], x, 0, 0, 0);
        return x;
    };

    // first run over the keys: the row's maximum
    i32x4 kr[LOADS], vr[LOADS];
    i32x16 start;
#pragma unroll
    for (int i = 0; i < 16; ++i) start[i] = 0;
    int32_t top = kI32Min;
    if (most > 0) {
        load(kp, A.k_stride, 0, kr);
        stage_k(0, kr);
    }
    __syncthreads();
    int buffer = 0;
    for (int32_t at = 0; at < most; at += kKeys, buffer ^= 1) {
        const bool more = at + kKeys < most;
        load(kp, A.k_stride, more ? at + kKeys : 0, kr);      // the next tile, behind the last one the first again
        if (!more) load(vp, A.v_stride, 0, vr);
        if (at + kKeys <= wave_least) {
            const i32x16 x = scores(buffer, 0, start), y = scores(buffer, 1, start);
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(max(top, x[i]), y[i]);
        } else
#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b) {
            const int32_t k1 = at + 32 * b;
            if (k1 >= wave_most) break;
            const i32x16 x = scores(buffer, b, start);
            if (k1 + 32 <= wave_least) {
#pragma unroll
                for (int i = 0; i < 16; ++i) top = max(top, x[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) top = k1 + 16 * half + i < limit ? max(top, x[i]) : top;
            }
        }
        stage_k(buffer ^ 1, kr);
        if (!more) stage_v(buffer ^ 1, vr);
        __syncthreads();
    }
    top = max(top, __shfl_xor(top, 32));
    {
        const int32_t v = score_start(top, A.P.shift);
#pragma unroll
        for (int i = 0; i < 16; ++i) start[i] = v;
    }

    // second run: weights and weighted values
    i32x16 acc_hi[STEPS], acc_lo[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_hi[s][i] = acc_lo[s][i] = 0;
    uint32_t sum = 0;
    // the lane's part of a transposing read: key (lane % 16) / 2 of eight, channels 16 (lane / 16 % 2) + 8 (lane % 2) of 32
    const int v_lane = (16 * half + (lane >> 1 & 7)) * VROW + 16 * (lane >> 4 & 1) + 8 * (lane & 1);
    for (int32_t at = 0; at < most; at += kKeys, buffer ^= 1) {
        const bool more = at + kKeys < most;
        if (more) {
            load(kp, A.k_stride, at + kKeys, kr);
            load(vp, A.v_stride, at + kKeys, vr);
        }
        auto values = [&](int b, const i32x4 &hi, const i32x4 &lo) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const i32x4 vf = values_of_block<VROW>(lds_v[buffer] + 32 * b * VROW + v_lane + 32 * s);
                acc_hi[s] = __builtin_amdgcn_mfma_i32_32x32x32_i8(vf, hi, acc_hi[s], 0, 0, 0);
                acc_lo[s] = __builtin_amdgcn_mfma_i32_32x32x32_i8(vf, lo, acc_lo[s], 0, 0, 0);
            }
        };
        if (at < wave_most) {
            i32x16 x = scores(buffer, 0, start), y = scores(buffer, 1, start);
            if (at + kKeys > wave_least) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[i] = at + 16 * half + i < limit ? x[i] : kI32Min;
                    y[i] = at + 32 + 16 * half + i < limit ? y[i] : kI32Min;
                }
            }
            i32x4 hi, lo;
            weights_of_scores<VARIANT>(x, A.P, &hi, &lo, &sum);
            values(0, hi, lo);
            weights_of_scores<VARIANT>(y, A.P, &hi, &lo, &sum);
            values(1, hi, lo);
        }
        if (more) {
            stage_k(buffer ^ 1, kr);
            stage_v(buffer ^ 1, vr);
        }
        __syncthreads();
    }
    sum += (uint32_t)__shfl_xor((int32_t)sum, 32);
    if (row >= nq) return;
    const uint64_t f = floor_div_scaled(1, 54, sum);
    int8_t *out = A.out + (int64_t)(T.q0 + row) * A.out_stride + head * D;
    if (__all(sum < 1u << 24)) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) store_block<true>(out + 32 * s, f, acc_hi[s], acc_lo[s], half, A);
    } else {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) store_block<false>(out + 32 * s, f, acc_hi[s], acc_lo[s], half, A);
    }
}

// Few queries: a workgroup has 32, and its wavefronts divide the keys, blocks of 32 in turn.  Each keeps to itself until
// the maxima are joined, and again until the sums are: whole numbers, so their order does not matter.  (The sums change hands as rows of
// LDS: 32 atomics a lane in their place took 0.5 us of 197 tokens' 6.)  Bound by latency: 197 tokens, 3 heads of 64, 21
// workgroups of one block per wavefront, take 5.7 us; of their 10,000 cycles 2200 are the first loads, 1100 the scores, 2600 the weights and
// their product, 2500 the two joins.
constexpr int kFewWaves = 8;

// The wavefronts' tiles, and in the same place their sums of weighted values at the end; the maxima, the sums of the weights.
template <int D> struct FewLds {
    static constexpr int KROW = D + 16, VROW = ValueRow<D>::bytes, stage = 32 * (KROW + VROW);      // of a wavefront
    static constexpr int units = D / 32 * 4 * 64, acc = units * 16;       // a wavefront's sums, four to a unit
    static constexpr int shared = kFewWaves * (acc > stage ? acc : stage);
    static constexpr size_t bytes = shared + 32 * 4 * (1 + kFewWaves);
};

template <int D, int VARIANT>
__global__ __launch_bounds__(64 * kFewWaves) void attention_i8_few_kernel(const AttentionArgs A)
{
    typedef FewLds<D> L;
    constexpr int STEPS = D / 32, KROW = L::KROW, VROW = L::VROW;
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    i32x4 *lds_acc = reinterpret_cast<i32x4 *>(lds);
    int32_t *lds_top = reinterpret_cast<int32_t *>(lds + L::shared);
    uint32_t *lds_sum = reinterpret_cast<uint32_t *>(lds_top + 32);

    AttentionTile T;
    if (!attention_tile(A, A.first_wg + blockIdx.x, 32, &T)) return;
    const int32_t nq = T.nq, nk = T.nk;
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t row = T.first + col;
    const int32_t limit = A.P.causal ? min(max(row + T.diag + 1, 0), nk) : nk;
    const int32_t most = A.P.causal ? min(max(min(T.first + 32, nq) + T.diag, 0), nk) : nk;        // that any row sees
    const int32_t least = A.P.causal ? min(max(T.first + T.diag + 1, 0), nk) : nk;                 // that every row sees
    int8_t *stage_k = lds + wave * L::stage, *stage_v = stage_k + 32 * KROW;

    const int8_t *kp = A.k + (int64_t)T.k0 * A.k_stride + T.kvh * D, *vp = A.v + (int64_t)T.k0 * A.v_stride + T.kvh * D;
    auto load = [&](const int8_t *base, int64_t stride, int32_t at, i32x4 (&r)[STEPS]) {
        int l = lane;
        asm volatile("" : "+v"(l));                       // (addresses are made again: kept, they would spill)
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int u = l + 64 * i, key = u / (D / 16);
            r[i] = *reinterpret_cast<const i32x4_a1 *>(base + (int64_t)min(at + key, nk - 1) * stride + 16 * (u - key * (D / 16)));
        }
    };
    auto put_k = [&](const i32x4 (&r)[STEPS]) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int u = lane + 64 * i, key = u / (D / 16);
            *reinterpret_cast<i32x4 *>(stage_k + key_row(key) * KROW + 16 * (u - key * (D / 16))) = r[i];
        }
    };
    auto put_v = [&](const i32x4 (&r)[STEPS]) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int u = lane + 64 * i, key = u / (D / 16);
            *reinterpret_cast<i32x4 *>(stage_v + key * VROW + 16 * (u - key * (D / 16))) = r[i];
        }
    };
    const int32_t from = 32 * wave, step = 32 * kFewWaves;
    const bool busy = from < most;
    i32x4 qf[STEPS], kr[STEPS], vr[STEPS];
    if (busy) {
        load(kp, A.k_stride, from, kr);
        load(vp, A.v_stride, from, vr);
    }
    {
        const int8_t *p = A.q + (int64_t)(T.q0 + min(row, nq - 1)) * A.q_stride + T.head * D + 16 * half;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) qf[s] = *reinterpret_cast<const i32x4_a1 *>(p + 32 * s);
    }
    if (threadIdx.x < 32) lds_top[threadIdx.x] = kI32Min;
    __syncthreads();
    auto scores = [&]() {
        i32x16 x = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
            x = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4 *>(stage_k + col * KROW + 32 * s + 16 * half), qf[s], x, 0, 0, 0);
        return x;
    };
    int32_t top = kI32Min;
    i32x16 x;
    for (int32_t at = from; at < most; at += step) {
        wave_lds_fence();
        put_k(kr);
        if (at + step < most) load(kp, A.k_stride, at + step, kr);
        wave_lds_fence();
        x = scores();
        if (at + 32 <= least) {
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(top, x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) top = at + 16 * half + i < limit ? max(top, x[i]) : top;
        }
    }
    top = max(top, __shfl_xor(top, 32));
    if (busy && half == 0) atomicMax(lds_top + col, top);
    __syncthreads();
    const int32_t start = score_start(lds_top[col], A.P.shift);
    i32x16 acc_hi[STEPS], acc_lo[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_hi[s][i] = acc_lo[s][i] = 0;
    if (busy) {
        uint32_t sum = 0;
        const int v_lane = (16 * half + (lane >> 1 & 7)) * VROW + 16 * (lane >> 4 & 1) + 8 * (lane & 1);
        const bool once = from + step >= most;            // its only block's scores are still there
        if (!once) load(kp, A.k_stride, from, kr);
        for (int32_t at = from; at < most; at += step) {
            wave_lds_fence();
            put_v(vr);
            if (!once) put_k(kr);
            if (at + step < most) {
                load(kp, A.k_stride, at + step, kr);
                load(vp, A.v_stride, at + step, vr);
            }
            wave_lds_fence();
            if (!once) x = scores();
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] += start;
            if (at + 32 > least) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = at + 16 * half + i < limit ? x[i] : kI32Min;
            }
            i32x4 hi, lo;
            weights_of_scores<VARIANT>(x, A.P, &hi, &lo, &sum);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const i32x4 vf = values_of_block<VROW>(stage_v + v_lane + 32 * s);
                acc_hi[s] = __builtin_amdgcn_mfma_i32_32x32x32_i8(vf, hi, acc_hi[s], 0, 0, 0);
                acc_lo[s] = __builtin_amdgcn_mfma_i32_32x32x32_i8(vf, lo, acc_lo[s], 0, 0, 0);
            }
        }
        sum += (uint32_t)__shfl_xor((int32_t)sum, 32);
        if (half == 0) lds_sum[32 * wave + col] = sum;
    }
    if (most <= 0 && threadIdx.x < 32) lds_sum[threadIdx.x] = 0;
    // The wavefronts' sums, joined by whoever makes the outputs: 256 hi + lo at once where it fits 32 bits (up to 508 keys; a wavefront's of
    // up to 508 of its own, added up in 64), else one half after the other.
    const int waves = max(min(kFewWaves, (most + 31) >> 5), 1);       // (without keys the first's zeros)
    constexpr int MINE = (L::units + 64 * kFewWaves - 1) / (64 * kFewWaves);
    auto join = [&](auto &total, bool whole) {
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) total[m][j] = 0;
        for (int part = whole ? 1 : 0; part < 2; ++part) {
            __syncthreads();
            if (wave < waves) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        i32x4 v;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int32_t h = acc_hi[s][4 * i + j], l = acc_lo[s][4 * i + j];
                            v[j] = whole ? (h << 8) + l : part == 0 ? h : l;
                        }
                        lds_acc[wave * L::units + (4 * s + i) * 64 + lane] = v;
                    }
            }
            __syncthreads();
            const int up = part == 0 ? 8 : 0;
#pragma unroll
            for (int m = 0; m < MINE; ++m) {
                const int u = threadIdx.x + 64 * kFewWaves * m;
                if (u >= L::units) break;
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) {
                    if (w >= waves) break;
                    const i32x4 v = lds_acc[w * L::units + u];
#pragma unroll
                    for (int j = 0; j < 4; ++j) total[m][j] += sizeof(total[m][j]) == 4 ? v[j] : (int64_t)v[j] << up;
                }
            }
        }
    };
    // a thread's query and four channels: 32 s + 8 i + 4 h
    const int q = threadIdx.x & 31, h = threadIdx.x >> 5 & 1;
    auto mean_factor = [&]() {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) sum += w < waves ? lds_sum[32 * w + q] : 0;
        return floor_div_scaled(1, 54, sum);
    };
    auto store = [&](int m, int32_t bytes) {
        const int u = threadIdx.x + 64 * kFewWaves * m, i = u >> 6 & 3, s = u >> 8;
        if (u < L::units) *reinterpret_cast<i32_a1 *>(A.out + (int64_t)(T.q0 + T.first + q) * A.out_stride + T.head * D + 32 * s + 8 * i + 4 * h) = bytes;
    };
    if (most <= 508) {
        int32_t total[MINE][4];
        join(total, true);
        if (T.first + q >= nq) return;
        const uint64_t f = mean_factor();
#pragma unroll
        for (int m = 0; m < MINE; ++m) store(m, means_of<true>(f, total[m], A));
    } else {
        int64_t total[MINE][4];
        join(total, most <= 15 * step);
        if (T.first + q >= nq) return;
        const uint64_t f = mean_factor();
#pragma unroll
        for (int m = 0; m < MINE; ++m) store(m, means_of<false>(f, total[m], A));
    }
}

hipError_t attention_i8_launch_32(const AttentionArgs &a, bool few, uint32_t grid, hipStream_t stream);
hipError_t attention_i8_launch_64(const AttentionArgs &a, bool few, uint32_t grid, hipStream_t stream);
hipError_t attention_i8_launch_96(const AttentionArgs &a, bool few, uint32_t grid, hipStream_t stream);
hipError_t attention_i8_launch_128(const AttentionArgs &a, bool few, uint32_t grid, hipStream_t stream);

// One file per head dimension instantiates its kernels.
#define IPTQ_ATTENTION_I8_OF(D)                                                                                          \
    hipError_t iptq::attention_i8_launch_##D(const AttentionArgs &a, bool few, uint32_t grid, hipStream_t stream)                  \
    {                                                                                                                    \
        auto kernel = a.P.variant == 0 ? attention_i8_kernel<D, 0> : a.P.variant == 1 ? attention_i8_kernel<D, 1>        \
                                                                                      : attention_i8_kernel<D, 2>;       \
        if (few)                                                                                                         \
            kernel = a.P.variant == 0 ? attention_i8_few_kernel<D, 0> : a.P.variant == 1 ? attention_i8_few_kernel<D, 1> \
                                                                                         : attention_i8_few_kernel<D, 2>; \
        launch_kernel(kernel, dim3(grid), dim3(64 * (few ? kFewWaves : kWaves)), few ? FewLds<D>::bytes : 0, stream, a); \
        return take_launch_status();                                                                                     \
    }

}  // namespace iptq
