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
// A wavefront owns 32 queries and computes transposed scores, keys x queries: in the accumulator's layout a lane
// then holds 16 scores of one query, and with the keys of a 32-key block read in the order
// pi(8 i + 4 h + c) = 16 h + 4 i + c these are keys 16 h .. 16 h + 15 (h the lane's half), which is what
// the second product wants of its right operand: weights stay in the lane that made them.
#pragma once

#include "block.h"

namespace iptq {

struct AttentionArgs {
    const int8_t *q, *k, *v;
    int8_t *out;
    int64_t q_stride, k_stride, v_stride, out_stride;
    const int32_t *q_offsets, *k_offsets;
    int32_t q_tokens, k_tokens, q_len, k_len, max_q;      // q_len, k_len: of every sequence where there are no offsets
    int32_t kv_heads, group;
    DivDev by_kv_heads, by_group, by_seq;                 // workgroup number -> kv head, head of its group, sequence, tile
    uint32_t tiles;
    AttentionDev P;
};

constexpr int kWaves = 4;             // 32 queries each
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
    for (int i = 0; i < 4; ++i) {
        uint32_t w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int32_t a = x[4 * i + 2 * j] >> P.shift, b = x[4 * i + 2 * j + 1] >> P.shift;
            i16x2 d = __builtin_bit_cast(i16x2, __builtin_amdgcn_cvt_pk_i16(a, b));
            d = __builtin_elementwise_max(d, least);
            w[j] = weights_of_pair<VARIANT>(d, P);
            *sum = __builtin_amdgcn_udot2(__builtin_bit_cast(u16x2_t, w[j]), (u16x2_t){1, 1}, *sum, false);
        }
        uint32_t h, l;
        split_weights(w[0], w[1], &h, &l);
        (*hi)[i] = (int32_t)h;
        (*lo)[i] = (int32_t)l;
    }
}

template <int D, int VARIANT>
__global__ __launch_bounds__(64 * kWaves) void attention_i8_kernel(const AttentionArgs A)
{
    constexpr int STEPS = D / 32;                     // 32-channel steps of the first product, blocks of the second
    constexpr int KROW = D + 16, VROW = kKeys + 16;   // LDS rows in bytes, padded
    __shared__ __attribute__((aligned(16))) int8_t lds_k[kKeys * KROW];
    __shared__ __attribute__((aligned(16))) int8_t lds_v[D * VROW];

    const uint32_t wg = blockIdx.x;
    const uint32_t r1 = div_by(wg, A.by_kv_heads), kvh = wg - r1 * (uint32_t)A.kv_heads;
    const uint32_t r2 = div_by(r1, A.by_group), head = kvh * (uint32_t)A.group + (r1 - r2 * (uint32_t)A.group);
    const uint32_t r3 = div_by(r2, A.by_seq), seq = r2 - r3 * A.by_seq.d;
    const int32_t tile0 = (int32_t)(A.tiles - 1 - r3) * kQueries;       // the longest rows first

    int32_t q0, k0, nq, nk;
    if (A.q_offsets) {
        clamped_range(A.q_offsets[seq], A.q_offsets[seq + 1], A.q_tokens, &q0, &nq);
        clamped_range(A.k_offsets[seq], A.k_offsets[seq + 1], A.k_tokens, &k0, &nk);
        if (nk > IPTQ_KEYS_MAX) return;               // not served: its rows are left as they were
    } else {
        nq = A.q_len; nk = A.k_len;
        q0 = (int32_t)seq * nq; k0 = (int32_t)seq * nk;
    }
    const int32_t diag = nk - nq;                     // causal: query i sees keys 0 .. i + diag
    nq = min(nq, A.max_q);
    if (tile0 >= nq) return;

    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t first = tile0 + 32 * wave;          // the wavefront's first query
    const int32_t row = first + col;
    const int32_t limit = A.P.causal ? min(max(row + diag + 1, 0), nk) : nk;
    // keys that any / every row of the wavefront sees, and that any row of the workgroup sees
    const int32_t wave_most = first >= nq ? 0 : A.P.causal ? min(max(min(first + 32, nq) + diag, 0), nk) : nk;
    const int32_t wave_least = A.P.causal ? min(max(first + diag + 1, 0), nk) : nk;
    const int32_t most = A.P.causal ? min(max(min(tile0 + kQueries, nq) + diag, 0), nk) : nk;

    i32x4 qf[STEPS];
    {
        const int8_t *p = A.q + (int64_t)(q0 + min(row, nq - 1)) * A.q_stride + head * D + 16 * half;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) qf[s] = *reinterpret_cast<const i32x4_a1 *>(p + 32 * s);
    }
    const int8_t *kp = A.k + (int64_t)k0 * A.k_stride + kvh * D, *vp = A.v + (int64_t)k0 * A.v_stride + kvh * D;

    auto stage_k = [&](int32_t at) {
        for (int u = threadIdx.x; u < kKeys * D / 16; u += 64 * kWaves) {
            const int key = u / (D / 16), c = u - key * (D / 16);
            const i32x4 t = *reinterpret_cast<const i32x4_a1 *>(kp + (int64_t)min(at + key, nk - 1) * A.k_stride + 16 * c);
            *reinterpret_cast<i32x4 *>(lds_k + key_row(key) * KROW + 16 * c) = t;
        }
    };
    auto stage_v = [&](int32_t at) {                  // transposed: four keys' bytes of one channel side by side
        for (int u = threadIdx.x; u < kKeys * D / 16; u += 64 * kWaves) {
            const int g = u / (D / 4), c = u - g * (D / 4);
            uint32_t t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                t[j] = *reinterpret_cast<const i32_a1 *>(vp + (int64_t)min(at + 4 * g + j, nk - 1) * A.v_stride + 4 * c);
            const uint32_t a = __builtin_amdgcn_perm(t[1], t[0], 0x05010400u), b = __builtin_amdgcn_perm(t[1], t[0], 0x07030602u);
            const uint32_t e = __builtin_amdgcn_perm(t[3], t[2], 0x05010400u), f = __builtin_amdgcn_perm(t[3], t[2], 0x07030602u);
            uint32_t *o = reinterpret_cast<uint32_t *>(lds_v + 4 * c * VROW + 4 * g);
            o[0] = __builtin_amdgcn_perm(e, a, 0x05040100u);
            o[VROW / 4] = __builtin_amdgcn_perm(e, a, 0x07060302u);
            o[2 * VROW / 4] = __builtin_amdgcn_perm(f, b, 0x05040100u);
            o[3 * VROW / 4] = __builtin_amdgcn_perm(f, b, 0x07060302u);
        }
    };
    // transposed scores of keys [32 b, 32 b + 32) of the staged tile; init: where the sums start
    auto scores = [&](int b, int32_t init) {
        i32x16 x;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = init;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const i32x4 kf = *reinterpret_cast<const i32x4 *>(lds_k + (32 * b + col) * KROW + 32 * s + 16 * half);
            x = __builtin_amdgcn_mfma_i32_32x32x32_i8(kf, qf[s], x, 0, 0, 0);
        }
        return x;
    };

    // first run over the keys: the row's maximum
    int32_t top = kI32Min;
    for (int32_t at = 0; at < most; at += kKeys) {
        __syncthreads();
        stage_k(at);
        __syncthreads();
#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b) {
            const int32_t k1 = at + 32 * b;
            if (k1 >= wave_most) break;
            const i32x16 x = scores(b, 0);
            if (k1 + 32 <= wave_least) {
#pragma unroll
                for (int i = 0; i < 16; ++i) top = max(top, x[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) top = k1 + 16 * half + i < limit ? max(top, x[i]) : top;
            }
        }
    }
    top = max(top, __shfl_xor(top, 32));
    // x' - max x' == (x + rounding - (max x' << shift)) >> shift: the sums start at what lies behind x
    const int32_t rounding = A.P.shift > 0 ? 1 << (A.P.shift - 1) : 0;
    const int32_t init = top == kI32Min ? 0 : rounding - (((top + rounding) >> A.P.shift) << A.P.shift);

    // second run: weights and weighted values
    i32x16 acc_hi[STEPS], acc_lo[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc_hi[s][i] = acc_lo[s][i] = 0;
    uint32_t sum = 0;
    for (int32_t at = 0; at < most; at += kKeys) {
        __syncthreads();
        stage_k(at);
        stage_v(at);
        __syncthreads();
#pragma unroll
        for (int b = 0; b < kKeys / 32; ++b) {
            const int32_t k1 = at + 32 * b;
            if (k1 >= wave_most) break;
            i32x16 x = scores(b, init);
            if (k1 + 32 > wave_least) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = k1 + 16 * half + i < limit ? x[i] : kI32Min;
            }
            i32x4 hi, lo;
            weights_of_scores<VARIANT>(x, A.P, &hi, &lo, &sum);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const i32x4 vf = *reinterpret_cast<const i32x4 *>(lds_v + (32 * s + col) * VROW + 32 * b + 16 * half);
                acc_hi[s] = __builtin_amdgcn_mfma_i32_32x32x32_i8(vf, hi, acc_hi[s], 0, 0, 0);
                acc_lo[s] = __builtin_amdgcn_mfma_i32_32x32x32_i8(vf, lo, acc_lo[s], 0, 0, 0);
            }
        }
    }
    sum += (uint32_t)__shfl_xor((int32_t)sum, 32);
    if (row >= nq) return;
    const uint64_t f = floor_div_u64((uint64_t)1 << 54, sum);
    int8_t *out = A.out + (int64_t)(q0 + row) * A.out_stride + head * D;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t bytes = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t acc = (int64_t)acc_hi[s][4 * i + j] * 256 + acc_lo[s][4 * i + j];
                bytes |= (uint32_t)(mean_byte(f, acc, 46, A.P.post) & 255) << (8 * j);
            }
            *reinterpret_cast<i32_a1 *>(out + 32 * s + 8 * i + 4 * half) = (int32_t)bytes;
        }
}

hipError_t attention_i8_launch_32(const AttentionArgs &a, uint32_t grid, hipStream_t stream);
hipError_t attention_i8_launch_64(const AttentionArgs &a, uint32_t grid, hipStream_t stream);
hipError_t attention_i8_launch_96(const AttentionArgs &a, uint32_t grid, hipStream_t stream);
hipError_t attention_i8_launch_128(const AttentionArgs &a, uint32_t grid, hipStream_t stream);

// One file per head dimension instantiates its kernels.
#define IPTQ_ATTENTION_I8_OF(D)                                                                                          \
    hipError_t iptq::attention_i8_launch_##D(const AttentionArgs &a, uint32_t grid, hipStream_t stream)                  \
    {                                                                                                                    \
        auto kernel = a.P.variant == 0 ? attention_i8_kernel<D, 0> : a.P.variant == 1 ? attention_i8_kernel<D, 1>        \
                                                                                      : attention_i8_kernel<D, 2>;       \
        launch_kernel(kernel, dim3(grid), dim3(64 * kWaves), 0, stream, a);                                              \
        return take_launch_status();                                                                                     \
    }

}  // namespace iptq
