// Operators of a transformer block beside its softmax and GELU: launch records, host entry points of the
// kernel files and the integer helpers they share.  Like the kernels one folder up these hold integer
// instructions only; the products of queries with keys and of weights with values run on the matrix cores'
// integer forms (v_mfma_i32).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../device_common.h"
#include "../plan.h"

namespace iptq {

typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

constexpr uint32_t kLaunchMost = 1u << 22;                // workgroups of a launch: its threads are counted in 32 bits
constexpr int kGroup = 64;            // channels that share one step of the 4-bit cache

// Unsigned division by a run-time constant (the compiler's own goes through floating point).
struct DivDev {
    uint32_t d, magic;
    int32_t sh;
};
inline DivDev div_of(uint32_t d)      // 1 <= d, dividends below 2^31
{
    DivDev v = {d, 0, 0};
    if (d > 1) make_magic_u32(d, 31, &v.magic, &v.sh);
    return v;
}
IPTQ_HD uint32_t div_by(uint32_t n, const DivDev &D) { return D.d == 1 ? n : mulhi_u32(n, D.magic) >> D.sh; }

// rshr_round(x m, s) for |x| < 2^31, |m| < 2^15.  fast (s >= 16): one multiplication and a shift of its upper half (mul and rnd
// moved up to where the result's lowest bit is the upper half's), and the result fits 32 bits.
struct ShiftDev {
    int32_t m, s;
    int32_t mul, sh;
    int64_t rnd;
};
inline ShiftDev shift_of(int32_t m, int32_t s, bool fast)
{
    ShiftDev v = {m, s, 0, 0, s > 0 ? (int64_t)1 << (s - 1) : 0};
    if (fast) {
        v.mul = (int32_t)((uint32_t)m << (s <= 32 ? 32 - s : 0));
        v.sh = s > 32 ? s - 32 : 0;
        if (s <= 32) v.rnd = (int64_t)1 << 31;
    }
    return v;
}

// Constants of an attention's exponentials and of its output step.
struct AttentionDev {
    int32_t variant, i0, i0n, n_shift;
    int32_t d_clamp;                  // deltas below -D have weight 0
    int32_t div8;                     // byte divider by i0 (SoftmaxDev::div8)
    uint32_t d2_magic;                // second degree: division by 2 i0
    int32_t d2_sh;
    int32_t shift;                    // scores are brought to i0's scale by a rounding shift
    int32_t causal;
    DyadicDev post;
    ShiftDev post_shift;
};

struct AttentionCall {
    const int8_t *q, *k, *v;
    int8_t *out;
    int64_t q_stride, k_stride, v_stride, out_stride;     // bytes between two tokens
    const int32_t *q_offsets, *k_offsets;                 // [n_seq + 1] on the device, or nullptr: equal lengths
    int64_t q_tokens, k_tokens;
    int32_t n_seq, max_q, heads, kv_heads, dim;
    AttentionDev P;
};

struct CacheDev {
    uint8_t *k_codes, *k_steps, *v_codes, *v_steps;
    int32_t n_pages, page_tokens, page_log, kv_heads, dim;
};

struct CacheAttentionCall {
    const int8_t *q;
    int8_t *out;
    int64_t q_stride, out_stride;
    const int32_t *pages, *lengths;
    int32_t n_seq, max_pages, q_tokens, heads;
    void *work;
    CacheDev C;
    AttentionDev P;
};

struct CacheStoreCall {
    const int8_t *k, *v;
    int64_t k_stride, v_stride;
    const int32_t *slots;
    int64_t tokens;
    CacheDev C;
};

struct RmsnormCall {
    const int32_t *x, *residual;
    int32_t *residual_out;
    const int16_t *gain;
    int8_t *out;
    int32_t *row_scales;
    int64_t rows;
    int32_t cols;
    int32_t in_m, in_s;
    int64_t eps_sum;                  // cols * eps
    uint32_t root_cols;               // floor(sqrt(cols) 2^16)
    DyadicDev post;
};

hipError_t attention_i8_dispatch(const AttentionCall &c, hipStream_t stream);
hipError_t cache_store_i4_dispatch(const CacheStoreCall &c, hipStream_t stream);
int64_t attention_cache_i4_workspace_bytes(const CacheAttentionCall &c);
hipError_t attention_cache_i4_dispatch(const CacheAttentionCall &c, hipStream_t stream);
hipError_t rmsnorm_i32_dispatch(const RmsnormCall &c, hipStream_t stream);
hipError_t requant_rows_dispatch(const int32_t *in, const int32_t *row_scales, int32_t row_shift, void *out, int64_t rows,
                                 int32_t cols, const DyadicDev &P, hipStream_t stream);

// 2^63 / (den << k), k the zeros in front of den >= 1: never above it and at most 6 below (Newton's iteration, as floor_pow2_div;
// within 2 of it for every y, less 4).
IPTQ_HD uint32_t reciprocal_of(uint32_t den, int k)
{
    const uint32_t y = den << k;
    uint32_t r = (3031741620u - mulhi_u32(y, 2021161080u)) << 1;
    for (int it = 0; it < 3; ++it) r = mulhi_u32(r, 0u - mulhi_u32(y, r)) << 1;
    return r - 4;
}

// floor(2^61 / den) for 2^30 <= den < 2^31: half of the reciprocal is at most four short.
IPTQ_HD uint32_t floor_div_2_61(uint32_t den)
{
    uint32_t q = reciprocal_of(den, 1) >> 1;
    uint64_t left = ((uint64_t)1 << 61) - (uint64_t)q * den;
    while (left >= den) {
        left -= den;
        ++q;
    }
    return q;
}

// floor(c 2^n / den) for 32 <= n, c 2^n <= 2^54 (0 for den == 0): the reciprocal is the first quotient, shifted; what it leaves
// is below den + 6 c 2^(n - 31), below 2^32 while den is below 2^31, so its low word, that of -q den, is all of it, and one more quotient is at
// most one short.  (The weights of 131072 keys may add up to more than 2^31.)
IPTQ_HD uint64_t floor_div_scaled(uint32_t c, int n, uint32_t den)
{
    if (den == 0) return 0;
    const int k = clz_u32(den), down = 63 - n - k;
    const uint32_t r = reciprocal_of(den, k);
    uint64_t q = (uint64_t)r * c;
    q = down >= 0 ? q >> down : q << -down;
    if (k == 0) return q + (((uint64_t)c << n) - q * den >= den ? 1 : 0);
    uint32_t left = 0u - (uint32_t)q * den;
    const uint32_t e = mulhi_u32(left, r) >> (31 - k);
    left -= e * den;
    return q + e + (left >= den ? 1 : 0);
}

// floor(sqrt(v)) for 2^60 <= v < 2^62: Newton's iteration for 1 / sqrt(a), a = v / 2^62 in [1/4, 1), in 32 bits, one step of the
// remainder in 64, and the last unit by trial.  (Bit by bit it was the longest part of a short call's chain.)
IPTQ_HD uint32_t root_u62(uint64_t v)
{
    const uint32_t a = (uint32_t)(v >> 30);               // Q32
    uint32_t y = 2469606196u - mulhi_u32(a, 1471026135u); // 2.3 - 1.37 a in Q30: within a seventh
    for (int i = 0; i < 5; ++i) {                         // y (3 - a y^2) / 2
        const uint32_t t = mulhi_u32(a, mulhi_u32(y, y)); // Q28, about 1
        y = mulhi_u32(y, 805306368u - t) << 3;
    }
    uint32_t r = mulhi_u32(a, y) << 1;                    // Q32 Q30 -> Q30, wanted in Q31
    const int64_t left = (int64_t)(v - (uint64_t)r * r);
    r += (uint32_t)(((left >> 8) * (int64_t)y) >> 54);    // 1 / (2 sqrt(v)) = y / 2^32
    while ((uint64_t)r * r > v) --r;
    while ((uint64_t)(r + 1) * (r + 1) <= v) ++r;
    return r;
}

// ---- what the device reads of tables and offsets, kept inside the tensors -----------------------------------
// Tokens [from, from + n) of a sequence with offsets a and b, inside [0, tokens).
IPTQ_HD void clamped_range(int32_t a, int32_t b, int32_t tokens, int32_t *from, int32_t *n)
{
    *from = a < 0 ? 0 : a > tokens ? tokens : a;
    *n = (b < *from ? *from : b > tokens ? tokens : b) - *from;
}

// The page of a sequence's key, or -1 where the sequence or the cache has none.
IPTQ_HD int32_t page_of_key(const int32_t *table, int page_log, int32_t n_pages, int32_t key, int32_t length)
{
    if (key >= length) return -1;
    const int32_t page = table[key >> page_log];
    return page >= 0 && page < n_pages ? page : -1;
}

// ---- weights ------------------------------------------------------------------------------------
// The bit-shifting exponentials of 2 N scores in 16-bit halves: `d` are stabilised scores, clamped at -D, the results
// (base << N) >> q below 2^15 - 128 (Eq. 7-10, 13-14; the second degree).  Every packed step is N independent
// instructions side by side: a pair alone is one chain, each of whose links waits for the one before.
// The compiler would undo that to save registers: only products, scalar and memory instructions may pass the ends of a step.
IPTQ_DEV void end_of_step() { __builtin_amdgcn_sched_barrier(0x9c); }
template <int N> struct Pairs { uint32_t v[N]; };
template <int VARIANT, int N>
IPTQ_DEV void weights_of_pairs(uint32_t (&d)[N], const AttentionDev &P)
{
    typedef short S __attribute__((ext_vector_type(2 * N)));
    typedef unsigned short U __attribute__((ext_vector_type(2 * N)));
    typedef Pairs<N> W;
    const S x = __builtin_bit_cast(S, *reinterpret_cast<W *>(d));
    const S half = x >> (short)1;
    end_of_step();
    const S more = x + half;
    end_of_step();
    const S sixteenth = x >> (short)4;
    end_of_step();
    const S m = more - sixteenth;                                      // Qp of Eq. 7, in (-2^15, 0]
    end_of_step();
    const W mw = __builtin_bit_cast(W, m);
    // Eq. 8: (-m) div i0 is the top byte of (-m) ceil(2^24 / i0), both factors negated
    W qw;
    uint32_t a[N], b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        a[i] = (uint32_t)__mul24((int32_t)(int16_t)mw.v[i], P.div8);
        b[i] = (uint32_t)__mul24((int32_t)mw.v[i] >> 16, P.div8);
    }
    end_of_step();
#pragma unroll
    for (int i = 0; i < N; ++i) qw.v[i] = __builtin_amdgcn_perm(b[i], a[i], 0x0c070c03u);
    end_of_step();
    const U q = __builtin_bit_cast(U, qw);
    const S nr = (S)(q * (unsigned short)P.i0 + (U)m);                 // -r in (-i0, 0]
    end_of_step();
    S fr = nr >> (short)1;                                             // Eq. 10
    if (VARIANT >= 1) {                                                // Eq. 13
        end_of_step();
        const S eighth = nr >> (short)3;
        end_of_step();
        fr = fr + eighth;
        const S last = nr >> (short)4;
        end_of_step();
        fr = fr + last;
    }
    if (VARIANT == 2) {                                                // Eq. 11, second degree
        S t;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) {
            const int32_t y = fr[i];
            t[i] = (short)(mulhi_u32((uint32_t)__mul24(y, y), P.d2_magic) >> P.d2_sh);
        }
        fr = fr + t;
    }
    end_of_step();
    const U base = (U)fr * (unsigned short)(1u << P.n_shift) + (unsigned short)P.i0n;
    end_of_step();
    *reinterpret_cast<W *>(d) = __builtin_bit_cast(W, (U)(base >> q)); // q <= 15
    end_of_step();
}

// Weights as the two 8-bit factors of a signed matrix product: w = 256 hi + lo with lo in [-128, 127], so
// hi = (w + 128) >> 8 is at most 127 for w <= 32639.  Two pairs of weights -> four bytes of each.
IPTQ_DEV void split_weights(uint32_t w01, uint32_t w23, uint32_t *hi, uint32_t *lo)
{
    const u16x2_t half = {128, 128};
    const uint32_t a = __builtin_bit_cast(uint32_t, (u16x2_t)(__builtin_bit_cast(u16x2_t, w01) + half));
    const uint32_t b = __builtin_bit_cast(uint32_t, (u16x2_t)(__builtin_bit_cast(u16x2_t, w23) + half));
    *hi = __builtin_amdgcn_perm(b, a, 0x07050301u);
    *lo = __builtin_amdgcn_perm(w23, w01, 0x06040200u);
}

IPTQ_DEV int32_t shifted_fast(int32_t x, const ShiftDev &S) { return (int32_t)(((int64_t)x * S.mul + S.rnd) >> 32) >> S.sh; }
IPTQ_DEV int64_t shifted(int32_t x, const ShiftDev &S) { return ((int64_t)x * S.m + S.rnd) >> S.s; }

// clamp(rshr_round(x m, s) + zp, qmin, qmax)
template <bool FAST>
IPTQ_DEV int32_t code_of(int32_t x, const ShiftDev &S, const DyadicDev &P)
{
    if (FAST) return clamp_i32(shifted_fast(x, S) + P.zp, P.qmin, P.qmax);      // (|x m| < 2^46: 2^30 at most, and zp 2^24)
    int64_t v = shifted(x, S) + P.zp;
    v = v < P.qmin ? P.qmin : v > P.qmax ? P.qmax : v;
    return (int32_t)v;
}
IPTQ_DEV uint32_t four_bytes(const int32_t (&c)[4])
{
    const uint32_t a = __builtin_amdgcn_perm((uint32_t)c[1], (uint32_t)c[0], 0x0c0c0400u);
    return __builtin_amdgcn_perm((uint32_t)c[3], (uint32_t)c[2], 0x04000c0cu) | a;
}

// (f * acc) >> shift for 32 <= shift, the product below 2^63 in magnitude: the mean of the weighted values
IPTQ_DEV int32_t mean_of(uint64_t f, int64_t acc, int shift)
{
    const uint32_t fl = (uint32_t)f, fh = (uint32_t)(f >> 32), al = (uint32_t)acc, ah = (uint32_t)((uint64_t)acc >> 32);
    const uint32_t hi = __umulhi(fl, al) + fl * ah + fh * al;
    return (int32_t)hi >> (shift - 32);
}
// Four means of a query's outputs -> their bytes.
IPTQ_DEV uint32_t mean_bytes(uint64_t f, const int64_t (&acc)[4], int shift, const ShiftDev &S, const DyadicDev &P)
{
    int32_t c[4];
    if (S.s >= 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = code_of<true>(mean_of(f, acc[i], shift), S, P);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = code_of<false>(mean_of(f, acc[i], shift), S, P);
    }
    return four_bytes(c);
}

}  // namespace iptq
