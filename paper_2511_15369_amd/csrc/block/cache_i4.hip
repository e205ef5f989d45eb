// The 4-bit key/value cache: what writes it.
//
// Bound by HBM: a row's head_dim bytes in, half as many out, keys and values.  A workgroup takes 64 tokens of one kv head, eight
// lanes and 16 channels each to a token: rows come in whole lines, a group's step is a maximum over four lanes.  The
// keys' codes leave as they are; the values' change places in LDS, since the cache holds a channel pair's
// tokens side by side, and leave 16 tokens at a time where these have consecutive slots of a page (a
// prompt's), byte by byte where not (a decoding step's).
#include "block.h"

namespace iptq {

constexpr int kStoreTokens = 64;

struct CacheStoreArgs {
    const int8_t *k, *v;
    int64_t k_stride, v_stride;
    const int32_t *slots;
    int32_t tokens;
    DivDev by_kv_heads;
    CacheDev C;
};

typedef i32x4 __attribute__((aligned(1))) i32x4_any;

// 16 codes of a lane's channels, two a byte, and the step of the channels' group (which four lanes share).
// c = sign(x) floor((14 |x| + a) / (2 a)) = (x R + 2^15, less 1 for a negative x) >> 16 with R = ceil(7 2^16 / a): |x| (R - 7 2^16 / a) < 2^7 is
// less than half of 2^16 / a, the distance of the quotients, and ties go away from zero.
IPTQ_DEV u32x2_t codes_of(const i32x4 &x, int32_t *step)
{
    int32_t most = 0, least = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int32_t b = (int8_t)(x[i >> 2] >> (8 * (i & 3)));
        most = max(most, b);
        least = min(least, b);
    }
    const int32_t a = group_max_i32<4>(max(most, -least));
    uint32_t r = (7u * floor_pow2_div(24, (uint32_t)a)) >> 8;
    r += r * (uint32_t)a < 7u << 16 ? 1 : 0;
    r += r * (uint32_t)a < 7u << 16 ? 1 : 0;
    *step = a;
    u32x2_t out = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int32_t t = __mul24((int8_t)(x[i >> 2] >> (8 * (i & 3))), (int32_t)r);
        const uint32_t c = (uint32_t)(t + (t >> 31) + 32768) >> 16 & 15u;
        out[i >> 3] |= c << (4 * (i & 7));
    }
    return out;
}

template <int D>
__global__ __launch_bounds__(256) void cache_store_i4_kernel(const CacheStoreArgs A)
{
    constexpr int CHUNKS = D / 16, G = (D + kGroup - 1) / kGroup, PAIRS = D / 2;
    __shared__ __attribute__((aligned(16))) uint8_t codes[PAIRS][kStoreTokens + 16];
    __shared__ int32_t slots[kStoreTokens];
    const CacheDev &C = A.C;
    const uint32_t tile = div_by(blockIdx.x, A.by_kv_heads), h = blockIdx.x - tile * A.by_kv_heads.d;
    const int32_t first = (int32_t)tile * kStoreTokens, unit = threadIdx.x & 7;

    i32x4 x[2][2];
    int32_t slot[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {                         // two tokens a thread
        const int32_t token = first + 32 * j + (threadIdx.x >> 3);
        slot[j] = token < A.tokens ? A.slots[token] : -1;
        x[0][j] = x[1][j] = (i32x4){0, 0, 0, 0};
        if (token < A.tokens && unit < CHUNKS) {
            x[0][j] = *reinterpret_cast<const i32x4_any *>(A.k + token * A.k_stride + h * D + 16 * unit);
            x[1][j] = *reinterpret_cast<const i32x4_any *>(A.v + token * A.v_stride + h * D + 16 * unit);
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if (slot[j] < 0 || slot[j] >= C.n_pages << C.page_log) slot[j] = -1;
        const int t = 32 * j + (threadIdx.x >> 3);
        if (unit == 0) slots[t] = slot[j];
        const int64_t row = ((int64_t)(slot[j] >> C.page_log) * C.kv_heads + h) * C.page_tokens + (slot[j] & (C.page_tokens - 1));
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            int32_t step;
            const u32x2_t c = codes_of(x[which][j], &step);
            if (slot[j] >= 0 && unit < CHUNKS) {
                if (which == 0) *reinterpret_cast<u32x2_t *>(C.k_codes + row * PAIRS + 8 * unit) = c;
                if ((unit & 3) == 0) (which ? C.v_steps : C.k_steps)[row * G + (unit >> 2)] = (uint8_t)step;
            }
            if (which == 1 && unit < CHUNKS) {
#pragma unroll
                for (int i = 0; i < 8; ++i) codes[8 * unit + i][t] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
            }
        }
    }
    __syncthreads();
    // values: 16 tokens of a channel pair at a time
    for (int u = threadIdx.x; u < PAIRS * (kStoreTokens / 16); u += 256) {
        const int pair = u >> 2, t = 16 * (u & 3);
        const int32_t s = slots[t];
        bool together = s >= 0 && (s & (C.page_tokens - 1)) + 15 < C.page_tokens;
#pragma unroll
        for (int i = 1; i < 16; ++i) together = together && slots[t + i] == s + i;
        if (together) {
            const int64_t at = (((int64_t)(s >> C.page_log) * C.kv_heads + h) * PAIRS + pair) * C.page_tokens + (s & (C.page_tokens - 1));
            *reinterpret_cast<u32x4_a1 *>(C.v_codes + at) = *reinterpret_cast<const u32x4 *>(&codes[pair][t]);
        } else {
            for (int i = 0; i < 16; ++i) {
                const int32_t w = slots[t + i];
                if (w >= 0)
                    C.v_codes[(((int64_t)(w >> C.page_log) * C.kv_heads + h) * PAIRS + pair) * C.page_tokens + (w & (C.page_tokens - 1))] = codes[pair][t + i];
            }
        }
    }
}

hipError_t cache_store_i4_dispatch(const CacheStoreCall &c, hipStream_t stream)
{
    CacheStoreArgs a = {c.k, c.v, c.k_stride, c.v_stride, c.slots, (int32_t)c.tokens, div_of((uint32_t)c.C.kv_heads), c.C};
    const int64_t tiles = (c.tokens + kStoreTokens - 1) / kStoreTokens;
    auto kernel = c.C.dim == 32 ? cache_store_i4_kernel<32> : c.C.dim == 64 ? cache_store_i4_kernel<64>
                  : c.C.dim == 96 ? cache_store_i4_kernel<96> : cache_store_i4_kernel<128>;
    launch_kernel(kernel, dim3((uint32_t)(tiles * c.C.kv_heads)), dim3(256), 0, stream, a);
    return take_launch_status();
}

}  // namespace iptq
