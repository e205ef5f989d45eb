// The 4-bit key/value cache: what writes it.
//
// Bound by HBM: a row's head_dim bytes in, half as many out, keys and values.  A workgroup takes 16 tokens of one kv head, eight
// lanes and 16 channels each to a token's keys and to its values: rows come in whole lines, a group's step is a maximum over four
// lanes.  The keys' codes leave as they are; the values' change places in LDS, since the cache holds a channel pair's
// tokens side by side, and leave 16 tokens at a time where these have consecutive slots of a page (a
// prompt's), byte by byte where not (a decoding step's; each of these bytes is a line's transaction, so that they are better spread over many
// compute units).  16384 tokens of 8 heads of 128: 14.4 us (3.5 TB/s), 64 scattered ones 3.8 us with the call, 3.4 without; with 64 tokens
// and 512 threads a workgroup 15.4 and 6.2.
#include "block.h"

namespace iptq {

constexpr int kStoreTokens = 16;

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
    __shared__ __attribute__((aligned(16))) uint8_t codes[PAIRS][2 * kStoreTokens];
    const CacheDev &C = A.C;
    const uint32_t tile = div_by(blockIdx.x, A.by_kv_heads), h = blockIdx.x - tile * A.by_kv_heads.d;
    const int32_t first = (int32_t)tile * kStoreTokens;
    auto slot_of = [&](int t) {                           // -1: none
        const int32_t s = first + t < A.tokens ? A.slots[first + t] : -1;
        return s >= 0 && s < C.n_pages << C.page_log ? s : -1;
    };
    {
        const bool value = threadIdx.x >= 128;
        const int t = threadIdx.x >> 3 & (kStoreTokens - 1), unit = threadIdx.x & 7;
        const int32_t slot = slot_of(t);
        i32x4 x = {0, 0, 0, 0};
        if (first + t < A.tokens && unit < CHUNKS)
            x = *reinterpret_cast<const i32x4_any *>((value ? A.v : A.k) + (int64_t)(first + t) * (value ? A.v_stride : A.k_stride) + h * D + 16 * unit);
        int32_t step;
        const u32x2_t c = codes_of(x, &step);
        if (slot >= 0 && unit < CHUNKS) {
            const int64_t row = ((int64_t)(slot >> C.page_log) * C.kv_heads + h) * C.page_tokens + (slot & (C.page_tokens - 1));
            if (!value) *reinterpret_cast<u32x2_t *>(C.k_codes + row * PAIRS + 8 * unit) = c;
            if ((unit & 3) == 0) (value ? C.v_steps : C.k_steps)[row * G + (unit >> 2)] = (uint8_t)step;
        }
        if (value && unit < CHUNKS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) codes[8 * unit + i][t] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
        }
    }
    const int token = threadIdx.x & (kStoreTokens - 1);   // the values' way out: a lane a token
    const int32_t slot = slot_of(token), head = __shfl(slot, 0, kStoreTokens), in_page = head & (C.page_tokens - 1);
    const bool together = head >= 0 && in_page + kStoreTokens <= C.page_tokens && __all(slot == head + token);
    __syncthreads();
    const int64_t at = ((int64_t)(slot >> C.page_log) * C.kv_heads + h) * PAIRS * C.page_tokens + (slot & (C.page_tokens - 1));
    if (together) {                                       // the tokens of a channel pair at once
        if (threadIdx.x < PAIRS)
            *reinterpret_cast<u32x4_a1 *>(C.v_codes + (at - token) + (int64_t)threadIdx.x * C.page_tokens) = *reinterpret_cast<const u32x4 *>(codes[threadIdx.x]);
    } else if (slot >= 0) {
        for (int pair = threadIdx.x / kStoreTokens; pair < PAIRS; pair += 256 / kStoreTokens) C.v_codes[at + (int64_t)pair * C.page_tokens] = codes[pair][token];
    }
}

hipError_t cache_store_i4_dispatch(const CacheStoreCall &c, hipStream_t stream)
{
    const CacheStoreArgs a = {c.k, c.v, c.k_stride, c.v_stride, c.slots, (int32_t)c.tokens, div_of((uint32_t)c.C.kv_heads), c.C};
    auto kernel = c.C.dim == 32 ? cache_store_i4_kernel<32> : c.C.dim == 64 ? cache_store_i4_kernel<64>
                  : c.C.dim == 96 ? cache_store_i4_kernel<96> : cache_store_i4_kernel<128>;
    const uint32_t tiles = ((uint32_t)c.tokens + kStoreTokens - 1) / kStoreTokens;
    launch_kernel(kernel, dim3(tiles * (uint32_t)c.C.kv_heads), dim3(256), 0, stream, a);
    return take_launch_status();
}

}  // namespace iptq
