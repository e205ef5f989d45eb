// The 4-bit key/value cache: what writes it.
#include "block.h"

namespace iptq {

struct CacheStoreArgs {
    const int8_t *k, *v;
    int64_t k_stride, v_stride;
    const int32_t *slots;
    CacheDev C;
};

// One token of one kv head per wavefront: the steps of its groups, then its codes.
__global__ __launch_bounds__(64) void cache_store_i4_kernel(const CacheStoreArgs A)
{
    const CacheDev &C = A.C;
    const int64_t token = blockIdx.x;
    const int32_t slot = A.slots[token];
    if (slot < 0 || slot >= C.n_pages << C.page_log) return;
    const int32_t page = slot >> C.page_log, pos = slot & (C.page_tokens - 1);
    const int groups = (C.dim + kGroup - 1) / kGroup, lane = threadIdx.x;
    for (int h = 0; h < C.kv_heads; ++h) {
        const int64_t head = (int64_t)page * C.kv_heads + h;
        for (int which = 0; which < 2; ++which) {
            const int8_t *src = which ? A.v + token * A.v_stride + (int64_t)h * C.dim : A.k + token * A.k_stride + (int64_t)h * C.dim;
            const bool live = 2 * lane < C.dim;            // channels 2 lane, 2 lane + 1; a group is 32 lanes
            const int32_t a = live ? src[2 * lane] : 0, b = live ? src[2 * lane + 1] : 0;
            const int32_t pa = a < 0 ? -a : a, pb = b < 0 ? -b : b;
            int32_t most = max(pa, pb);
            for (int d = 1; d < 32; d <<= 1) most = max(most, __shfl_xor(most, d));
            const int32_t ca = (int32_t)floor_div_u64((uint64_t)(14 * pa + most), 2u * (uint32_t)most);
            const int32_t cb = (int32_t)floor_div_u64((uint64_t)(14 * pb + most), 2u * (uint32_t)most);
            const uint8_t code = (uint8_t)(((a < 0 ? -ca : ca) & 15) | ((b < 0 ? -cb : cb) & 15) << 4);
            if (live) {
                if (which) C.v_codes[(head * (C.dim / 2) + lane) * C.page_tokens + pos] = code;
                else C.k_codes[(head * C.page_tokens + pos) * (C.dim / 2) + lane] = code;
            }
            if ((lane & 31) == 0 && lane / 32 < groups)
                (which ? C.v_steps : C.k_steps)[(head * C.page_tokens + pos) * groups + lane / 32] = (uint8_t)most;
        }
    }
}

hipError_t cache_store_i4_dispatch(const CacheStoreCall &c, hipStream_t stream)
{
    const CacheStoreArgs a = {c.k, c.v, c.k_stride, c.v_stride, c.slots, c.C};
    launch_kernel(cache_store_i4_kernel, dim3((uint32_t)c.tokens), dim3(64), 0, stream, a);
    return take_launch_status();
}

}  // namespace iptq
