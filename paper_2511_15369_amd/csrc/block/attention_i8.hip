// Attention over packed prompts: the launches.
#include <algorithm>

#include "attention_i8.h"

namespace iptq {

hipError_t attention_i8_dispatch(const AttentionCall &c, hipStream_t stream)
{
    AttentionArgs a;
    a.q = c.q; a.k = c.k; a.v = c.v; a.out = c.out;
    a.q_stride = c.q_stride; a.k_stride = c.k_stride; a.v_stride = c.v_stride; a.out_stride = c.out_stride;
    a.q_offsets = c.q_offsets; a.k_offsets = c.k_offsets;
    a.q_tokens = (int32_t)c.q_tokens; a.k_tokens = (int32_t)c.k_tokens;
    a.q_len = (int32_t)(c.q_tokens / c.n_seq); a.k_len = (int32_t)(c.k_tokens / c.n_seq);
    a.max_q = c.max_q;
    a.by_kv_heads = div_of((uint32_t)c.kv_heads);
    a.by_group = div_of((uint32_t)(c.heads / c.kv_heads));
    a.by_seq = div_of((uint32_t)c.n_seq);
    a.P = c.P;
    a.post = narrow_post_of(c.P.post.m, c.P.post.s);
    // Workgroups of 128 queries, or of 32 with their keys divided over the wavefronts where the former do not reach every
    // compute unit: 197 tokens of 3 heads 6.0 us (128 queries: 9.5), 512 of 32 heads 20.1 (21.1), 4000 of 4 heads 55 (116), 8000 of 4
    // heads, 252 workgroups, 178 (229); from 256 on the other way, 900 of 32 heads 44 (32), 2000 129 (65), 64 images of 49 9.1 (6.0).
    const uint32_t pairs = (uint32_t)c.n_seq * (uint32_t)c.heads;
    a.tiles = ((uint32_t)c.max_q + kQueries - 1) / kQueries;
    const bool few = (int64_t)a.tiles * pairs < 256;
    if (few) a.tiles = ((uint32_t)c.max_q + 31) / 32;
    const uint32_t wgs = a.tiles * pairs;                 // below 2^31: checked
    for (a.first_wg = 0; a.first_wg < wgs; a.first_wg += kLaunchMost) {
        const uint32_t grid = std::min(wgs - a.first_wg, kLaunchMost);
        hipError_t e;
        switch (c.dim) {
        case 32: e = attention_i8_launch_32(a, few, grid, stream); break;
        case 64: e = attention_i8_launch_64(a, few, grid, stream); break;
        case 96: e = attention_i8_launch_96(a, few, grid, stream); break;
        default: e = attention_i8_launch_128(a, few, grid, stream);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace iptq
