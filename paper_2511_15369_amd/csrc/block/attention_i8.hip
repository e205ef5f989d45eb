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
    a.by_seq = div_of((uint32_t)c.n_seq);
    a.P = c.P;
    a.post = narrow_post_of(c.P.post.m, c.P.post.s);
    // Workgroups of 128 queries, or of 32 with their keys divided over eight wavefronts.  In time of a block of 32 keys on a wavefront, with K blocks
    // to a row and R workgroups of 32 queries to a compute unit: the latter take R (K / 4 + F), the former K + F while they find a compute
    // unit each, F = 7.5 for the rest of a workgroup's life.  Causal rows are half as long on average, which only many short workgroups
    // make use of: R (K / 8 + F).  So 32 queries where R is at most 1, or K (4 - R) > 4 F (R - 1), 8 in place of 4 for causal rows.
    // Measured, us, 32 queries and 128: 197 tokens of 3 heads of 64 5.5 and 9.6, 512 of 32 heads of 128 16.9 and 21.3, 640 24.0 and 24.6, 900 38 and
    // 33, 1500 74 and 51; 4000 of 8 heads 97 and 119, 8000 of 4 166 and 230, 16000 of 4 597 and 471; 8 sequences of 197, 12 heads of 64, 12.2 and
    // 9.7, 32 of 49, 8 heads of 32, 5.1 and 4.8, 8 of 100, 32 heads of 128, 21 and 10.
    const uint32_t pairs = (uint32_t)c.n_seq * (uint32_t)c.heads;
    const int64_t keys = std::max<int64_t>(c.max_q, c.k_tokens / c.n_seq), blocks = (keys + 31) / 32, spread = c.P.causal ? 8 : 4;
    const int64_t of_32 = ((int64_t)c.max_q + 31) / 32 * pairs;
    const bool few = of_32 <= 256 || 2 * blocks * (256 * spread - of_32) > 15 * spread * (of_32 - 256);
    // The wavefronts of the others take 32 queries of four heads, or 64 of two, where a group of heads has them: all read the same keys, and
    // rows of like length leave none waiting for another and fewer places empty behind a sequence's last row.  That counts
    // where there are more workgroups than the chip holds at once, two to a compute unit, or no second 128 queries: us, four heads and one, 64
    // sequences of 200, 32 heads on 8 of 128, 85 and 106, 4 of 700 36 and 41, one of 3000 110 and 117, 64 of 49, 8 heads of 32, 5.0 and 5.9; one of
    // 2000, 512 workgroups, 66.4 and 66.1, of 900 36.3 and 33.5, 4 of 300 16.7 and 15.0, where fewer wavefronts do all the work at once.
    const uint32_t group = (uint32_t)(c.heads / c.kv_heads);
    const bool shared = !few && (c.max_q <= kQueries || ((int64_t)c.max_q + kQueries - 1) / kQueries * pairs > 512);
    a.together = !shared ? 0 : group % 4 == 0 ? 2 : group % 2 == 0 ? 1 : 0;
    a.by_group = div_of(group >> a.together);
    const uint32_t queries = few ? 32 : kQueries >> a.together;
    a.tiles = ((uint32_t)c.max_q + queries - 1) / queries;
    const uint32_t wgs = a.tiles * (pairs >> a.together); // below 2^31: checked
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
