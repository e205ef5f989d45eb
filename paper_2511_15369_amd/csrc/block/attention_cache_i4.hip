// Attention over the 4-bit cache: how the keys are divided, the launches, and the last one, which adds up the splits.
#include <algorithm>

#include "attention_cache_i4.h"

namespace iptq {

// The sums of the splits and a column's outputs: 16 threads of eight channels each, PARTS of these over the splits (4: a wavefront per
// column; 16: a workgroup).  A split without keys has written nothing: what is read there is not added, but read all the
// same, so that the loads of several splits are under way together.
template <int PARTS>
__global__ __launch_bounds__(256) void attention_cache_i4_join_kernel(const CacheAttentionArgs A)
{
    const uint32_t number = PARTS == 4 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
    if (number >= A.all_columns) return;
    const uint32_t pair = div_by(number, A.by_columns), column = number - pair * A.by_columns.d;
    const uint32_t seq = div_by(pair, A.by_kv_heads), kvh = pair - seq * A.by_kv_heads.d;
    const int dim = A.C.dim, unit = threadIdx.x & 15, part = threadIdx.x >> 4 & (PARTS - 1);
    const int32_t length = length_of(A, seq), split_keys = wave_keys_of(A, length) * A.key_waves;
    int64_t v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    uint32_t s = 0;
    if (8 * unit < dim) {
#pragma unroll 4
        for (int32_t i = part; i < A.splits; i += PARTS) {
            const int64_t at = ((int64_t)pair * A.splits + i) * A.columns + column;
            const i32x4 *o = reinterpret_cast<const i32x4 *>(A.partial + at * dim + 8 * unit);
            const i32x4 a = o[0], b = o[1];
            const uint32_t t = A.sums[at];
            const bool some = i * split_keys < length;
#pragma unroll
            for (int j = 0; j < 4; ++j) { v[j] += some ? a[j] : 0; v[4 + j] += some ? b[j] : 0; }
            s += some ? t : 0;
        }
    }
#pragma unroll
    for (int m = 16; m < 64; m <<= 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += __shfl_xor((long long)v[j], m);
        s += (uint32_t)__shfl_xor((int32_t)s, m);
    }
    if (PARTS == 16) {
        __shared__ int64_t parts[4][16][8];
        __shared__ uint32_t totals[4];
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) < 16) {
#pragma unroll
            for (int j = 0; j < 8; ++j) parts[wave][unit][j] = v[j];
            if (unit == 0) totals[wave] = s;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = parts[0][unit][j] + parts[1][unit][j] + parts[2][unit][j] + parts[3][unit][j];
        s = totals[0] + totals[1] + totals[2] + totals[3];
    }
    if (part != 0 || 8 * unit >= dim) return;
    const uint64_t f = floor_div_scaled(1, 54, s);
    const uint32_t token = div_by(column, A.by_group), head = kvh * (uint32_t)A.group + (column - token * (uint32_t)A.group);
    store_means(A.out + ((int64_t)seq * A.q_tokens + token) * A.out_stride + head * dim + 8 * unit, f, v, A.P);
}

struct CachePlan {
    int halves, chunks;               // weights' halves side by side; workgroups over the columns
    bool whole;                       // one workgroup has all keys
    int key_waves, splits, tiles;
    size_t lds;
    int64_t pairs, deltas, refs, tops, partial, sums;      // workspace bytes
};

static int64_t up_to(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

static CachePlan plan_of(const CacheAttentionCall &c)
{
    CachePlan p;
    const int columns = c.heads / c.C.kv_heads * c.q_tokens;
    p.halves = columns <= 8 ? 2 : 1;
    const int queries = 16 / p.halves;
    p.chunks = (columns + queries - 1) / queries;
    p.pairs = (int64_t)c.n_seq * c.C.kv_heads;
    const int64_t keys = (int64_t)c.max_pages * c.C.page_tokens;           // at most
    p.tiles = (int)((keys + kTile - 1) / kTile);
    // Up to 1024 keys: a tile a wavefront, up to sixteen of these, and all of a sequence's scores in registers: one launch (64 sequences of
    // 1000 tokens, 32 heads on 8, 21.8 us, in two phases 34.8; one of 500 6.0 and 11.9).
    p.whole = keys <= 1024 && p.pairs * p.chunks <= (int64_t)kLaunchMost;
    p.key_waves = p.whole ? std::max(p.tiles, 1) : 4;
    p.splits = 1;
    if (!p.whole) {
        // A wavefront has 64 to 1024 keys.  Up to eight queries: twice as many workgroups as the chip holds, for the sake of sequences of
        // different lengths (64 of 200 to 8192 tokens 75 us, with half as many workgroups 80; of equal lengths the other way: 64 of 4000 72 to 76
        // and 69).  More queries: once, as each split writes and reads a sum per column and channel (two of 65536 tokens, 32 columns, 76 and 93).
        const int64_t most = (keys + kTile * p.key_waves - 1) / (kTile * p.key_waves), least = (keys + 1024 * p.key_waves - 1) / (1024 * p.key_waves);
        const int64_t wanted = (columns > 8 ? 1024 : 2048) / (p.pairs * p.chunks);
        p.splits = (int)std::min<int64_t>(std::max(std::max<int64_t>(wanted, least), (int64_t)1), std::min<int64_t>(most, 128));
    }
    const size_t blocks = c.C.dim / 32, stage = std::max(blocks * 4 * 288, (size_t)kTile * c.C.dim / 2 + 256);       // CacheAttention::STAGE
    p.lds = (size_t)p.key_waves * stage + (size_t)(32 + c.C.dim / 32 * 512) * 4;
    const int64_t rows = p.whole ? 0 : p.pairs * columns;
    p.deltas = rows * p.tiles * kTile * 2;
    p.refs = up_to(rows * p.tiles * 4, 16);
    p.tops = up_to(rows * p.splits * 4, 16);
    p.partial = rows * p.splits * c.C.dim * 4;
    p.sums = up_to(rows * p.splits * 4, 16);
    return p;
}

int64_t attention_cache_i4_workspace_bytes(const CacheAttentionCall &c)
{
    if (c.n_seq == 0) return 0;
    const CachePlan p = plan_of(c);
    return p.deltas + p.refs + p.tops + p.partial + p.sums;
}

static hipError_t launch(const CacheAttentionArgs &a, int halves, int phases, uint32_t grid, uint32_t block, size_t lds, hipStream_t stream)
{
    switch (a.C.dim) {
    case 32: return attention_cache_i4_launch_32(a, halves, phases, grid, block, lds, stream);
    case 64: return attention_cache_i4_launch_64(a, halves, phases, grid, block, lds, stream);
    case 96: return attention_cache_i4_launch_96(a, halves, phases, grid, block, lds, stream);
    default: return attention_cache_i4_launch_128(a, halves, phases, grid, block, lds, stream);
    }
}

hipError_t attention_cache_i4_dispatch(const CacheAttentionCall &c, hipStream_t stream)
{
    const CachePlan p = plan_of(c);
    CacheAttentionArgs a;
    a.q = c.q; a.out = c.out; a.q_stride = c.q_stride; a.out_stride = c.out_stride;
    a.pages = c.pages; a.lengths = c.lengths; a.max_pages = c.max_pages; a.q_tokens = c.q_tokens;
    a.group = c.heads / c.C.kv_heads;
    a.columns = a.group * c.q_tokens;
    a.by_group = div_of((uint32_t)a.group);
    a.by_kv_heads = div_of((uint32_t)c.C.kv_heads);
    a.by_chunks = div_of((uint32_t)p.chunks);
    a.by_splits = div_of((uint32_t)p.splits);
    a.by_span = div_of((uint32_t)(kTile * p.key_waves * p.splits));
    a.by_columns = div_of((uint32_t)a.columns);
    a.all_columns = (uint32_t)(p.pairs * a.columns);
    a.key_waves = p.key_waves;
    a.splits = p.splits; a.tiles = p.tiles;
    char *w = static_cast<char *>(c.work);
    a.deltas = reinterpret_cast<int16_t *>(w); w += p.deltas;
    a.partial = reinterpret_cast<int32_t *>(w); w += p.partial;
    a.refs = reinterpret_cast<int32_t *>(w); w += p.refs;
    a.tops = reinterpret_cast<int32_t *>(w); w += p.tops;
    a.sums = reinterpret_cast<uint32_t *>(w);
    a.C = c.C; a.P = c.P;
    const uint32_t grid = (uint32_t)(p.pairs * p.chunks * p.splits);
    const uint32_t block = 64u * p.key_waves;
    if (p.whole) return launch(a, p.halves, 3, grid, block, p.lds, stream);
    hipError_t e = launch(a, p.halves, 1, grid, block, p.lds, stream);
    if (e != hipSuccess) return e;
    e = launch(a, p.halves, 2, grid, block, p.lds, stream);
    if (e != hipSuccess) return e;
    // (4 splits, 64 sequences of 4000 tokens, 69 to 72 us, in the other form 74 to 76; 16 splits, 16 of 3000, 19.1 and 17.5; 128, one of 131072, 52 and 48)
    if (p.splits <= 8) launch_kernel(attention_cache_i4_join_kernel<4>, dim3((a.all_columns + 3) / 4), dim3(256), 0, stream, a);
    else launch_kernel(attention_cache_i4_join_kernel<16>, dim3(a.all_columns), dim3(256), 0, stream, a);
    return take_launch_status();
}

}  // namespace iptq
