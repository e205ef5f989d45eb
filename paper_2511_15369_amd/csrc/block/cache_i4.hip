// The 4-bit key/value cache: what writes it, and the attention of single tokens over it.
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

// ---- attention ----------------------------------------------------------------------------------
// Columns are the queries that share a kv head: e = token * group + head of the group; 16 of them make the narrow
// side of v_mfma_i32_16x16x64_i8.  Keys go by 64, in blocks of 16 that never cross a page.  Scores are
// transposed, keys x columns: lane (column l % 16, p = l / 16) holds rows 4 p + r of each of the four products,
// which read their keys in the order kappa(s, 4 p + r) = 16 p + 4 s + r, so that its 16 scores are the keys
// 16 p .. 16 p + 15 of the tile, one block, and its 16 weights the right operand of the second product.
//
// Codes go into the products as 16 c, the nibble in the byte's upper half: no sign extension, and exact,
// the factor 16 leaves with a shift (x) or a division without remainder (values).
struct CacheAttentionArgs {
    const int8_t *q;
    int8_t *out;
    int64_t q_stride, out_stride;
    const int32_t *pages, *lengths;
    int32_t max_pages, q_tokens, group, columns;      // columns = group * q_tokens
    DivDev by_group, by_tiles, by_kv_heads;
    CacheDev C;
    AttentionDev P;
};

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

typedef i32x4 __attribute__((aligned(1))) i32x4_any;

template <int D, int VARIANT>
__global__ __launch_bounds__(256) void attention_cache_i4_kernel(const CacheAttentionArgs A)
{
    constexpr int GROUPS = (D + kGroup - 1) / kGroup, PAIRS = D / 2, BLOCKS = D / 32;      // blocks of 16 channel pairs
    __shared__ int32_t tops[4][16];
    __shared__ uint32_t sums[4][16];
    __shared__ int32_t parts[4][BLOCKS * 2 * 4 * 64];

    const CacheDev &C = A.C;
    const uint32_t wg = blockIdx.x;
    const uint32_t r1 = div_by(wg, A.by_kv_heads), kvh = wg - r1 * A.by_kv_heads.d;
    const uint32_t seq = div_by(r1, A.by_tiles), e0 = (r1 - seq * A.by_tiles.d) * 16;
    const int lane = threadIdx.x & 63, col = lane & 15, p = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const int32_t capacity = A.max_pages << C.page_log;
    const int32_t length = min(max(A.lengths[seq], 0), capacity);
    const uint32_t e = min(e0 + col, (uint32_t)A.columns - 1);           // columns past the last repeat it
    const uint32_t token = div_by(e, A.by_group), head = kvh * (uint32_t)A.group + (e - token * (uint32_t)A.group);
    const int64_t q_row = (int64_t)seq * A.q_tokens + token;
    const int32_t limit = A.P.causal ? length - (A.q_tokens - 1 - (int32_t)token) : length;

    i32x4 qf[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        qf[g] = (i32x4){0, 0, 0, 0};
        if (kGroup * g + 16 * p < D)
            qf[g] = in_nibble_order(*reinterpret_cast<const i32x4_any *>(A.q + q_row * A.q_stride + head * D + kGroup * g + 16 * p));
    }
    const int32_t *table = A.pages + (int64_t)seq * A.max_pages;
    auto page_of = [&](int32_t key) { return page_of_key(table, C.page_log, C.n_pages, key, length); };
    // transposed scores of keys [at, at + 64): x[4 s + r] of key at + 16 p + 4 s + r, times 16
    auto scores = [&](int32_t at, int32_t (&x)[16]) {
        const int32_t mine = at + 16 * p, page = page_of(mine);                       // the block of the lane's scores
        const int32_t theirs = at + 16 * (col >> 2), key_page = max(page_of(theirs), 0);    // the block whose keys it loads
        const int64_t head_at = (int64_t)key_page * C.kv_heads + kvh;
        const int64_t key_row = head_at * C.page_tokens + (theirs & (C.page_tokens - 1)) + (col & 3);
        const int64_t step_row = ((int64_t)max(page, 0) * C.kv_heads + kvh) * C.page_tokens + (mine & (C.page_tokens - 1));
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int r = 0; r < 4; ++r) x[4 * s + r] = 0;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                u32x2_t codes = {0, 0};
                if (kGroup * g + 16 * p < D)
                    codes = *reinterpret_cast<const u32x2_t *>(C.k_codes + (key_row + 4 * s) * PAIRS + kGroup / 2 * g + 8 * p);
                const i32x4 y = __builtin_amdgcn_mfma_i32_16x16x64_i8(upper_nibbles(codes), qf[g], (i32x4){0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) x[4 * s + r] += __mul24((int32_t)C.k_steps[(step_row + 4 * s + r) * GROUPS + g], y[r]);
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = page >= 0 && mine + i < limit ? x[i] : kI32Min;
        return page;
    };

    int32_t top = kI32Min;
    for (int32_t at = 64 * wave; at < length; at += 256) {
        int32_t x[16];
        scores(at, x);
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, x[i]);
    }
    top = max(top, __shfl_xor(top, 16));
    top = max(top, __shfl_xor(top, 32));
    if (p == 0) tops[wave][col] = top;
    __syncthreads();
    top = max(max(tops[0][col], tops[1][col]), max(tops[2][col], tops[3][col]));
    // scores are 16 times their value: one shift more
    const int32_t shift = A.P.shift + 4, rounding = A.P.shift > 0 ? 1 << (shift - 1) : 0;
    const int32_t base = top == kI32Min ? 0 : rounding - (((top + rounding) >> shift) << shift);

    i32x4 acc[BLOCKS][2][2];                              // channel pairs of 16, low / high nibble, upper / lower half
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[b][n >> 1][n & 1] = (i32x4){0, 0, 0, 0};
    uint32_t sum = 0;
    const i16x2 least = {(short)-A.P.d_clamp, (short)-A.P.d_clamp};
    for (int32_t at = 64 * wave; at < length; at += 256) {
        int32_t x[16];
        const int32_t page = scores(at, x), mine = at + 16 * p;
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // masked scores stay far below every other one
            const int32_t a = x[2 * i] == kI32Min ? kI32Min : (x[2 * i] + base) >> shift;
            const int32_t b = x[2 * i + 1] == kI32Min ? kI32Min : (x[2 * i + 1] + base) >> shift;
            const i16x2 d = __builtin_elementwise_max(__builtin_bit_cast(i16x2, __builtin_amdgcn_cvt_pk_i16(a, b)), least);
            w[i] = weights_of_pair<VARIANT>(d, A.P);
            sum = __builtin_amdgcn_udot2(__builtin_bit_cast(u16x2_t, w[i]), (u16x2_t){1, 1}, sum, false);
        }
        const int64_t head_at = (int64_t)max(page, 0) * C.kv_heads + kvh;
        const int32_t pos = mine & (C.page_tokens - 1);
        i32x4 hi[GROUPS], lo[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t u[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint8_t *steps = C.v_steps + (head_at * C.page_tokens + pos + 4 * i + 2 * j) * GROUPS + g;
                    const uint32_t ww = w[2 * i + j];
                    u[j] = ((ww & 0xffff) * steps[0] + 64) >> 7 | (((ww >> 16) * steps[GROUPS] + 64) >> 7) << 16;
                }
                uint32_t h, l;
                split_weights(u[0], u[1], &h, &l);
                hi[g][i] = (int32_t)h;
                lo[g][i] = (int32_t)l;
            }
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(C.v_codes + (head_at * PAIRS + 16 * b + col) * C.page_tokens + pos);
            const int g = 32 * b / kGroup;
            const i32x4 even = __builtin_bit_cast(i32x4, v << 4 & 0xf0f0f0f0u), odd = __builtin_bit_cast(i32x4, v & 0xf0f0f0f0u);
            acc[b][0][0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(even, hi[g], acc[b][0][0], 0, 0, 0);
            acc[b][0][1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(even, lo[g], acc[b][0][1], 0, 0, 0);
            acc[b][1][0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(odd, hi[g], acc[b][1][0], 0, 0, 0);
            acc[b][1][1] = __builtin_amdgcn_mfma_i32_16x16x64_i8(odd, lo[g], acc[b][1][1], 0, 0, 0);
        }
    }
    sum += (uint32_t)__shfl_xor((int32_t)sum, 16);
    sum += (uint32_t)__shfl_xor((int32_t)sum, 32);
    if (p == 0) sums[wave][col] = sum;
    // the four wavefronts' sums of the upper halves, then of the lower: wavefront w adds up blocks w, w + 4, ...
    int32_t total[2][(BLOCKS + 3) / 4][2][4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (half) __syncthreads();
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) parts[wave][((b * 2 + n) * 4 + r) * 64 + lane] = acc[b][n][half][r];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < (BLOCKS + 3) / 4; ++j)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = ((min(wave + 4 * j, BLOCKS - 1) * 2 + n) * 4 + r) * 64 + lane;
                    total[half][j][n][r] = parts[0][at] + parts[1][at] + parts[2][at] + parts[3][at];
                }
    }
    const uint64_t f = floor_div_u64((uint64_t)1 << 54, sums[0][col] + sums[1][col] + sums[2][col] + sums[3][col]);
    if (e0 + col >= (uint32_t)A.columns) return;
    // rows 4 p + r of block b are the channel pairs 16 b + 4 p + r; every sum is a multiple of 16
#pragma unroll
    for (int j = 0; j < (BLOCKS + 3) / 4; ++j) {
        const int b = wave + 4 * j;
        if (b >= BLOCKS) break;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int64_t t = (int64_t)total[0][j][n][r] * 16 + (total[1][j][n][r] >> 4);
                A.out[q_row * A.out_stride + head * D + 2 * (16 * b + 4 * p + r) + n] = (int8_t)mean_byte(f, t, 39, A.P.post);
            }
    }
}

int64_t attention_cache_i4_workspace_bytes(const CacheAttentionCall &) { return 0; }

template <int D>
static void launch_of(const CacheAttentionArgs &a, uint32_t grid, hipStream_t stream)
{
    auto kernel = a.P.variant == 0 ? attention_cache_i4_kernel<D, 0> : a.P.variant == 1 ? attention_cache_i4_kernel<D, 1>
                                                                                       : attention_cache_i4_kernel<D, 2>;
    launch_kernel(kernel, dim3(grid), dim3(256), 0, stream, a);
}

hipError_t attention_cache_i4_dispatch(const CacheAttentionCall &c, hipStream_t stream)
{
    CacheAttentionArgs a;
    a.q = c.q; a.out = c.out; a.q_stride = c.q_stride; a.out_stride = c.out_stride;
    a.pages = c.pages; a.lengths = c.lengths; a.max_pages = c.max_pages; a.q_tokens = c.q_tokens;
    a.group = c.heads / c.C.kv_heads;
    a.columns = a.group * c.q_tokens;
    const uint32_t tiles = ((uint32_t)a.columns + 15) / 16;
    a.by_group = div_of((uint32_t)a.group);
    a.by_tiles = div_of(tiles);
    a.by_kv_heads = div_of((uint32_t)c.C.kv_heads);
    a.C = c.C; a.P = c.P;
    const uint32_t grid = (uint32_t)c.n_seq * tiles * (uint32_t)c.C.kv_heads;
    switch (c.C.dim) {
    case 32: launch_of<32>(a, grid, stream); break;
    case 64: launch_of<64>(a, grid, stream); break;
    case 96: launch_of<96>(a, grid, stream); break;
    default: launch_of<128>(a, grid, stream);
    }
    return take_launch_status();
}

}  // namespace iptq
