// Root-mean-square norm with the residual's addition, and requantization by row scales.
//
// Both are bound by HBM: 13 bytes per value of the norm (product, residual, its new value, code), 5 of the requantization.
// 8192 rows of 5120 take 97 us (5.6 TB/s), 8192 of 6144 requantized 40.5 us (6.2 TB/s); 64 rows of either, 4.4 and 3.8 us, are the call.
// A row stays in the registers of the wavefronts that hold it, so every byte crosses once.  Rows are read in chunks of four
// values at their natural alignment; where four does not divide a row its last chunk ends with it and starts
// earlier, and the values it shares with the chunk before count once.
#include <algorithm>

#include "block.h"

namespace iptq {

constexpr int32_t kResidualMost = (1 << 23) - 1;

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef i16x4 __attribute__((aligned(2))) i16x4_a2;

struct RmsnormArgs {
    const int32_t *x, *residual;
    int32_t *residual_out;
    const int16_t *gain;
    int8_t *out;
    int32_t *row_scales;
    int32_t rows, cols;
    int64_t eps_sum;
    uint32_t root_cols;
    ShiftDev in, post;
    DyadicDev p;
};

// The factor of a row from its sum of squares, and the shift that goes with it: z = rshr_round(r c, 41 - t).
IPTQ_DEV uint32_t row_factor(uint64_t total, uint32_t root_cols, int *t)
{
    *t = 0;
    if (total == 0) return 0;
    const uint32_t top = (uint32_t)(total >> 32);
    const int bits = top != 0 ? 64 - clz_u32(top) : 32 - clz_u32((uint32_t)total);
    *t = (62 - bits) >> 1;
    const uint32_t inverse = floor_div_2_61(root_u62(total << (2 * *t)));
    return (uint32_t)(((uint64_t)root_cols * inverse) >> 24);
}
IPTQ_DEV uint64_t at_most_62_bits(uint64_t v) { return v >= ((uint64_t)1 << 62) ? ((uint64_t)1 << 62) - 1 : v; }

// WAVES wavefronts per row (1: four rows a workgroup, no barrier), CHUNKS chunks of four values per lane.
// FAST: both steps' shifts are 16 and more.
template <int WAVES, int CHUNKS, bool FAST>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void rmsnorm_i32_kernel(const RmsnormArgs A)
{
    constexpr int T = 64 * WAVES;
    __shared__ uint32_t parts[2][WAVES];
    __shared__ uint32_t tops[WAVES];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int tid = WAVES == 1 ? lane : threadIdx.x;
    const int64_t row = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (WAVES == 1 && row >= A.rows) return;
    const int64_t at = row * A.cols;
    const int cols = A.cols;

    int start[CHUNKS];
    bool mine[CHUNKS];
    i32x4 r[CHUNKS], add[CHUNKS];
    i16x4 g[CHUNKS];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int c = 4 * (tid + T * i);
        mine[i] = c < cols;
        start[i] = min(c, cols - 4);                      // (lanes past the row read its last chunk)
        r[i] = A.x ? load_i32x4(A.x + at + start[i]) : (i32x4){0, 0, 0, 0};
        add[i] = A.residual ? load_i32x4(A.residual + at + start[i]) : (i32x4){0, 0, 0, 0};
        g[i] = *reinterpret_cast<const i16x4_a2 *>(A.gain + start[i]);
    }
    uint64_t ss = 0;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int skip = mine[i] ? 4 * (tid + T * i) - start[i] : 4;      // values that the chunk before has counted
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            int32_t v;
            if (FAST) {
                v = sat_add_i32(A.x ? shifted_fast(r[i][e], A.in) : 0, add[i][e]);
                v = clamp_i32(v, -kResidualMost, kResidualMost);
            } else {
                int64_t w = (A.x ? shifted(r[i][e], A.in) : 0) + add[i][e];
                v = (int32_t)(w > kResidualMost ? kResidualMost : w < -kResidualMost ? -kResidualMost : w);
            }
            r[i][e] = v;
            const int32_t counted = e >= skip ? v : 0;
            ss += (uint64_t)((int64_t)counted * counted);
        }
    }
    // two parts of 26 bits and what is above, either a sum of 64 lanes in 32 bits
    uint32_t lo = wave_sum_u32((uint32_t)ss & 0x3ffffffu), hi = wave_sum_u32((uint32_t)(ss >> 26));
    uint64_t total = (uint64_t)lo + ((uint64_t)hi << 26);
    if (WAVES > 1) {
        if (lane == 0) { parts[0][wave] = (uint32_t)total; parts[1][wave] = (uint32_t)(total >> 32); }
        __syncthreads();
        total = 0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) total += (uint64_t)parts[0][i] | (uint64_t)parts[1][i] << 32;
    }
    // (behind the loads of the whole row: the stream may be updated in place)
    if (A.residual_out) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            if (mine[i]) *reinterpret_cast<i32x4_a4 *>(A.residual_out + at + start[i]) = r[i];
        }
    }
    int t;
    const uint32_t c = row_factor(at_most_62_bits(total + (uint64_t)A.eps_sum), A.root_cols, &t);
    const int64_t half = (int64_t)1 << (40 - t);
    const int shift = 41 - t;
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int32_t z = (int32_t)(((int64_t)r[i][e] * (int32_t)c + half) >> shift);
            const int32_t y = (int32_t)(((int64_t)z * g[i][e] + 32) >> 6);
            r[i][e] = y;
            most = max(most, (uint32_t)max(y, -y));
        }
    }
    if (A.row_scales) {
        most = (uint32_t)wave_max_i32((int32_t)most);
        if (WAVES > 1) {
            if (lane == 0) tops[wave] = most;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i) most = max(most, tops[i]);
        }
        if (tid == 0) A.row_scales[row] = (int32_t)most;
        // y f / 2^40 with f = floor(127 2^40 / most): y's and f's upper parts carry it, but the rounding wants all of it
        const uint64_t f = floor_div_scaled(127, 40, most);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            int32_t code[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) code[e] = (int32_t)(((int64_t)r[i][e] * (int64_t)f + ((int64_t)1 << 39)) >> 40);
            if (mine[i]) *reinterpret_cast<u32_a1 *>(A.out + at + start[i]) = four_bytes(code);
        }
    } else {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            int32_t code[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) code[e] = code_of<FAST>(r[i][e], A.post, A.p);
            if (mine[i]) *reinterpret_cast<u32_a1 *>(A.out + at + start[i]) = four_bytes(code);
        }
    }
}

// Rows of one to three values: one per thread.
__global__ __launch_bounds__(256) void rmsnorm_narrow_kernel(const RmsnormArgs A)
{
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= A.rows) return;
    int32_t r[3] = {0, 0, 0};
    uint64_t ss = (uint64_t)A.eps_sum;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (i >= A.cols) break;
        int64_t w = A.x ? shifted(A.x[row * A.cols + i], A.in) : 0;
        if (A.residual) w += A.residual[row * A.cols + i];
        r[i] = (int32_t)(w > kResidualMost ? kResidualMost : w < -kResidualMost ? -kResidualMost : w);
        ss += (uint64_t)((int64_t)r[i] * r[i]);
        if (A.residual_out) A.residual_out[row * A.cols + i] = r[i];
    }
    int t;
    const uint32_t c = row_factor(at_most_62_bits(ss), A.root_cols, &t);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (i >= A.cols) break;
        const int32_t z = (int32_t)(((int64_t)r[i] * (int32_t)c + ((int64_t)1 << (40 - t))) >> (41 - t));
        r[i] = (int32_t)(((int64_t)z * A.gain[i] + 32) >> 6);
        most = max(most, (uint32_t)max(r[i], -r[i]));
    }
    if (A.row_scales) A.row_scales[row] = (int32_t)most;
    const uint64_t f = A.row_scales ? floor_div_scaled(127, 40, most) : 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (i >= A.cols) break;
        A.out[row * A.cols + i] = (int8_t)(A.row_scales ? (int32_t)(((int64_t)r[i] * (int64_t)f + ((int64_t)1 << 39)) >> 40) : code_of<false>(r[i], A.post, A.p));
    }
}

template <int WAVES, int CHUNKS>
static void rmsnorm_launch(const RmsnormArgs &a, bool fast, hipStream_t stream)
{
    const uint32_t grid = WAVES == 1 ? ((uint32_t)a.rows + 3) / 4 : (uint32_t)a.rows;
    launch_kernel(fast ? rmsnorm_i32_kernel<WAVES, CHUNKS, true> : rmsnorm_i32_kernel<WAVES, CHUNKS, false>, dim3(grid),
                  dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, stream, a);
}

// `rows` of a call's rows, from `first` on
static void rmsnorm_rows(const RmsnormCall &c, int64_t first, int64_t rows, hipStream_t stream)
{
    const int64_t at = first * c.cols;
    RmsnormArgs a;
    a.x = c.x ? c.x + at : nullptr; a.residual = c.residual ? c.residual + at : nullptr;
    a.residual_out = c.residual_out ? c.residual_out + at : nullptr; a.row_scales = c.row_scales ? c.row_scales + first : nullptr;
    a.gain = c.gain; a.out = c.out + at;
    a.rows = (int32_t)rows; a.cols = c.cols; a.eps_sum = c.eps_sum; a.root_cols = c.root_cols;
    a.p = c.post;
    const bool fast = c.cols >= 4 && c.in_s >= 16 && (c.post.s >= 16 || c.row_scales);
    a.in = shift_of(c.in_m, c.in_s, fast);
    a.post = shift_of(c.post.m, c.post.s, fast && c.post.s >= 16);
    if (c.cols < 4) {
        launch_kernel(rmsnorm_narrow_kernel, dim3(((uint32_t)rows + 255) / 256), dim3(256), 0, stream, a);
        return;
    }
    const int chunks = (c.cols + 3) / 4;
    // A row has as few wavefronts as hold it: one up to 512 values, four up to 8192, eight beyond, with the chunks a lane
    // that its length needs (12288 values in the eight of 16384: 67 us in place of 51 for 2000 rows).  Sixteen wavefronts with fewer chunks
    // each took longer whatever the number of rows: 1 x 4096 4.7 in place of 3.9 us, 1000 x 4096 14.6 and 10.2, as did two
    // (1 x 2048 3.7 and 3.2).  Rows of 513 to 1024 values: four wavefronts and one chunk each where latency counts (200 x 768 3.4, one wavefront
    // 4.0 us), one from 512 rows on (1000 x 768 4.4 and 4.8, 8192 x 768 15.5 and 19.1).
    auto fits = [&](int waves, int most) { return chunks <= 64 * waves * most; };
    if (fits(1, 1)) rmsnorm_launch<1, 1>(a, fast, stream);
    else if (fits(1, 2)) rmsnorm_launch<1, 2>(a, fast, stream);
    else if (fits(1, 4) && rows >= 512) rmsnorm_launch<1, 4>(a, fast, stream);
    else if (fits(4, 1)) rmsnorm_launch<4, 1>(a, fast, stream);
    else if (fits(4, 2)) rmsnorm_launch<4, 2>(a, fast, stream);
    else if (fits(4, 3)) rmsnorm_launch<4, 3>(a, fast, stream);
    else if (fits(4, 4)) rmsnorm_launch<4, 4>(a, fast, stream);
    else if (fits(4, 5)) rmsnorm_launch<4, 5>(a, fast, stream);
    else if (fits(4, 6)) rmsnorm_launch<4, 6>(a, fast, stream);
    else if (fits(4, 8)) rmsnorm_launch<4, 8>(a, fast, stream);
    else if (fits(8, 6)) rmsnorm_launch<8, 6>(a, fast, stream);
    else rmsnorm_launch<8, 8>(a, fast, stream);
}

hipError_t rmsnorm_i32_dispatch(const RmsnormCall &c, hipStream_t stream)
{
    for (int64_t r = 0; r < c.rows; r += kLaunchMost) rmsnorm_rows(c, r, std::min<int64_t>(c.rows - r, kLaunchMost), stream);
    return take_launch_status();
}

// ---- requantization by row scales ---------------------------------------------------------------
struct RequantRowsArgs {
    const int32_t *in, *row_scales;
    uint8_t *out;
    int64_t rnd;                      // of row_shift
    int32_t cols, row_shift;
    uint32_t chunks, wgs;             // of the launch
    DivDev by_row;                    // chunks of a row
    ShiftDev S;
    DyadicDev P;
};

IPTQ_DEV int32_t saturated(int64_t v)
{
    const int32_t lo = (int32_t)v, hi = (int32_t)(v >> 32);
    return hi == lo >> 31 ? lo : hi >> 31 ^ 0x7fffffff;
}

// WIDTH 4: chunks of four values; 1: rows of fewer, one value each.
template <int WIDTH, bool FAST>
__global__ __launch_bounds__(256) void requant_rows_kernel(const RequantRowsArgs A)
{
    const uint32_t step = 256 * A.wgs;
    for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < A.chunks; i += step) {
        const uint32_t row = div_by(i, A.by_row);
        const int c = WIDTH * (int)(i - row * A.by_row.d), start = WIDTH == 4 ? min(c, A.cols - 4) : c;
        const int64_t at = (int64_t)row * A.cols + start;
        const int32_t scale = A.row_scales[row];
        if (WIDTH == 4) {
            const i32x4 x = stream_load_i32x4(A.in + at);
            int32_t code[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) code[e] = code_of<FAST>(saturated(((int64_t)x[e] * scale + A.rnd) >> A.row_shift), A.S, A.P);
            stream_store_bytes4(four_bytes(code), A.out + at);
        } else {
            A.out[at] = (uint8_t)code_of<FAST>(saturated(((int64_t)A.in[at] * scale + A.rnd) >> A.row_shift), A.S, A.P);
        }
    }
}

hipError_t requant_rows_dispatch(const int32_t *in, const int32_t *row_scales, int32_t row_shift, void *out, int64_t rows,
                                 int32_t cols, const DyadicDev &P, hipStream_t stream)
{
    RequantRowsArgs a;
    a.rnd = row_shift > 0 ? (int64_t)1 << (row_shift - 1) : 0;
    a.cols = cols; a.row_shift = row_shift;
    a.S = shift_of(P.m, P.s, P.s >= 16);
    a.P = P;
    const int width = cols < 4 ? 1 : 4;
    const int64_t per_row = (cols + width - 1) / width, most_rows = (((int64_t)1 << 30) / per_row);
    a.by_row = div_of((uint32_t)per_row);
    for (int64_t r = 0; r < rows; r += most_rows) {       // (chunks are counted in 32 bits)
        const int64_t n = rows - r < most_rows ? rows - r : most_rows;
        a.in = in + r * cols; a.row_scales = row_scales + r; a.out = static_cast<uint8_t *>(out) + r * cols;
        a.chunks = (uint32_t)(n * per_row);
        a.wgs = std::min((a.chunks + 255) / 256, 16384u);
        auto kernel = width == 4 ? (P.s >= 16 ? requant_rows_kernel<4, true> : requant_rows_kernel<4, false>)
                                 : (P.s >= 16 ? requant_rows_kernel<1, true> : requant_rows_kernel<1, false>);
        launch_kernel(kernel, dim3(a.wgs), dim3(256), 0, stream, a);
    }
    return take_launch_status();
}

}  // namespace iptq
