// Root-mean-square norm with the residual's addition, and requantization by row scales.
#include "block.h"

namespace iptq {

struct RmsnormArgs {
    const int32_t *x, *residual;
    int32_t *residual_out;
    const int16_t *gain;
    int8_t *out;
    int32_t *row_scales;
    int32_t cols;
    int32_t in_m, in_s;
    int64_t eps_sum;
    uint32_t root_cols;
    DyadicDev post;
};

constexpr int32_t kResidualMost = (1 << 23) - 1;

IPTQ_DEV int64_t rounded_shift(int64_t v, int s) { return s > 0 ? (v + ((int64_t)1 << (s - 1))) >> s : v; }

// A row in LDS: sum of squares, root and factor, then the codes.
__global__ __launch_bounds__(256) void rmsnorm_i32_kernel(const RmsnormArgs A)
{
    extern __shared__ int32_t row[];
    __shared__ uint64_t parts[4];
    __shared__ uint32_t tops[4];
    const int64_t at = (int64_t)blockIdx.x * A.cols;
    uint64_t ss = 0;
    for (int i = threadIdx.x; i < A.cols; i += 256) {
        int64_t v = A.x ? rounded_shift((int64_t)A.x[at + i] * A.in_m, A.in_s) : 0;
        if (A.residual) v += A.residual[at + i];
        v = v > kResidualMost ? kResidualMost : v < -kResidualMost ? -kResidualMost : v;
        row[i] = (int32_t)v;
        if (A.residual_out) A.residual_out[at + i] = (int32_t)v;
        ss += (uint64_t)(v * v);
    }
    for (int d = 1; d < 64; d <<= 1) ss += __shfl_xor((unsigned long long)ss, d);
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = ss;
    __syncthreads();
    uint64_t total = parts[0] + parts[1] + parts[2] + parts[3] + (uint64_t)A.eps_sum;
    total = total >= ((uint64_t)1 << 62) ? ((uint64_t)1 << 62) - 1 : total;
    uint32_t c = 0;
    int t = 0;
    if (total != 0) {
        const uint32_t top = (uint32_t)(total >> 32);
        const int bits = top != 0 ? 64 - clz_u32(top) : 32 - clz_u32((uint32_t)total);
        t = (62 - bits) >> 1;
        const uint32_t inv = (uint32_t)floor_div_u64((uint64_t)1 << 61, root_u62(total << (2 * t)));
        c = (uint32_t)(((uint64_t)A.root_cols * inv) >> 24);
    }
    uint32_t most = 0;
    for (int i = threadIdx.x; i < A.cols; i += 256) {
        const int32_t z = (int32_t)(((int64_t)row[i] * c + ((int64_t)1 << (40 - t))) >> (41 - t));
        const int32_t y = (int32_t)(((int64_t)z * A.gain[i] + 32) >> 6);
        row[i] = y;
        most = max(most, (uint32_t)(y < 0 ? -y : y));
    }
    if (A.row_scales) {
        for (int d = 1; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = most;
        __syncthreads();
        most = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
        if (threadIdx.x == 0) A.row_scales[blockIdx.x] = (int32_t)most;
        const int64_t f = (int64_t)floor_div_u64((uint64_t)127 << 40, most);
        for (int i = threadIdx.x; i < A.cols; i += 256) A.out[at + i] = (int8_t)((row[i] * f + ((int64_t)1 << 39)) >> 40);
    } else {
        for (int i = threadIdx.x; i < A.cols; i += 256)
            A.out[at + i] = (int8_t)requant_dev<false>(row[i], A.post.m, A.post.s, A.post.zp, A.post.qmin, A.post.qmax);
    }
}

hipError_t rmsnorm_i32_dispatch(const RmsnormCall &c, hipStream_t stream)
{
    RmsnormArgs a;
    a.x = c.x; a.residual = c.residual; a.residual_out = c.residual_out; a.gain = c.gain; a.out = c.out; a.row_scales = c.row_scales;
    a.cols = c.cols; a.in_m = c.in_m; a.in_s = c.in_s; a.eps_sum = c.eps_sum; a.root_cols = c.root_cols; a.post = c.post;
    launch_kernel(rmsnorm_i32_kernel, dim3((uint32_t)c.rows), dim3(256), (size_t)c.cols * 4, stream, a);
    return take_launch_status();
}

struct RequantRowsArgs {
    const int32_t *in, *row_scales;
    uint8_t *out;
    int32_t cols, row_shift;
    DyadicDev P;
};

__global__ __launch_bounds__(256) void requant_rows_kernel(const RequantRowsArgs A)
{
    const int64_t at = (int64_t)blockIdx.x * A.cols;
    const int64_t scale = A.row_scales[blockIdx.x];
    for (int i = threadIdx.x; i < A.cols; i += 256) {
        int64_t v = rounded_shift(A.in[at + i] * scale, A.row_shift);
        v = v > INT32_MAX ? INT32_MAX : v < INT32_MIN ? INT32_MIN : v;
        A.out[at + i] = (uint8_t)requant_dev<false>((int32_t)v, A.P.m, A.P.s, A.P.zp, A.P.qmin, A.P.qmax);
    }
}

hipError_t requant_rows_dispatch(const int32_t *in, const int32_t *row_scales, int32_t row_shift, void *out, int64_t rows,
                                 int32_t cols, const DyadicDev &P, hipStream_t stream)
{
    const RequantRowsArgs a = {in, row_scales, static_cast<uint8_t *>(out), cols, row_shift, P};
    launch_kernel(requant_rows_kernel, dim3((uint32_t)rows), dim3(256), 0, stream, a);
    return take_launch_status();
}

}  // namespace iptq
