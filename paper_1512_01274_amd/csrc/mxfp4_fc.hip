// FullyConnected on a filter in microscaled 4-bit floating point.
#include "mxfp4.h"

namespace mxc {
namespace {

__device__ __forceinline__ float e2m1_value(unsigned code)
{
    const unsigned m = code & 1u, e = (code >> 1) & 3u;
    const float v = e ? __uint_as_float(((e + 126u) << 23) | (m << 22)) : 0.5f * (float)m;
    return code & 8u ? -v : v;
}

// simplest product: 16x16 outputs a workgroup, one block of 32 columns decoded into LDS at a time
template <typename T>
__global__ __launch_bounds__(256) void mxfp4_fc_kernel(int N, int C, int K, int blocks, int scale_row, const unsigned char *xc, const unsigned char *xs,
                                                       const unsigned char *wc, const unsigned char *ws, const float *bias, int relu, T *y)
{
    __shared__ float a[16][33], b[16][33];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const long long n0 = (long long)blockIdx.y * 16, k0 = (long long)blockIdx.x * 16;
    float sum = 0.f;
    for (int blk = 0; blk < blocks; ++blk) {
        __syncthreads();
        // thread (ty, tx): row ty of either tile, byte tx of the block
        for (int side = 0; side < 2; ++side) {
            const long long row = (side ? k0 : n0) + ty;
            float lo = 0.f, hi = 0.f;
            if (row < (side ? K : N)) {
                const unsigned char c = (side ? wc : xc)[((size_t)row * blocks + blk) * 16 + tx];
                const float sc = e8m0_value((side ? ws : xs)[(size_t)row * scale_row + blk]);
                lo = e2m1_value(c & 15u) * sc;
                hi = e2m1_value(c >> 4) * sc;
            }
            (side ? b : a)[ty][2 * tx] = lo;
            (side ? b : a)[ty][2 * tx + 1] = hi;
        }
        __syncthreads();
        for (int c = 0; c < 32; ++c) sum += a[ty][c] * b[tx][c];
    }
    const long long n = n0 + ty, k = k0 + tx;
    if (n >= N || k >= K) return;
    if (bias) sum += bias[k];
    if (relu && sum < 0.f) sum = 0.f;
    if constexpr (sizeof(T) == 2) y[(size_t)n * K + k] = (bf16_t)pack_bf16x2(sum, sum);
    else y[(size_t)n * K + k] = sum;
}

}  // namespace

size_t mxfp4_fc_workspace(int N, int C, int K, int dtype)
{
    return align_up((size_t)N * mxfp4_code_row(C), 256) + align_up((size_t)N * mxfp4_scale_row(C), 256);
}

int mxfp4_fc(int N, int C, int K, int dtype, const void *x, const void *w_codes, const void *w_scales, const float *bias, int relu, void *y,
             void *workspace, hipStream_t st)
{
    const int blocks = (int)(mxfp4_code_row(C) / 16), scale_row = (int)mxfp4_scale_row(C);
    unsigned char *xc = (unsigned char *)workspace, *xs = xc + align_up((size_t)N * mxfp4_code_row(C), 256);
    const int rc = mxfp4_quantize(N, C, dtype, x, xc, xs, st);
    if (rc != MXC_OK) return rc;
    const unsigned gx = (unsigned)((K + 15ll) / 16), gy = (unsigned)((N + 15ll) / 16);
    if (gy > 65535u) return MXC_ERR_SHAPE;
    if (dtype == MXC_BF16)
        hipLaunchKernelGGL(mxfp4_fc_kernel<bf16_t>, dim3(gx, gy), dim3(256), 0, st, N, C, K, blocks, scale_row, xc, xs, (const unsigned char *)w_codes,
                           (const unsigned char *)w_scales, bias, relu, (bf16_t *)y);
    else
        hipLaunchKernelGGL(mxfp4_fc_kernel<float>, dim3(gx, gy), dim3(256), 0, st, N, C, K, blocks, scale_row, xc, xs, (const unsigned char *)w_codes,
                           (const unsigned char *)w_scales, bias, relu, (float *)y);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

}  // namespace mxc
