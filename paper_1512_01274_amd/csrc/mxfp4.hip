// Microscaled 4-bit floating point: values to codes and scales, and back.  A block of 32 values of a row has one scale
// 2^(b - 127), b = floor(log2(largest)) - 2 + 127, so that the largest lies in [4, 8) of it and rounds to 4 or 6.
#include "mxc_internal.h"

namespace mxc {
namespace {

// 0, .5, 1, 1.5, 2, 3, 4, 6 nearest to a >= 0, half way the one of the even code
__device__ __forceinline__ unsigned e2m1(float a)
{
    return (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
}

__device__ __forceinline__ float e2m1_value(unsigned code)
{
    const unsigned m = code & 1u, e = (code >> 1) & 3u;
    const float v = e ? __uint_as_float(((e + 126u) << 23) | (m << 22)) : 0.5f * (float)m;
    return code & 8u ? -v : v;
}

__device__ __forceinline__ float scale_value(unsigned b) { return b == 255u ? __uint_as_float(0x7FC00000u) : b ? __uint_as_float(b << 23) : __uint_as_float(1u << 22); }

// one thread a block; the thread behind a row's last block clears the row's remaining scales
template <typename T>
__global__ __launch_bounds__(256) void mxfp4_quantize_kernel(int N, int C, int blocks, int scale_row, const T *x, unsigned char *codes, unsigned char *scales)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    const size_t row = i / scale_row;
    const int b = (int)(i % scale_row);
    if (row >= (size_t)N) return;
    if (b >= blocks) {
        scales[i] = 0;
        return;
    }
    const T *src = x + row * C + (size_t)b * 32;
    const int n = min(32, C - b * 32);
    unsigned largest = 0;
    for (int k = 0; k < n; ++k) largest = max(largest, __float_as_uint(load_f32(src + k)) & 0x7FFFFFFFu);
    const unsigned field = largest >> 23;
    const unsigned byte = field == 255u ? 255u : field > 2u ? field - 2u : 0u;
    const float up = __uint_as_float((254u - byte) << 23);       // 1/scale (byte <= 252)
    scales[i] = (unsigned char)byte;
    unsigned char *dst = codes + (row * blocks + b) * 16;
    for (int j = 0; j < 16; ++j) {
        unsigned two = 0;
        for (int h = 0; h < 2; ++h) {
            if (2 * j + h >= n || byte == 255u) continue;
            const float v = load_f32(src + 2 * j + h);
            two |= (e2m1(fabsf(v) * up) | (v < 0.f ? 8u : 0u)) << (4 * h);
        }
        dst[j] = (unsigned char)two;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void mxfp4_dequantize_kernel(int N, int C, int blocks, int scale_row, const unsigned char *codes, const unsigned char *scales,
                                                               T *y)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    const size_t row = i / blocks;
    const int b = (int)(i % blocks);
    if (row >= (size_t)N) return;
    const float scale = scale_value(scales[row * scale_row + b]);
    const unsigned char *src = codes + i * 16;
    T *dst = y + row * C + (size_t)b * 32;
    const int n = min(32, C - b * 32);
    for (int k = 0; k < n; ++k) {
        const float v = e2m1_value(src[k / 2] >> (4 * (k & 1))) * scale;
        if constexpr (sizeof(T) == 2) dst[k] = (bf16_t)pack_bf16x2(v, v);
        else dst[k] = v;
    }
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
                const float sc = scale_value((side ? ws : xs)[(size_t)row * scale_row + blk]);
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

int mxfp4_quantize(int N, int C, int dtype, const void *x, void *codes, void *scales, hipStream_t st)
{
    const int blocks = (int)(mxfp4_code_row(C) / 16), scale_row = (int)mxfp4_scale_row(C);
    const size_t grid = ((size_t)N * scale_row + 255) / 256;
    if (grid > 0x7FFFFFFFu) return MXC_ERR_SHAPE;
    if (dtype == MXC_BF16)
        hipLaunchKernelGGL(mxfp4_quantize_kernel<bf16_t>, dim3((unsigned)grid), dim3(256), 0, st, N, C, blocks, scale_row, (const bf16_t *)x,
                           (unsigned char *)codes, (unsigned char *)scales);
    else
        hipLaunchKernelGGL(mxfp4_quantize_kernel<float>, dim3((unsigned)grid), dim3(256), 0, st, N, C, blocks, scale_row, (const float *)x,
                           (unsigned char *)codes, (unsigned char *)scales);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

int mxfp4_dequantize(int N, int C, int dtype, const void *codes, const void *scales, void *y, hipStream_t st)
{
    const int blocks = (int)(mxfp4_code_row(C) / 16), scale_row = (int)mxfp4_scale_row(C);
    const size_t grid = ((size_t)N * blocks + 255) / 256;
    if (grid > 0x7FFFFFFFu) return MXC_ERR_SHAPE;
    if (dtype == MXC_BF16)
        hipLaunchKernelGGL(mxfp4_dequantize_kernel<bf16_t>, dim3((unsigned)grid), dim3(256), 0, st, N, C, blocks, scale_row, (const unsigned char *)codes,
                           (const unsigned char *)scales, (bf16_t *)y);
    else
        hipLaunchKernelGGL(mxfp4_dequantize_kernel<float>, dim3((unsigned)grid), dim3(256), 0, st, N, C, blocks, scale_row, (const unsigned char *)codes,
                           (const unsigned char *)scales, (float *)y);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

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
