// Microscaled 4-bit floating point: values to codes and scales, and back.  A block of 32 values of a row has one scale
// 2^(b - 127), b = floor(log2(largest)) - 2 + 127, so that the largest lies in [4, 8) of it and rounds to 4 or 6.
#include "mxfp4.h"

namespace mxc {
namespace {

// (row, block) of the i-th of a workgroup's 64 blocks, for a workgroup that begins at (row0, b0)
__device__ __forceinline__ void locate(FastDiv blocks, size_t row0, int b0, int i, size_t *row, int *b)
{
    const int q = blocks.div(b0 + i);
    *row = row0 + q;
    *b = b0 + i - q * blocks.d;
}

// Memory bounds both directions: 4096 x 9216 from fp32 29 us, 5.8 TB/s, and to bf16 15.3 us, 6.2 TB/s.
// Four lanes a block, eight values a lane: a wave reads 1 KB (bf16) or 2 KB at consecutive addresses and writes 256 bytes of codes; the block's
// largest value is met in registers.
template <typename T>
__global__ __launch_bounds__(256) void mxfp4_quantize_kernel(int N, int C, FastDiv blocks, int scale_row, const T *x, unsigned *codes, unsigned char *scales)
{
    const size_t first = (size_t)blockIdx.x * 64;
    size_t row;
    int b;
    locate(blocks, first / (unsigned)blocks.d, (int)(first % (unsigned)blocks.d), threadIdx.x >> 2, &row, &b);
    if (row >= (size_t)N) return;
    const int quarter = threadIdx.x & 3, at = b * 32 + quarter * 8;
    float v[8];
    load8_edge(x + row * C + at, C - at, v);
    const unsigned byte = mxfp4_scale_byte(max_quad(largest8(v)));
    codes[(row * blocks.d + b) * 4 + quarter] = mxfp4_codes8(v, byte);
    if (quarter != 0) return;
    unsigned char *s = scales + row * scale_row + b;
    s[0] = (unsigned char)byte;
    if (b == blocks.d - 1)
        for (int k = blocks.d; k < scale_row; ++k) s[k - b] = 0;
}

// eight values a lane again; value times scale in fp32, where a subnormal result is kept, and one rounding
template <typename T>
__global__ __launch_bounds__(256) void mxfp4_dequantize_kernel(int N, int C, FastDiv blocks, int scale_row, const unsigned *codes, const unsigned char *scales, T *y)
{
    const size_t first = (size_t)blockIdx.x * 64;
    size_t row;
    int b;
    locate(blocks, first / (unsigned)blocks.d, (int)(first % (unsigned)blocks.d), threadIdx.x >> 2, &row, &b);
    if (row >= (size_t)N) return;
    const int quarter = threadIdx.x & 3, at = b * 32 + quarter * 8;
    const unsigned c = codes[(row * blocks.d + b) * 4 + quarter];
    const float scale = e8m0_value(scales[row * scale_row + b]);
    float v[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        typedef float f32x2_t __attribute__((ext_vector_type(2)));
        const f32x2_t two = k == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 0) : k == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 1)
                            : k == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 2) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 3);
        v[2 * k] = two.x * scale;
        v[2 * k + 1] = two.y * scale;
    }
    T *dst = y + row * C + at;
    const int left = C - at;
    if (left >= 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x4_any *>(dst) = u32x4_any{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        } else {
            *reinterpret_cast<f32x4_any *>(dst) = f32x4_any{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_any *>(dst + 4) = f32x4_any{v[4], v[5], v[6], v[7]};
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < left) {
            if constexpr (sizeof(T) == 2) dst[k] = (bf16_t)pack_bf16x2(v[k], v[k]);
            else dst[k] = v[k];
        }
}

template <typename T>
int quantize(int N, int C, const void *x, void *codes, void *scales, hipStream_t st)
{
    const FastDiv blocks((int)(mxfp4_code_row(C) / 16));
    const size_t grid = ((size_t)N * blocks.d + 63) / 64;
    if (!one_launch(grid, 256)) return MXC_ERR_SHAPE;
    hipLaunchKernelGGL(mxfp4_quantize_kernel<T>, dim3((unsigned)grid), dim3(256), 0, st, N, C, blocks, (int)mxfp4_scale_row(C), (const T *)x, (unsigned *)codes,
                       (unsigned char *)scales);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

template <typename T>
int dequantize(int N, int C, const void *codes, const void *scales, void *y, hipStream_t st)
{
    const FastDiv blocks((int)(mxfp4_code_row(C) / 16));
    const size_t grid = ((size_t)N * blocks.d + 63) / 64;
    if (!one_launch(grid, 256)) return MXC_ERR_SHAPE;
    hipLaunchKernelGGL(mxfp4_dequantize_kernel<T>, dim3((unsigned)grid), dim3(256), 0, st, N, C, blocks, (int)mxfp4_scale_row(C), (const unsigned *)codes,
                       (const unsigned char *)scales, (T *)y);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

}  // namespace

int mxfp4_quantize(int N, int C, int dtype, const void *x, void *codes, void *scales, hipStream_t st)
{
    return dtype == MXC_BF16 ? quantize<bf16_t>(N, C, x, codes, scales, st) : quantize<float>(N, C, x, codes, scales, st);
}

int mxfp4_dequantize(int N, int C, int dtype, const void *codes, const void *scales, void *y, hipStream_t st)
{
    return dtype == MXC_BF16 ? dequantize<bf16_t>(N, C, codes, scales, y, st) : dequantize<float>(N, C, codes, scales, y, st);
}

}  // namespace mxc
