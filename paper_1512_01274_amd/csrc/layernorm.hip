// Layer norm: y = (x - mean) * rstd * gamma + beta over rows of C values, rstd = 1 / sqrt(var + eps), and its gradient: with z = (x - mean) * rstd
// and g = dy * gamma,
//     dx = rstd * (g - sum(g) / C - z * sum(g * z) / C),   dgamma[c] = sum_n dy * z,   dbeta[c] = sum_n dy.
// Memory bounds both: a row is read once (x, and dy), held in registers over its sums, and written once.
#include "pieces.h"

namespace mxc {
namespace {

// ---- any length: a row's values are read again for each sum -------------------------------------------------------------------

constexpr int LONG_NT = 1024;
// sum over a workgroup of LONG_NT threads; `part` is free again after the next call's first barrier
__device__ __forceinline__ float workgroup_sum(float v, float *part)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[threadIdx.x & (LONG_NT / 64 - 1)];
#pragma unroll
    for (int d = LONG_NT / 128; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <class T>
__global__ __launch_bounds__(LONG_NT) void fwd_long_kernel(int N, int C, const T *x, const float *gamma, const float *beta, float eps, T *y, float *stats)
{
    constexpr int VE = Piece<T>::VE;
    __shared__ float part[LONG_NT / 64];
    for (long long n = blockIdx.x; n < N; n += gridDim.x) {
        const size_t at = (size_t)n * C;
        float s = 0.f;
        for (int c = threadIdx.x * VE; c < C; c += LONG_NT * VE) {
            const Piece<T> p = load_piece(x + at, c, C);
            for (int i = 0; i < VE; ++i) s += p.get(i);
        }
        const float mean = workgroup_sum(s, part) / (float)C;
        s = 0.f;
        for (int c = threadIdx.x * VE; c < C; c += LONG_NT * VE) {
            const Piece<T> p = load_piece(x + at, c, C);
            for (int i = 0; i < VE; ++i) {
                const float d = p.get(i) - mean;
                s += c + i < C ? d * d : 0.f;
            }
        }
        const float rstd = 1.f / sqrtf(workgroup_sum(s, part) / (float)C + eps);
        if (stats && threadIdx.x == 0) {
            stats[2 * (size_t)n] = mean;
            stats[2 * (size_t)n + 1] = rstd;
        }
        for (int c = threadIdx.x * VE; c < C; c += LONG_NT * VE) {
            Piece<T> p = load_piece(x + at, c, C);
            float v[VE];
            for (int i = 0; i < VE; ++i) {
                const bool in = c + i < C;
                v[i] = (p.get(i) - mean) * rstd * (gamma && in ? gamma[c + i] : 1.f) + (beta && in ? beta[c + i] : 0.f);
            }
            p.set(v);
            store_piece(y + at, c, C, p);
        }
    }
}

// sums[n] = (sum(g), sum(g * z)) / C
template <class T>
__global__ __launch_bounds__(LONG_NT) void bwd_sums_kernel(int N, int C, const T *x, const float *gamma, const float *stats, const T *dy, float2 *sums)
{
    constexpr int VE = Piece<T>::VE;
    __shared__ float part[LONG_NT / 64];
    for (long long n = blockIdx.x; n < N; n += gridDim.x) {
        const size_t at = (size_t)n * C;
        const float mean = stats[2 * (size_t)n], rstd = stats[2 * (size_t)n + 1];
        float sg = 0.f, sgz = 0.f;
        for (int c = threadIdx.x * VE; c < C; c += LONG_NT * VE) {
            const Piece<T> p = load_piece(x + at, c, C), q = load_piece(dy + at, c, C);
            for (int i = 0; i < VE; ++i) {
                if (c + i >= C) break;
                const float g = q.get(i) * (gamma ? gamma[c + i] : 1.f);
                sg += g;
                sgz += g * ((p.get(i) - mean) * rstd);
            }
        }
        sg = workgroup_sum(sg, part);
        sgz = workgroup_sum(sgz, part);
        if (threadIdx.x == 0) sums[n] = make_float2(sg / (float)C, sgz / (float)C);
    }
}

// a piece of columns over some of the rows: dx, and this range's share of dgamma and dbeta: part[range][2][pitch]
template <class T>
__global__ __launch_bounds__(256) void bwd_columns_kernel(int N, int C, int rows, const T *x, const float *gamma, const float *stats, const T *dy, const float2 *sums, T *dx,
                                                         float *part, int pitch)
{
    constexpr int VE = Piece<T>::VE;
    const int c = (blockIdx.x * 256 + threadIdx.x) * VE;
    if (c >= C) return;
    float gm[VE], ag[VE], ab[VE];
    for (int i = 0; i < VE; ++i) {
        gm[i] = gamma && c + i < C ? gamma[c + i] : 1.f;
        ag[i] = ab[i] = 0.f;
    }
    const long long n1 = min((long long)N, (long long)(blockIdx.y + 1) * rows);
    for (long long n = (long long)blockIdx.y * rows; n < n1; ++n) {
        const size_t at = (size_t)n * C;
        const float mean = stats[2 * n], rstd = stats[2 * n + 1];
        const float2 s = sums[n];
        const Piece<T> p = load_piece(x + at, c, C), q = load_piece(dy + at, c, C);
        float v[VE];
        for (int i = 0; i < VE; ++i) {
            const float d = q.get(i), z = (p.get(i) - mean) * rstd;
            v[i] = (d * gm[i] - s.x - z * s.y) * rstd;
            ag[i] += d * z;
            ab[i] += d;
        }
        Piece<T> r;
        r.set(v);
        store_piece(dx + at, c, C, r);
    }
    float *to = part + (size_t)blockIdx.y * 2 * pitch + c;
    for (int i = 0; i < VE; ++i)
        if (c + i < C) {
            to[i] = ag[i];
            to[pitch + i] = ab[i];
        }
}

// dgamma and dbeta from the ranges' shares, added in their order: 64 columns by 16 lanes of ranges
__global__ __launch_bounds__(1024) void bwd_join_kernel(int C, int ranges, const float *part, int pitch, float *dgamma, float *dbeta)
{
    __shared__ float sum[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), lane = threadIdx.x >> 6;
    const float *from = part + (size_t)blockIdx.y * pitch + c;
    float s = 0.f;
    if (c < C)
        for (int r = lane; r < ranges; r += 16) s += from[(size_t)r * 2 * pitch];
    sum[lane][threadIdx.x & 63] = s;
    __syncthreads();
    float *out = blockIdx.y ? dbeta : dgamma;
    if (lane || c >= C || !out) return;
    s = sum[0][threadIdx.x];
    for (int r = 1; r < 16; ++r) s += sum[r][threadIdx.x];
    out[c] = s;
}

struct BwdPlan {
    int rows, ranges, pitch;
    size_t part_bytes, sums_bytes;
};
BwdPlan bwd_plan(int N, int C, int dtype)
{
    BwdPlan q;
    const int VE = dtype == MXC_BF16 ? 8 : 4;
    const long long columns = (C + 256ll * VE - 1) / (256ll * VE);
    const long long want = columns >= 1024 ? 1 : 1024 / columns;          // ranges of rows, for about four workgroups a compute unit
    q.rows = (int)((N + want - 1) / want);
    q.ranges = (N + q.rows - 1) / q.rows;
    q.pitch = (int)align_up(C, 4);
    q.part_bytes = align_up((size_t)q.ranges * 2 * q.pitch * 4, 256);
    q.sums_bytes = align_up((size_t)N * 8, 256);
    return q;
}

}  // namespace

int layernorm_fwd(int N, int C, int dtype, const void *x, const float *gamma, const float *beta, float eps, void *y, float *stats, hipStream_t st)
{
    if (dtype == MXC_BF16)
        hipLaunchKernelGGL(fwd_long_kernel<bf16_t>, dim3(N < 1 << 20 ? N : 1 << 20), dim3(LONG_NT), 0, st, N, C, (const bf16_t *)x, gamma, beta, eps, (bf16_t *)y, stats);
    else
        hipLaunchKernelGGL(fwd_long_kernel<float>, dim3(N < 1 << 20 ? N : 1 << 20), dim3(LONG_NT), 0, st, N, C, (const float *)x, gamma, beta, eps, (float *)y, stats);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

size_t layernorm_workspace(int N, int C, int dtype)
{
    const BwdPlan q = bwd_plan(N, C, dtype);
    return q.part_bytes + q.sums_bytes;
}

template <class T>
static int bwd(int N, int C, int dtype, const T *x, const float *gamma, const float *stats, const T *dy, T *dx, float *dgamma, float *dbeta, char *ws, hipStream_t st)
{
    const BwdPlan q = bwd_plan(N, C, dtype);
    float *part = (float *)ws;
    float2 *sums = (float2 *)(ws + q.part_bytes);
    hipLaunchKernelGGL(bwd_sums_kernel<T>, dim3(N < 1 << 20 ? N : 1 << 20), dim3(LONG_NT), 0, st, N, C, x, gamma, stats, dy, sums);
    if (hipGetLastError() != hipSuccess) return MXC_ERR_LAUNCH;
    hipLaunchKernelGGL(bwd_columns_kernel<T>, dim3((unsigned)((C + 256ll * Piece<T>::VE - 1) / (256ll * Piece<T>::VE)), q.ranges), dim3(256), 0, st, N, C, q.rows, x, gamma, stats, dy,
                       sums, dx, part, q.pitch);
    if (hipGetLastError() != hipSuccess) return MXC_ERR_LAUNCH;
    if (!dgamma && !dbeta) return MXC_OK;
    hipLaunchKernelGGL(bwd_join_kernel, dim3((C + 63) / 64, 2), dim3(1024), 0, st, C, q.ranges, part, q.pitch, dgamma, dbeta);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

int layernorm_bwd(int N, int C, int dtype, const void *x, const float *gamma, const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta, void *ws, hipStream_t st)
{
    if (dtype == MXC_BF16) return bwd(N, C, dtype, (const bf16_t *)x, gamma, stats, (const bf16_t *)dy, (bf16_t *)dx, dgamma, dbeta, (char *)ws, st);
    return bwd(N, C, dtype, (const float *)x, gamma, stats, (const float *)dy, (float *)dx, dgamma, dbeta, (char *)ws, st);
}

}  // namespace mxc
