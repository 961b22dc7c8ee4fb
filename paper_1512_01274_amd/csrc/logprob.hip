// Log probabilities of given tokens under softmax(scale*z), entropies, the most probable tokens, and the gradient of a weighted
// sum of log probabilities and entropies.  With d = scale*(z - max), S = sum exp(d), T = sum exp(d)*d:
//     logp = d[label] - log S,    entropy = log S - T/S,    dz = e*(A + B*d) + [k == label]*scale*dlogp,
//     e = exp(d), A = scale/S*(dentropy*T/S - dlogp), B = -scale/S*dentropy.
// fp32 arithmetic whatever the storage type.
#include "mxc_internal.h"

namespace mxc {
namespace {

constexpr float LOWEST = -3.402823466e38f;

// where exp(d) is 0 the product exp(d)*d is 0, also at d = minus infinity
constexpr float NO_WEIGHT = -200.f;

// a larger key is a larger value, of equal ones the one of the lower index; 0 is no entry.  -0 counts as 0.
__device__ __forceinline__ unsigned long long rank_key(float z, unsigned index)
{
    const int b = __float_as_int(z + 0.f);
    const unsigned o = (unsigned)(b < 0 ? b ^ 0x7FFFFFFF : b) ^ 0x80000000u;
    return ((unsigned long long)o << 32) | (0xFFFFFFFFu - index);
}

constexpr int THREADS = 256;

template <class T, class F>
__device__ __forceinline__ T block_join(T v, T *red, F f)
{
    red[threadIdx.x] = v;
    __syncthreads();
    for (int half = THREADS / 2; half > 0; half >>= 1) {
        if ((int)threadIdx.x < half) red[threadIdx.x] = f(red[threadIdx.x], red[threadIdx.x + half]);
        __syncthreads();
    }
    const T r = red[0];
    __syncthreads();
    return r;
}

template <typename T>
__device__ void write_gradient(const LogprobArgs &a, const T *z, T *dz, size_t row, float m, float S, float TS, bool empty)
{
    const int label = a.labels ? a.labels[row] : -1;
    const float dl = a.dlogp && (unsigned)label < (unsigned)a.K ? a.dlogp[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f;
    const float A = a.scale / S * (dh * TS - dl), B = -a.scale / S * dh;
    for (int k = threadIdx.x; k < a.K; k += THREADS) {
        const float d = (load_f32(z + k) - m) * a.scale;
        const float g = expf(d) * (A + B * fmaxf(d, NO_WEIGHT)) + (k == label ? a.scale * dl : 0.f);
        store_f32(dz + k, empty ? 0.f : g);
    }
}

template <typename T>
__global__ __launch_bounds__(THREADS) void logprob_kernel(LogprobArgs a)
{
    __shared__ float red[THREADS];
    __shared__ unsigned long long redk[THREADS];
    const size_t row = blockIdx.x;
    const T *z = (const T *)a.z + row * a.ld;
    auto max2 = [](float x, float y) { return fmaxf(x, y); };
    auto add2 = [](float x, float y) { return x + y; };
    float m = LOWEST;
    for (int k = threadIdx.x; k < a.K; k += THREADS) m = fmaxf(m, load_f32(z + k));
    m = block_join(m, red, max2);
    float s = 0.f, t = 0.f;
    for (int k = threadIdx.x; k < a.K; k += THREADS) {
        const float d = (load_f32(z + k) - m) * a.scale, e = expf(d);
        s += e;
        t += e * fmaxf(d, NO_WEIGHT);
    }
    s = block_join(s, red, add2);
    t = block_join(t, red, add2);
    const bool empty = s == 0.f;
    const float ls = empty ? 0.f : logf(s);
    if (threadIdx.x == 0) {
        const int label = a.labels ? a.labels[row] : -1;
        if (a.logp) a.logp[row] = (unsigned)label >= (unsigned)a.K ? 0.f : empty ? -INFINITY : (load_f32(z + label) - m) * a.scale - ls;
        if (a.entropy) a.entropy[row] = empty ? 0.f : ls - t / s;
        if (a.stats) {
            a.stats[2 * row] = empty ? -INFINITY : m;
            a.stats[2 * row + 1] = ls;
        }
    }
    unsigned long long last = ~0ull;
    for (int i = 0; i < a.top; ++i) {
        unsigned long long best = 0;
        for (int k = threadIdx.x; k < a.K; k += THREADS) {
            const unsigned long long key = rank_key(load_f32(z + k), (unsigned)k);
            if (key < last && key > best) best = key;
        }
        last = block_join(best, redk, [](unsigned long long x, unsigned long long y) { return x > y ? x : y; });
        if (threadIdx.x == 0) {
            const int k = last ? (int)(0xFFFFFFFFu - (unsigned)last) : -1;
            a.top_index[row * a.top + i] = k;
            a.top_logp[row * a.top + i] = k < 0 || empty ? -INFINITY : (load_f32(z + k) - m) * a.scale - ls;
        }
    }
    if (a.dz) write_gradient(a, z, (T *)a.dz + row * a.ld, row, m, s, t / s, empty);
}

template <typename T>
__global__ __launch_bounds__(THREADS) void logprob_bwd_kernel(LogprobArgs a, const float *stats, const float *entropy)
{
    const size_t row = blockIdx.x;
    const float m = stats[2 * row], ls = stats[2 * row + 1];
    write_gradient(a, (const T *)a.z + row * a.ld, (T *)a.dz + row * a.ld, row, m, expf(ls), entropy ? ls - entropy[row] : 0.f, m == -INFINITY);
}

}  // namespace

size_t logprob_workspace(int N, int K, int dtype, int top) { return 0; }

int logprob_rows(const LogprobArgs &a, void *workspace, hipStream_t st)
{
    if (a.dtype == MXC_BF16) hipLaunchKernelGGL(logprob_kernel<bf16_t>, dim3((unsigned)a.N), dim3(THREADS), 0, st, a);
    else hipLaunchKernelGGL(logprob_kernel<float>, dim3((unsigned)a.N), dim3(THREADS), 0, st, a);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

int logprob_bwd(const LogprobArgs &a, const float *stats, const float *entropy, hipStream_t st)
{
    if (a.dtype == MXC_BF16) hipLaunchKernelGGL(logprob_bwd_kernel<bf16_t>, dim3((unsigned)a.N), dim3(THREADS), 0, st, a, stats, entropy);
    else hipLaunchKernelGGL(logprob_bwd_kernel<float>, dim3((unsigned)a.N), dim3(THREADS), 0, st, a, stats, entropy);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

}  // namespace mxc
