// AdamW over many tensors: m' = beta1*m + (1 - beta1)*g, v' = beta2*v + (1 - beta2)*g*g,
// w' = keep*w - rate*m'/(sqrt(v')*root_scale + eps), with states in fp32, or m and r = sqrt(v) in 8 bits with a scale for
// every 32 values.  The tensors' pointers and sizes travel in the kernel's arguments, MXC_ADAMW_GROUP tensors a launch, so that
// nothing is copied to the device and a captured launch holds all that it needs.
#include "mxc_internal.h"

// every operation rounds by itself: where a code of 8 bits is decided, no product is kept unrounded in one place and not in another
#pragma clang fp contract(off)

namespace mxc {
namespace {

struct Tensor {
    float *w;
    const void *g;
    void *m;            // fp32, or the 8-bit states
    float *v;
    bf16_t *copy;
    size_t n;
};
struct Group {
    Tensor t[MXC_ADAMW_GROUP];
    unsigned first[MXC_ADAMW_GROUP + 1];        // workgroups before tensor i's
    int count, base;                            // base: tensors in the call before this group's
    AdamwFactors f;
    unsigned seed;
};
static_assert(sizeof(Group) <= 4096, "kernel arguments");

__device__ __forceinline__ float step_one(float &w, float g, float &m, float &v, const AdamwFactors &f)
{
    g = g * f.grad_scale;
    m = m * f.beta1 + g * f.one_beta1;
    v = v * f.beta2 + g * g * f.one_beta2;
    const float r = sqrtf(v);
    w = w * f.keep - m / (r * f.root_scale + f.eps) * f.rate;
    return r;
}

// the tensor of this workgroup
__device__ __forceinline__ int find_tensor(const Group &q)
{
    int lo = 0, hi = q.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (q.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

constexpr int CHUNK = 1024;     // values a workgroup

template <typename G>
__global__ __launch_bounds__(256) void adamw_kernel(Group q)
{
    const int i = find_tensor(q);
    const Tensor &t = q.t[i];
    const size_t at = (size_t)(blockIdx.x - q.first[i]) * CHUNK;
    for (int k = threadIdx.x; k < CHUNK && at + k < t.n; k += 256) {
        const size_t j = at + k;
        float w = t.w[j], m = ((float *)t.m)[j], v = t.v[j];
        step_one(w, load_f32((const G *)t.g + j), m, v, q.f);
        t.w[j] = w;
        ((float *)t.m)[j] = m;
        t.v[j] = v;
        if (t.copy) t.copy[j] = (bf16_t)pack_bf16x2(w, w);
    }
}

// 32 bits of x, well mixed
__device__ __forceinline__ unsigned mix(unsigned x)
{
    x = (x ^ (x >> 16)) * 0xBC0614A5u;
    x = (x ^ (x >> 15)) * 0xB0D9ED3Du;
    return x ^ (x >> 16);
}

__device__ __forceinline__ float scale_value(unsigned b) { return b == 255u ? __uint_as_float(0x7FC00000u) : b ? __uint_as_float(b << 23) : __uint_as_float(1u << 22); }

__device__ __forceinline__ float e4m3_value(unsigned c)
{
    const unsigned e = (c >> 3) & 15u, m = c & 7u;
    float v = e ? __uint_as_float(((e + 120u) << 23) | (m << 20)) : (float)m * 0x1p-9f;
    if ((c & 127u) == 127u) v = __uint_as_float(0x7FC00000u);
    return c & 128u ? -v : v;
}

// largest |x| of the block's eight lanes, as bits
__device__ __forceinline__ unsigned block_largest(const float *x)
{
    unsigned b = 0;
    for (int k = 0; k < 4; ++k) b = max(b, __float_as_uint(x[k]) & 0x7FFFFFFFu);
    for (int d = 1; d < 8; d <<= 1) b = max(b, (unsigned)__shfl_xor((int)b, d));
    return b;
}

// scale byte of a block: the smallest power of two with which its largest value is at most 448 = 1.75*2^8
__device__ __forceinline__ unsigned scale_byte(unsigned largest)
{
    const int field = (int)(largest >> 23);
    if (field == 255) return 255u;
    return (unsigned)max(field - 8 + ((largest & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
}

__device__ __forceinline__ unsigned e4m3_code(float x, unsigned byte, float u, bool root)
{
    if (byte == 255u) return 0u;
    const float y = fabsf(x) * __uint_as_float((254u - byte) << 23);
    const int E = max((int)(__float_as_uint(y) >> 23) - 120, 1);
    int k = (int)floorf(y * __uint_as_float((unsigned)(137 - E) << 23) + u) + (E - 1) * 8;
    if (root && k == 0 && x > 0.f) k = 1;
    return (unsigned)k | (x < 0.f ? 128u : 0u);
}

// a wave holds one record of 256 values, four a lane, eight lanes a block
template <typename G>
__global__ __launch_bounds__(256) void adamw8_kernel(Group q)
{
    const int i = find_tensor(q);
    const Tensor &t = q.t[i];
    const int lane = threadIdx.x & 63;
    const size_t record = (size_t)(blockIdx.x - q.first[i]) * (CHUNK / 256) + (threadIdx.x >> 6);
    if (record * 256 >= t.n) return;
    unsigned char *state = (unsigned char *)t.m + record * ADAMW8_RECORD;
    const unsigned key = mix(q.seed + (unsigned)(q.base + i + 1) * 0x9E3779B9u);
    const unsigned mc = *(const unsigned *)(state + lane * 4), rc = *(const unsigned *)(state + 256 + lane * 4);
    const float ms = scale_value(state[512 + lane / 8]), rs = scale_value(state[520 + lane / 8]);
    float m[4], r[4];
    for (int k = 0; k < 4; ++k) {
        const size_t j = record * 256 + lane * 4 + k;
        const bool in = j < t.n;
        m[k] = e4m3_value((mc >> (8 * k)) & 255u) * ms;
        r[k] = e4m3_value((rc >> (8 * k)) & 255u) * rs;
        float w = in ? t.w[j] : 0.f, v = r[k] * r[k];
        r[k] = step_one(w, in ? load_f32((const G *)t.g + j) : 0.f, m[k], v, q.f);
        if (in) {
            t.w[j] = w;
            if (t.copy) t.copy[j] = (bf16_t)pack_bf16x2(w, w);
        }
    }
    const unsigned mb = scale_byte(block_largest(m)), rb = scale_byte(block_largest(r));
    unsigned mo = 0, ro = 0;
    for (int k = 0; k < 4; ++k) {
        const unsigned bits = mix((unsigned)(record * 256 + lane * 4 + k) * 0x9E3779B9u + key);
        mo |= e4m3_code(m[k], mb, (float)(bits & 0xFFFFu) * 0x1p-16f, false) << (8 * k);
        ro |= e4m3_code(r[k], rb, (float)(bits >> 16) * 0x1p-16f, true) << (8 * k);
    }
    *(unsigned *)(state + lane * 4) = mo;
    *(unsigned *)(state + 256 + lane * 4) = ro;
    if (lane % 8 == 0) {
        state[512 + lane / 8] = (unsigned char)mb;
        state[520 + lane / 8] = (unsigned char)rb;
    }
}

}  // namespace

int adamw_update(int count, const size_t *sizes, void *const *w, const void *const *g, int grad_dtype, void *const *m, void *const *v,
                 void *const *w_bf16, const AdamwFactors &f, unsigned seed, hipStream_t st)
{
    for (int base = 0; base < count; base += MXC_ADAMW_GROUP) {
        Group q;
        q.count = count - base < MXC_ADAMW_GROUP ? count - base : MXC_ADAMW_GROUP;
        q.base = base;
        q.f = f;
        q.seed = seed;
        size_t blocks = 0;
        for (int i = 0; i < q.count; ++i) {
            const int k = base + i;
            q.t[i] = Tensor{(float *)w[k], g[k], m[k], v ? (float *)v[k] : nullptr, w_bf16 ? (bf16_t *)w_bf16[k] : nullptr, sizes[k]};
            q.first[i] = (unsigned)blocks;
            blocks += (sizes[k] + CHUNK - 1) / CHUNK;
            if (blocks > 0x7FFFFFFFu) return MXC_ERR_SHAPE;
        }
        q.first[q.count] = (unsigned)blocks;
        if (blocks == 0) continue;
        const dim3 grid((unsigned)blocks), block(256);
        if (v && grad_dtype == MXC_BF16) hipLaunchKernelGGL(adamw_kernel<bf16_t>, grid, block, 0, st, q);
        else if (v) hipLaunchKernelGGL(adamw_kernel<float>, grid, block, 0, st, q);
        else if (grad_dtype == MXC_BF16) hipLaunchKernelGGL(adamw8_kernel<bf16_t>, grid, block, 0, st, q);
        else hipLaunchKernelGGL(adamw8_kernel<float>, grid, block, 0, st, q);
        if (hipGetLastError() != hipSuccess) return MXC_ERR_LAUNCH;
    }
    return MXC_OK;
}

}  // namespace mxc
