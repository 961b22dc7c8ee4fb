// AdamW over many tensors: m' = beta1*m + (1 - beta1)*g, v' = beta2*v + (1 - beta2)*g*g,
// w' = keep*w - rate*m'/(sqrt(v')*root_scale + eps), with states in fp32, or m and r = sqrt(v) in 8 bits with a scale for
// every 32 values.  The tensors' pointers and sizes travel in the kernel's arguments, MXC_ADAMW_GROUP tensors a launch (with 8-bit states
// MXC_ADAMW8_GROUP), so that nothing is copied to the device and a captured launch holds all that it needs.  Memory bounds it, with every byte moved once:
// 65 million values, fp32 states, gradients and a bf16 copy, 30 bytes a value, 331 us, 5.9 TB/s; 204 million with 8-bit states and bf16 gradients, 14.1
// bytes, 522 us, 5.5 TB/s, where the vector units are busy throughout, too; 24 tensors of up to 4096 values are one launch, 5.7 us.
#include "mxc_internal.h"

// every operation rounds by itself: where a code of 8 bits is decided, no product is kept unrounded in one place and not in another
#pragma clang fp contract(off)

namespace mxc {
namespace {

struct Tensor {
    float *w;
    const void *g;
    float *m, *v;
    bf16_t *copy;
    size_t n;
};
struct Tensor8 {
    float *w;
    const void *g;
    unsigned char *state;
    bf16_t *copy;
    size_t n;
};
template <class TENSOR, int N>
struct Group {
    static constexpr int MOST = N;
    TENSOR t[N];
    unsigned first[N + 1];      // workgroups before tensor i's
    int count, base;            // base: tensors in the call before this group's
    AdamwFactors f;
    unsigned seed;
};
typedef Group<Tensor, MXC_ADAMW_GROUP> Group32;
typedef Group<Tensor8, MXC_ADAMW8_GROUP> Group8;
static_assert(sizeof(Group32) <= 4096 && sizeof(Group8) <= 4096, "kernel arguments");

__device__ __forceinline__ float step_one(float &w, float g, float &m, float &v, const AdamwFactors &f)
{
    g = g * f.grad_scale;
    m = m * f.beta1 + g * f.one_beta1;
    v = v * f.beta2 + g * g * f.one_beta2;
    const float r = sqrtf(v);
    w = w * f.keep - m / (r * f.root_scale + f.eps) * f.rate;
    return r;
}

// the tensor of this workgroup: the last one that begins at or before it (tensors of no values begin where the next one does).  Every lane
// looks at one place of the table, which is one access to the kernel's arguments where a binary search is seven in a row.
template <class GROUP>
__device__ __forceinline__ int find_tensor(const GROUP &q)
{
    const int lane = threadIdx.x & 63;
    int n = __popcll(__ballot(lane < q.count && q.first[lane] <= blockIdx.x));
    if (q.count > 64) n += __popcll(__ballot(64 + lane < q.count && q.first[min(64 + lane, GROUP::MOST)] <= blockIdx.x));
    return __builtin_amdgcn_readfirstlane(n - 1);
}

constexpr int CHUNK = 1024;     // values a workgroup: four a thread, a record of 256 a wave

// NT: past the caches.  A call that touches more than these hold gains by it (16 tensors, 1.95 GB: 360 -> 331 us, 5.9 TB/s; 161 of 29 million
// values with 8-bit states, 466 MB: 101 -> 91); of a smaller one the next layer's bf16 weights and the next step's states stay.
template <bool NT, class V>
__device__ __forceinline__ V load(const void *p)
{
    if constexpr (NT) return __builtin_nontemporal_load((const V *)p);
    else return *(const V *)p;
}
template <bool NT, class V>
__device__ __forceinline__ void store(void *p, V v)
{
    if constexpr (NT) __builtin_nontemporal_store(v, (V *)p);
    else *(V *)p = v;
}
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

template <bool NT>
__device__ __forceinline__ f32x4 load4(const float *p) { return load<NT, f32x4>(p); }
template <bool NT>
__device__ __forceinline__ f32x4 load4(const bf16_t *p)
{
    const u32x2 u = load<NT, u32x2>(p);
    return f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xFFFF0000u)};
}
template <bool NT>
__device__ __forceinline__ void store4(float *p, const float *v) { store<NT>(p, f32x4{v[0], v[1], v[2], v[3]}); }
template <bool NT>
__device__ __forceinline__ void store4(bf16_t *p, const float *v) { store<NT>(p, u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}); }

template <typename G, bool NT>
__global__ __launch_bounds__(256) void adamw_kernel(Group32 q)
{
    const int i = find_tensor(q);
    const Tensor &t = q.t[i];
    const size_t j = (size_t)(blockIdx.x - q.first[i]) * CHUNK + threadIdx.x * 4;
    float *const tm = t.m;
    const G *tg = (const G *)t.g;
    if (j + 4 <= t.n) {
        const f32x4 w4 = load4<NT>(t.w + j), m4 = load4<NT>(tm + j), v4 = load4<NT>(t.v + j), g4 = load4<NT>(tg + j);
        float w[4] = {w4.x, w4.y, w4.z, w4.w}, m[4] = {m4.x, m4.y, m4.z, m4.w}, v[4] = {v4.x, v4.y, v4.z, v4.w};
        const float g[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) step_one(w[k], g[k], m[k], v[k], q.f);
        store4<NT>(t.w + j, w);
        store4<NT>(tm + j, m);
        store4<NT>(t.v + j, v);
        if (t.copy) store4<NT>(t.copy + j, w);
        return;
    }
    for (size_t k = j; k < t.n; ++k) {
        float w = t.w[k], m = tm[k], v = t.v[k];
        step_one(w, load_f32(tg + k), m, v, q.f);
        t.w[k] = w;
        tm[k] = m;
        t.v[k] = v;
        if (t.copy) t.copy[k] = (bf16_t)pack_bf16x2(w, w);
    }
}

// 32 bits of x, well mixed
__device__ __forceinline__ unsigned mix(unsigned x)
{
    x = (x ^ (x >> 16)) * 0xBC0614A5u;
    x = (x ^ (x >> 15)) * 0xB0D9ED3Du;
    return x ^ (x >> 16);
}

// values of four codes (no code is the format's NaN) times the block's scale
__device__ __forceinline__ void decode4(unsigned codes, float scale, float *x)
{
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    x[0] = lo.x * scale;
    x[1] = lo.y * scale;
    x[2] = hi.x * scale;
    x[3] = hi.y * scale;
}

// largest |x| of the block's eight lanes, as bits
__device__ __forceinline__ unsigned block_largest(const float *x)
{
    unsigned b = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) b = max(b, __float_as_uint(x[k]) & 0x7FFFFFFFu);
    b = max(b, (unsigned)__builtin_amdgcn_update_dpp(0, (int)b, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2
    b = max(b, (unsigned)__builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xF, 0xF, true));      // lanes 2 3 0 1
    return max(b, (unsigned)__builtin_amdgcn_update_dpp(0, (int)b, 0x141, 0xF, 0xF, true));  // the other half of eight
}

// scale byte of a block: the smallest power of two with which its largest value is at most 448 = 1.75*2^8
__device__ __forceinline__ unsigned scale_byte(unsigned largest)
{
    const int field = (int)(largest >> 23);
    if (field == 255) return 255u;
    return (unsigned)max(field - 8 + ((largest & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
}

// Code of x by a random choice u = u16*2^-16 between its neighbours: floor(y*2^(10-E) + u) + 8*(E - 1), y = |x|/scale in [0, 448], E its
// exponent's field in the code, at least 1.  From y = 2^-6 on the sum has no more than the 24 bits of a float's mantissa, and the
// whole is one addition to the float's bits (a carry moves on to the next exponent by itself); below, E = 1 and the sum is a float's.
__device__ __forceinline__ unsigned e4m3_code(float x, float up, unsigned u16, bool root)
{
    const float y = fabsf(x) * up;
    const unsigned normal = ((__float_as_uint(y) + (u16 << 4)) >> 20) - 960u;
    unsigned k = y < 0x1p-6f ? (unsigned)(y * 512.f + (float)u16 * 0x1p-16f) : normal;
    if (root) k = max(k, x > 0.f ? 1u : 0u);
    return k | (x < 0.f ? 128u : 0u);
}

// a wave holds one record of 256 values, four a lane, eight lanes a block
template <typename G, bool NT>
__global__ __launch_bounds__(256) void adamw8_kernel(Group8 q)
{
    const int i = find_tensor(q);
    const Tensor8 &t = q.t[i];
    const int lane = threadIdx.x & 63;
    const size_t record = (size_t)(blockIdx.x - q.first[i]) * (CHUNK / 256) + (threadIdx.x >> 6);
    if (record * 256 >= t.n) return;
    unsigned char *state = t.state + record * ADAMW8_RECORD;
    const size_t j = record * 256 + lane * 4;
    const unsigned mc = load<NT, unsigned>(state + lane * 4), rc = load<NT, unsigned>(state + 256 + lane * 4);
    const unsigned msb = state[512 + lane / 8], rsb = state[520 + lane / 8];
    const G *tg = (const G *)t.g;
    const bool whole = j + 4 <= t.n;
    float w[4] = {0.f, 0.f, 0.f, 0.f}, g[4] = {0.f, 0.f, 0.f, 0.f}, m[4], r[4];
    if (whole) {
        const f32x4 w4 = load4<NT>(t.w + j), g4 = load4<NT>(tg + j);
        w[0] = w4.x; w[1] = w4.y; w[2] = w4.z; w[3] = w4.w;
        g[0] = g4.x; g[1] = g4.y; g[2] = g4.z; g[3] = g4.w;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (j + k < t.n) {
                w[k] = t.w[j + k];
                g[k] = load_f32(tg + j + k);
            }
    }
    decode4(mc, e8m0_value(msb), m);
    decode4(rc, e8m0_value(rsb), r);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float v = r[k] * r[k];
        r[k] = step_one(w[k], g[k], m[k], v, q.f);
    }
    if (whole) {
        store4<NT>(t.w + j, w);
        if (t.copy) store4<NT>(t.copy + j, w);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (j + k < t.n) {
                t.w[j + k] = w[k];
                if (t.copy) t.copy[j + k] = (bf16_t)pack_bf16x2(w[k], w[k]);
            }
    }
    const unsigned mb = scale_byte(block_largest(m)), rb = scale_byte(block_largest(r));
    const float mup = __uint_as_float((254u - mb) << 23), rup = __uint_as_float((254u - rb) << 23);       // 1/scale (at 255 nothing is read)
    const unsigned key = mix(q.seed + (unsigned)(q.base + i + 1) * 0x9E3779B9u);
    unsigned mo = 0, ro = 0, at = (unsigned)j * 0x9E3779B9u + key;
#pragma unroll
    for (int k = 0; k < 4; ++k, at += 0x9E3779B9u) {
        const unsigned bits = mix(at);
        mo |= e4m3_code(m[k], mup, bits & 0xFFFFu, false) << (8 * k);
        ro |= e4m3_code(r[k], rup, bits >> 16, true) << (8 * k);
    }
    store<NT>(state + lane * 4, mb == 255u ? 0u : mo);
    store<NT>(state + 256 + lane * 4, rb == 255u ? 0u : ro);
    if (lane % 8 == 0) {
        state[512 + lane / 8] = (unsigned char)mb;
        state[520 + lane / 8] = (unsigned char)rb;
    }
}

// one launch for every GROUP::MOST tensors, or for fewer where one launch does not hold these; tensor(k): the k-th one's entry
template <class GROUP, class F>
int launch_groups(void (*kernel)(GROUP), int count, const AdamwFactors &f, unsigned seed, hipStream_t st, F tensor)
{
    for (int base = 0; base < count;) {
        GROUP q;
        q.base = base;
        q.f = f;
        q.seed = seed;
        size_t blocks = 0;
        int i = 0;
        for (; i < GROUP::MOST && base + i < count; ++i) {
            q.t[i] = tensor(base + i);
            const size_t more = (q.t[i].n + CHUNK - 1) / CHUNK;
            if (!one_launch(blocks + more, 256)) break;        // (the first one fits: it has 2^33 values at most)
            q.first[i] = (unsigned)blocks;
            blocks += more;
        }
        q.count = i;
        q.first[i] = (unsigned)blocks;
        base += i;
        if (blocks == 0) continue;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, q);
        if (hipGetLastError() != hipSuccess) return MXC_ERR_LAUNCH;
    }
    return MXC_OK;
}

}  // namespace

int adamw_update(int count, const size_t *sizes, void *const *w, const void *const *g, int grad_dtype, void *const *m, void *const *v,
                 void *const *w_bf16, const AdamwFactors &f, unsigned seed, hipStream_t st)
{
    size_t values = 0;
    for (int i = 0; i < count; ++i) values += sizes[i];
    // what the call reads and writes, against the 256 MB of the last cache
    const bool bf16 = grad_dtype == MXC_BF16, past = values * (4 + elem_size(grad_dtype) + (v ? 8 : 2) + (w_bf16 ? 2 : 0)) > (size_t)256 << 20;
    auto copy = [&](int k) { return w_bf16 ? (bf16_t *)w_bf16[k] : nullptr; };
    if (v)
        return launch_groups<Group32>(bf16 ? (past ? adamw_kernel<bf16_t, true> : adamw_kernel<bf16_t, false>) : (past ? adamw_kernel<float, true> : adamw_kernel<float, false>),
                                      count, f, seed, st, [&](int k) { return Tensor{(float *)w[k], g[k], (float *)m[k], (float *)v[k], copy(k), sizes[k]}; });
    return launch_groups<Group8>(bf16 ? (past ? adamw8_kernel<bf16_t, true> : adamw8_kernel<bf16_t, false>) : (past ? adamw8_kernel<float, true> : adamw8_kernel<float, false>), count,
                                 f, seed, st, [&](int k) { return Tensor8{(float *)w[k], g[k], (unsigned char *)m[k], copy(k), sizes[k]}; });
}

}  // namespace mxc
