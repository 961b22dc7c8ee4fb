// Embedding: y[n] = scale * w[tokens[n]], and the gradient of the table, dw[v] = scale * sum of dy[n] over the places n where tokens[n] == v, in
// the order of n.  Memory bounds both: forward reads and writes each row once; the gradient reads dy once and writes a row of dw for every
// token of the vocabulary.  The gradient of more than a few places goes by the tokens' order: one launch sorts the places by their token,
// one adds each token's rows, with the many places of a common token cut into parts, and one joins these parts.
#include "pieces.h"

namespace mxc {
namespace {

constexpr int NT = 256;

// lanes that share a row: a power of two, at least one piece each
int row_lanes(int C, int VE)
{
    int L = 1;
    while (L < NT && (long long)L * VE < C) L *= 2;
    return L;
}

// ---- forward ----------------------------------------------------------------------------------------------------------------

template <class T>
__global__ __launch_bounds__(NT) void fwd_kernel(int N, int V, int C, int log_lanes, const int *tokens, const T *w, float scale, T *y)
{
    constexpr int VE = Piece<T>::VE;
    const int L = 1 << log_lanes, lane = threadIdx.x & (L - 1);
    const long long n = (long long)blockIdx.x * (NT >> log_lanes) + (threadIdx.x >> log_lanes);
    if (n >= N) return;
    const int t = tokens[n];
    T *to = y + (size_t)n * C;
    const bool there = (unsigned)t < (unsigned)V;
    const T *from = w + (size_t)(there ? t : 0) * C;
    for (int c = lane * VE; c < C; c += L * VE) {
        Piece<T> p;
        p.raw = make_uint4(0, 0, 0, 0);
        if (there) {
            p = load_piece(from, c, C);
            float v[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) v[i] = p.get(i) * scale;
            p.set(v);
        }
        store_piece(to, c, C, p);
    }
}

// ---- gradient -----------------------------------------------------------------------------------------------------------------

// to[0, VE) = scale * s, or to it added
template <int VE>
__device__ __forceinline__ void put(float *row, int c, int C, const float *s, float scale, bool add)
{
#pragma unroll
    for (int k = 0; k < VE; k += 4) {
        if (c + k >= C) break;
        Piece<float> p;
        float v[4];
        if (add) {
            p = load_piece(row, c + k, C);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = p.get(i) + s[k + i] * scale;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = s[k + i] * scale;
        }
        p.set(v);
        store_piece(row, c + k, C, p);
    }
}

// s[0, VE) = the sum of the pieces at column c of rows places[0, count), in their order
template <class T>
__device__ __forceinline__ void add_rows(const T *dy, int c, int C, const int *places, int count, float *s)
{
    constexpr int VE = Piece<T>::VE, AHEAD = 4;
#pragma unroll
    for (int i = 0; i < VE; ++i) s[i] = 0.f;
    int k = 0;
    for (; k + AHEAD <= count; k += AHEAD) {
        Piece<T> p[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) p[j] = load_piece(dy + (size_t)places[k + j] * C, c, C);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) s[i] += p[j].get(i);
    }
    for (; k < count; ++k) {
        const Piece<T> p = load_piece(dy + (size_t)places[k] * C, c, C);
#pragma unroll
        for (int i = 0; i < VE; ++i) s[i] += p.get(i);
    }
}

// Few places, one launch: the workgroup of a place looks for its token among all places and, if the place is the first that has it, adds their rows;
// workgroups behind them look which of ZERO_ROWS rows of dw have no place and clear these.
constexpr int FEW = 1024, ZERO_ROWS = 64;
template <class T>
__global__ __launch_bounds__(NT) void few_kernel(int N, int V, int C, const int *tokens, const T *dy, float scale, int add, float *dw)
{
    constexpr int VE = Piece<T>::VE;
    __shared__ int places[FEW];
    __shared__ int wave_count[NT / 64];
    const int nt = blockDim.x, waves = nt / 64, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    if ((int)blockIdx.x >= N) {
        int *found = places;
        const long long v0 = (long long)(blockIdx.x - N) * ZERO_ROWS;
        if (threadIdx.x < ZERO_ROWS) found[threadIdx.x] = 0;
        __syncthreads();
        for (int n = threadIdx.x; n < N; n += nt) {
            const long long d = tokens[n] - v0;
            if (d >= 0 && d < ZERO_ROWS) found[d] = 1;
        }
        __syncthreads();
        const int rows = (int)min((long long)ZERO_ROWS, V - v0);
        const float zeros[4] = {0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < rows; ++r)
            if (!found[r])
                for (int c = ((int)blockIdx.y * nt + threadIdx.x) * 4; c < C; c += nt * 4 * gridDim.y) put<4>(dw + (size_t)(v0 + r) * C, c, C, zeros, 1.f, false);
        return;
    }
    const int me = blockIdx.x, t = tokens[me];
    if ((unsigned)t >= (unsigned)V) return;
    int count = 0;
    for (int base = 0; base < N; base += nt) {
        const int n = base + threadIdx.x;
        const bool same = n < N && tokens[n] == t;
        if (__syncthreads_or(same && n < me)) return;
        const unsigned long long b = __ballot(same);
        if (lane == 0) wave_count[wave] = __popcll(b);
        __syncthreads();
        int at = count;
        for (int k = 0; k < waves; ++k) {
            at += k < wave ? wave_count[k] : 0;
            count += wave_count[k];
        }
        if (same) places[at + __popcll(b & ((1ull << lane) - 1))] = n;
    }
    __syncthreads();
    for (int c = ((int)blockIdx.y * nt + threadIdx.x) * VE; c < C; c += nt * VE * gridDim.y) {
        float s[VE];
        add_rows(dy, c, C, places, count, s);
        put<VE>(dw + (size_t)t * C, c, C, s, scale, add);
    }
}

// The places in the order of their tokens (of equal tokens in their own), and where each token's begin: a workgroup for `R` tokens reads all places
// twice, first to count.  Each of its waves has a range of the places and a counter for each token, so that no wave waits for another on the way.
constexpr int ORDER_NT = 1024, ORDER_WAVES = ORDER_NT / 64, ORDER_MOST = 768;
static_assert(ORDER_MOST <= ORDER_NT && ORDER_WAVES * ORDER_MOST * 4 <= 48 << 10, "a thread a token; LDS that any launch may ask for");
__global__ __launch_bounds__(ORDER_NT) void order_kernel(int N, int V, int R, const int *tokens, int *order, int *start)
{
    extern __shared__ int counts[];                 // [ORDER_WAVES][R]
    __shared__ int wave_sum[ORDER_WAVES], wave_before[ORDER_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const long long lo = (long long)blockIdx.x * R;
    const int here = (int)min((long long)R, V - lo);
    for (int i = threadIdx.x; i < ORDER_WAVES * R; i += ORDER_NT) counts[i] = 0;
    __syncthreads();
    int *own = counts + wave * R;
    const int share = (N + ORDER_NT - 1) / ORDER_NT * 64;              // places of a wave
    const long long n0 = (long long)wave * share, n1 = min((long long)N, n0 + share);
    int before = 0;
    for (long long n = n0 + lane; n < n1; n += 64) {
        const int t = tokens[n];
        before += t >= 0 && t < lo;
        if (t >= lo && t < lo + here) atomicAdd(own + (t - lo), 1);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
    if (lane == 0) wave_before[wave] = before;
    __syncthreads();
    int base = 0;
    for (int k = 0; k < ORDER_WAVES; ++k) base += wave_before[k];
    // from counts to where a wave's places of a token go: a token a thread
    const int t0 = threadIdx.x;
    int total = 0;
    if (t0 < here)
        for (int k = 0; k < ORDER_WAVES; ++k) total += counts[k * R + t0];
    int up = total;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(up, d);
        up += lane >= d ? v : 0;
    }
    if (lane == 63) wave_sum[wave] = up;
    __syncthreads();
    for (int k = 0; k < wave; ++k) base += wave_sum[k];
    int at = base + up - total;
    if (t0 < here) {
        start[lo + t0] = at;
        for (int k = 0; k < ORDER_WAVES; ++k) {
            const int c = counts[k * R + t0];
            counts[k * R + t0] = at;
            at += c;
        }
        if (lo + t0 == V - 1) start[V] = at;
    }
    __syncthreads();
    for (long long m = n0; m < n1; m += 64) {
        const long long n = m + lane;
        const int t = n < n1 ? tokens[n] : -1;
        const int d = t >= lo && t < lo + here ? (int)(t - lo) : -1;
        unsigned long long left = __ballot(d >= 0);
        while (left) {
            const int first = __ffsll(left) - 1, what = __shfl(d, first);
            const unsigned long long same = __ballot(d == what);
            const int to = own[what];
            if (d == what) order[to + __popcll(same & ((1ull << lane) - 1))] = (int)n;
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (lane == first) own[what] = to + __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            left &= ~same;
        }
    }
}

// A token of more than HEAVY places is added in parts: part p is what it has among the places PART * p ... of the order.  Such a token is longer than
// a part, so that a part meets two of them at most: slot 0 is for one that holds the part's first place, slot 1 for one that begins within it.
constexpr int HEAVY = 128, PART = 64;
template <class T>
__global__ __launch_bounds__(NT) void rows_kernel(int N, int V, int C, int log_lanes, int row_groups, const int *tokens, const int *order, const int *start, const T *dy, float scale,
                                                 int add, float *dw, float *parts)
{
    constexpr int VE = Piece<T>::VE;
    const int L = 1 << log_lanes, lane = threadIdx.x & (L - 1), G = NT >> log_lanes, group = threadIdx.x >> log_lanes;
    if ((int)blockIdx.x < row_groups) {
        const long long v = (long long)blockIdx.x * G + group;
        if (v >= V) return;
        const int s0 = start[v], count = start[v + 1] - s0;
        if (count > HEAVY || (add && count == 0)) return;
        for (int c = lane * VE; c < C; c += L * VE) {
            float s[VE];
            add_rows(dy, c, C, order + s0, count, s);
            put<VE>(dw + (size_t)v * C, c, C, s, scale, add);
        }
        return;
    }
    const long long p = (long long)(blockIdx.x - row_groups) * G + group;
    const int all = start[V];
    if (p * PART >= all) return;
    const int p0 = (int)p * PART, p1 = min(all, p0 + PART);
    int t = tokens[order[p0]];
    for (int slot = 0; slot < 2; ++slot) {
        const int s0 = start[t], s1 = start[t + 1];
        if (s1 - s0 > HEAVY) {
            const int a = max(s0, p0), b = min(s1, p1);
            float *to = parts + (size_t)(2 * p + slot) * C;
            for (int c = lane * VE; c < C; c += L * VE) {
                float s[VE];
                add_rows(dy, c, C, order + a, b - a, s);
                put<VE>(to, c, C, s, 1.f, false);
            }
        }
        const int last = tokens[order[p1 - 1]];
        if (last == t) break;
        t = last;
    }
}

// A part in which a heavy token begins adds up that token's parts.
__global__ __launch_bounds__(NT) void join_kernel(int V, int C, int log_lanes, const int *tokens, const int *order, const int *start, const float *parts, float scale, int add, float *dw)
{
    const int L = 1 << log_lanes, lane = threadIdx.x & (L - 1), G = NT >> log_lanes, group = threadIdx.x >> log_lanes;
    const long long p = (long long)blockIdx.x * G + group;
    const int all = start[V];
    if (p * PART >= all) return;
    const int p0 = (int)p * PART, p1 = min(all, p0 + PART);
    int t = tokens[order[p0]];
    if (start[t] != p0) t = tokens[order[p1 - 1]];           // the one that can begin here
    const int s0 = start[t], s1 = start[t + 1];
    if (s0 < p0 || s1 - s0 <= HEAVY) return;
    const int q1 = (s1 - 1) / PART;
    for (int c = lane * 4; c < C; c += L * 4) {
        float s[4];
        Piece<float> f = load_piece(parts + (size_t)(2 * p + (s0 == p0 ? 0 : 1)) * C, c, C);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = f.get(i);
        for (int q = (int)p + 1; q <= q1; ++q) {
            f = load_piece(parts + (size_t)(2 * (long long)q) * C, c, C);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += f.get(i);
        }
        put<4>(dw + (size_t)t * C, c, C, s, scale, add);
    }
}

struct OrderPlan {
    int R, workgroups;
    long long part_count;
    size_t order_bytes, start_bytes, part_bytes;
};
OrderPlan order_plan(int N, int V, int C)
{
    OrderPlan q = {};
    q.R = (V + 255) / 256;
    if (q.R > ORDER_MOST) q.R = ORDER_MOST;
    q.workgroups = (V + q.R - 1) / q.R;
    q.part_count = N > HEAVY ? ((long long)N + PART - 1) / PART : 0;
    q.order_bytes = align_up((size_t)N * 4, 256);
    q.start_bytes = align_up(((size_t)V + 1) * 4, 256);
    q.part_bytes = align_up((size_t)q.part_count * 2 * C * 4, 256);
    return q;
}

int log2_of(int L)
{
    int k = 0;
    while ((1 << k) < L) ++k;
    return k;
}
int launched() { return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH; }

template <class T>
int fwd(int N, int V, int C, const int *tokens, const T *w, float scale, T *y, hipStream_t st)
{
    const int L = row_lanes(C, Piece<T>::VE);
    const unsigned grid = (unsigned)(((long long)N * L + NT - 1) / NT);
    hipLaunchKernelGGL(fwd_kernel<T>, dim3(grid), dim3(NT), 0, st, N, V, C, log2_of(L), tokens, w, scale, y);
    return launched();
}

template <class T>
int bwd(int N, int V, int C, const int *tokens, const T *dy, float scale, int add, float *dw, char *ws, hipStream_t st)
{
    constexpr int VE = Piece<T>::VE;
    if (N <= FEW) {
        const int L = row_lanes(C, VE), nt = L < 64 ? 64 : L;
        const unsigned grid = (unsigned)(N + (add ? 0 : ((long long)V + ZERO_ROWS - 1) / ZERO_ROWS)), columns = (unsigned)(((long long)C + nt * VE - 1) / (nt * VE));
        hipLaunchKernelGGL(few_kernel<T>, dim3(grid, columns), dim3(nt), 0, st, N, V, C, tokens, dy, scale, add, dw);
        return launched();
    }
    const OrderPlan q = order_plan(N, V, C);
    int *order = (int *)ws, *start = (int *)(ws + q.order_bytes);
    float *parts = (float *)(ws + q.order_bytes + q.start_bytes);
    hipLaunchKernelGGL(order_kernel, dim3(q.workgroups), dim3(ORDER_NT), (size_t)ORDER_WAVES * q.R * 4, st, N, V, q.R, tokens, order, start);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    const int L = row_lanes(C, VE), G = NT / L;
    const int row_groups = (int)(((long long)V + G - 1) / G);
    hipLaunchKernelGGL(rows_kernel<T>, dim3((unsigned)(row_groups + (q.part_count + G - 1) / G)), dim3(NT), 0, st, N, V, C, log2_of(L), row_groups, tokens, order, start, dy, scale, add, dw,
                       parts);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    const int LJ = row_lanes(C, 4), GJ = NT / LJ;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)((q.part_count + GJ - 1) / GJ)), dim3(NT), 0, st, V, C, log2_of(LJ), tokens, order, start, parts, scale, add, dw);
    return launched();
}

}  // namespace

int embedding_fwd(int N, int V, int C, int dtype, const int *tokens, const void *w, float scale, void *y, hipStream_t st)
{
    return dtype == MXC_BF16 ? fwd(N, V, C, tokens, (const bf16_t *)w, scale, (bf16_t *)y, st) : fwd(N, V, C, tokens, (const float *)w, scale, (float *)y, st);
}

size_t embedding_workspace(int N, int V, int C)
{
    if (N <= FEW) return 0;
    const OrderPlan q = order_plan(N, V, C);
    return q.order_bytes + q.start_bytes + q.part_bytes;
}

int embedding_bwd(int N, int V, int C, int dtype, const int *tokens, const void *dy, float scale, int add, float *dw, void *ws, hipStream_t st)
{
    return dtype == MXC_BF16 ? bwd(N, V, C, tokens, (const bf16_t *)dy, scale, add, dw, (char *)ws, st) : bwd(N, V, C, tokens, (const float *)dy, scale, add, dw, (char *)ws, st);
}

}  // namespace mxc
