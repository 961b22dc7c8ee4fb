// Layer norm: y = (x - mean) * rstd * gamma + beta over rows of C values, rstd = 1 / sqrt(var + eps), and its gradient: with z = (x - mean) * rstd
// and g = dy * gamma,
//     dx = rstd * (g - sum(g) / C - z * sum(g * z) / C),   dgamma[c] = sum_n dy * z,   dbeta[c] = sum_n dy.
// Memory bounds both: a row is read once (x, and dy), held in registers over its sums, and written once; rows that registers do not hold are read again.
// Sums are fp32: a thread's values one after the other, then lanes and waves as a tree; squares are of differences from the mean.  16384 x 4096 bf16: forward 48 us,
// 5.6 TB/s, gradient 78, 5.2 TB/s with the shares of dgamma and dbeta; rows of 4097 values, which begin at any element, 62 and 96; 128 x 1000 fp32 4.4 and 4.7, a launch
// each.
#include <type_traits>

#include "pieces.h"

namespace mxc {
namespace {

// ---- any length: a row's values are read again for each sum -------------------------------------------------------------------
//
// 2048 x 20000 bf16: forward 170 us, where a row's three passes follow one another, gradient 151 in two launches: 1.0 and 1.6 TB/s of what has to be read and written.

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

// Whether a row's values lie close together far from zero, where the rounding of the mean, some ulps of it, counts beside them (2^20 in 49 places had z = 1 or -1): then `rest`, the mean of
// the differences from the rounded mean, is taken from these before they are squared, and from z.  Other rows go without: both for every row 16384 x 4096 bf16 52.6 us for 48.7.
__device__ __forceinline__ bool is_near(float mean, float var, float eps) { return mean * mean > 256.f * (var + eps); }

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
        // sum over the row of f(x - mean)
        auto sum_of = [&](auto f) {
            float v = 0.f;
            for (int c = threadIdx.x * VE; c < C; c += LONG_NT * VE) {
                const Piece<T> p = load_piece(x + at, c, C);
                for (int i = 0; i < VE; ++i) v += c + i < C ? f(p.get(i) - mean) : 0.f;
            }
            return workgroup_sum(v, part);
        };
        float rest = 0.f, var = sum_of([](float d) { return d * d; }) / (float)C;
        if (is_near(mean, var, eps)) {
            rest = sum_of([](float d) { return d; }) / (float)C;
            var = sum_of([&](float d) { return (d - rest) * (d - rest); }) / (float)C;
        }
        const float rstd = 1.f / sqrtf(var + eps), off = -rest * rstd;
        if (stats && threadIdx.x == 0) {
            stats[2 * (size_t)n] = mean + rest;
            stats[2 * (size_t)n + 1] = rstd;
        }
        for (int c = threadIdx.x * VE; c < C; c += LONG_NT * VE) {
            Piece<T> p = load_piece(x + at, c, C);
            float v[VE];
            for (int i = 0; i < VE; ++i) {
                const bool in = c + i < C;
                v[i] = __builtin_fmaf(p.get(i) - mean, rstd, off) * (gamma && in ? gamma[c + i] : 1.f) + (beta && in ? beta[c + i] : 0.f);
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

// dgamma and dbeta from the ranges' shares: 32 columns by LANES lanes of ranges
template <int LANES>
__global__ __launch_bounds__(32 * LANES) void bwd_join_kernel(int C, int ranges, const float *part, int pitch, float *dgamma, float *dbeta)
{
    __shared__ float sum[LANES][33];
    const int col = threadIdx.x & 31, lane = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
    const float *from = part + (size_t)blockIdx.y * pitch + (c < C ? c : 0);
    float s = 0.f;
#pragma unroll 8
    for (int r = lane; r < ranges; r += LANES) s += from[(size_t)r * 2 * pitch];
    sum[lane][col] = s;
    __syncthreads();
    float *out = blockIdx.y ? dbeta : dgamma;
    if (lane || c >= C || !out) return;
    s = 0.f;
#pragma unroll
    for (int r = 0; r < LANES; ++r) s += sum[r][col];
    out[c] = s;
}

// ---- rows that a workgroup's registers hold ---------------------------------------------------------------------------------------
//
// A row is shared by TPR lanes of a wave (4 to 64), or with TPR = 0 by the workgroup's waves, PC pieces a lane; workgroups walk over the rows with the next
// row's loads under way, the weights (and the sums of their gradients) staying in registers.

struct __attribute__((packed, aligned(4))) Two { float x, y; };         // stats may begin at any float

constexpr int ROW_NT = 256;                // workgroup of rows that lanes share
template <int TPR> __device__ __forceinline__ int groups() { return TPR ? ROW_NT / (TPR ? TPR : 1) : 1; }

// sums over a row's lanes; `part` alternates between calls, so that one barrier keeps them apart
template <int TPR, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*part)[16])
{
    if constexpr (TPR) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = lane_sum<TPR>(v[k]);
    } else {
        const int waves = blockDim.x / 64;
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = lane_sum<64>(v[k]);
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) part[k][threadIdx.x >> 6] = v[k];
        __syncthreads();
        const int at = threadIdx.x & 15;
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = lane_sum<16>(at < waves ? part[k][at] : 0.f);
    }
}

template <class T, int TPR, int PC, bool PAST>
struct Lane {       // which pieces of a row are this lane's
    static constexpr int VE = Piece<T>::VE, V = PC * VE;
    int group, first, step;
    __device__ __forceinline__ Lane()
    {
        const int lanes = TPR ? TPR : blockDim.x;
        group = TPR ? threadIdx.x / lanes : 0;
        first = (TPR ? threadIdx.x % lanes : threadIdx.x) * VE;
        step = lanes * VE;
    }
    __device__ __forceinline__ int at(int k) const { return first + k * step; }
    __device__ __forceinline__ void load(Piece<T> (&p)[PC], const T *row, int C) const
    {
#pragma unroll
        for (int k = 0; k < PC; ++k) p[k] = begin_piece<PAST>(row, at(k), C);
    }
    __device__ __forceinline__ void settle(Piece<T> (&p)[PC], int C) const
    {
#pragma unroll
        for (int k = 0; k < PC; ++k) settle_piece(p[k], at(k), C);
    }
    __device__ __forceinline__ void weights(float (&g)[V], const float *from, float without, int C) const
    {
#pragma unroll
        for (int k = 0; k < PC; ++k)
#pragma unroll
            for (int i = 0; i < VE; i += 4) {
                if (from) {
                    const Piece<float> q = load_piece(from, at(k) + i, C);
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[k * VE + i + j] = q.get(j);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[k * VE + i + j] = without;
                }
            }
    }
};

template <class T, int TPR, int PC, bool PAST>
__global__ __launch_bounds__(TPR ? ROW_NT : 1024) void fwd_rows_kernel(int N, int C, const T *x, const float *gamma, const float *beta, float eps, T *y, float *stats)
{
    constexpr int VE = Piece<T>::VE, V = PC * VE;
    __shared__ float part[4][1][16];
    const Lane<T, TPR, PC, PAST> l;
    const int G = groups<TPR>();
    float gm[V], bt[V];
    l.weights(gm, gamma, 1.f, C);
    l.weights(bt, beta, 0.f, C);
    const float by = 1.f / (float)C;
    long long n = (long long)blockIdx.x * G + l.group;
    const long long step = (long long)gridDim.x * G, turns = (N - (long long)blockIdx.x * G + step - 1) / step;
    Piece<T> p[PC], next[PC];
    l.load(p, x + (size_t)(n < N ? n : 0) * C, C);
    for (long long turn = 0; turn < turns; ++turn, n += step) {
        const bool in = n < N;
        if (turn + 1 < turns) l.load(next, x + (size_t)(n + step < N ? n + step : 0) * C, C);
        l.settle(p, C);
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < PC; ++k)
#pragma unroll
            for (int i = 0; i < VE; ++i) s[0] += p[k].get(i);       // (zeros past the row)
        row_sums<TPR>(s, part[0]);
        const float mean = in_32_bits(s[0] * by);
        s[0] = 0.f;
#pragma unroll
        for (int k = 0; k < PC; ++k) {
            if (l.at(k) + VE <= C) {
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const float d = p[k].get(i) - mean;
                    s[0] = __builtin_fmaf(d, d, s[0]);
                }
            } else {                        // the row ends in this piece, or before it
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const float d = l.at(k) + i < C ? p[k].get(i) - mean : 0.f;
                    s[0] = __builtin_fmaf(d, d, s[0]);
                }
            }
        }
        row_sums<TPR>(s, part[1]);
        float rest = 0.f, var = s[0] * by;
        const bool near = is_near(mean, var, eps);
        if (TPR ? __any(near) : near) {
            // sum over the row of f(x - mean)
            auto sum_of = [&](auto f, float (*room)[16]) __attribute__((always_inline)) {
                s[0] = 0.f;
#pragma unroll
                for (int k = 0; k < PC; ++k) {
                    held(p[k].raw);
#pragma unroll
                    for (int i = 0; i < VE; ++i) s[0] += l.at(k) + i < C ? f(p[k].get(i) - mean) : 0.f;
                }
                row_sums<TPR>(s, room);
                return in_32_bits(s[0] * by);
            };
            const float r = sum_of([](float d) { return d; }, part[2]), v = sum_of([&](float d) { return (d - r) * (d - r); }, part[3]);
            rest = near ? r : 0.f;
            var = near ? v : var;
        }
        const float rstd = 1.f / sqrtf(var + eps), off = -rest * rstd;
#pragma unroll
        for (int k = 0; k < PC; ++k) held(p[k].raw);
        if (in) {
            if (stats && l.first == 0) *reinterpret_cast<Two *>(stats + 2 * n) = Two{mean + rest, rstd};
#pragma unroll
            for (int k = 0; k < PC; ++k) {
                float v[VE];
#pragma unroll
                for (int i = 0; i < VE; ++i) v[i] = __builtin_fmaf(p[k].get(i) - mean, rstd, off) * gm[k * VE + i] + bt[k * VE + i];
                Piece<T> r;
                r.set(v);
                store_piece<PAST>(y + (size_t)n * C, l.at(k), C, r);
            }
        }
#pragma unroll
        for (int k = 0; k < PC; ++k) p[k] = next[k];
    }
}

// dgamma and dbeta of COLUMNS columns over all rows, from the stats alone: by 8 lanes of four columns, the others sharing the rows
constexpr int COLUMNS = 32;
template <class T>
__device__ __forceinline__ void columns_of(int N, int C, int c0, const T *x, const float *stats, const T *dy, float *dgamma, float *dbeta, float *room)
{
    constexpr int AHEAD = 4;
    const int share = threadIdx.x / 8, shares = blockDim.x / 8, c = c0 + threadIdx.x % 8 * 4, at = c < C ? c : c0;
    float ag[4] = {0.f, 0.f, 0.f, 0.f}, ab[4] = {0.f, 0.f, 0.f, 0.f};
    for (int n0 = share; n0 < N; n0 += AHEAD * shares) {
        decltype(begin_quad(x, 0, 0)) p[AHEAD], q[AHEAD];
        Two st[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const size_t n = (size_t)min(n0 + j * shares, N - 1);
            p[j] = begin_quad(x + n * C, at, C);
            q[j] = begin_quad(dy + n * C, at, C);
            st[j] = *reinterpret_cast<const Two *>(stats + 2 * n);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (n0 + j * shares >= N) break;
            settle_quad(p[j], at, C);
            settle_quad(q[j], at, C);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = q[j].get(i);
                ag[i] += d * ((p[j].get(i) - st[j].x) * st[j].y);
                ab[i] += d;
            }
        }
    }
    float4 *const to = reinterpret_cast<float4 *>(room + share * 2 * COLUMNS);
    to[threadIdx.x % 8] = make_float4(ag[0], ag[1], ag[2], ag[3]);
    to[8 + threadIdx.x % 8] = make_float4(ab[0], ab[1], ab[2], ab[3]);
    __syncthreads();
    if (threadIdx.x >= 2 * COLUMNS) return;
    float s = 0.f;
#pragma unroll 8
    for (int k = 0; k < shares; ++k) s += room[k * 2 * COLUMNS + threadIdx.x];
    float *const out = threadIdx.x < COLUMNS ? dgamma : dbeta;
    if (out && c0 + (int)threadIdx.x % COLUMNS < C) out[c0 + threadIdx.x % COLUMNS] = s;
}

// FEW rows: workgroups behind those of the rows make dgamma and dbeta in the same launch, reading the rows again.  AHEAD: with the next row's loads under way; rows of
// more than 8 waves of several pieces have no registers for it (fp32 rows of four pieces keep 16 in scratch as it is): 4096 x 12000 bf16 84 us, 2048 x 12000 fp32 82, 3.5 TB/s
template <class T, int TPR, int PC, bool AHEAD, bool PAST, bool FEW>
__global__ __launch_bounds__(TPR ? ROW_NT : AHEAD && PC > 1 ? 512 : 1024) void bwd_rows_kernel(int N, int C, const T *x, const float *gamma, const float *stats, const T *dy, T *dx, float *parts, int pitch,
                                                                                                int row_groups, float *dgamma, float *dbeta)
{
    if constexpr (FEW) {
        extern __shared__ __attribute__((aligned(16))) float room[];
        if ((int)blockIdx.x >= row_groups) return columns_of(N, C, ((int)blockIdx.x - row_groups) * COLUMNS, x, stats, dy, dgamma, dbeta, room);
    }
    constexpr int VE = Piece<T>::VE, V = PC * VE;
    __shared__ float part[2][2][16];
    __shared__ float4 meet[TPR ? ROW_NT : 1];
    const Lane<T, TPR, PC, PAST> l;
    const int G = groups<TPR>();
    float gm[V], ag[V], ab[V];
    if (AHEAD) l.weights(gm, gamma, 1.f, C);
#pragma unroll
    for (int i = 0; i < V; ++i) ag[i] = ab[i] = 0.f;
    const float by = 1.f / (float)C;
    long long n = (long long)blockIdx.x * G + l.group;
    const long long step = (long long)(FEW ? row_groups : (int)gridDim.x) * G, turns = (N - (long long)blockIdx.x * G + step - 1) / step;
    Piece<T> p[PC], q[PC], p1[PC], q1[PC];
    auto fetch = [&](Piece<T> (&a)[PC], Piece<T> (&b)[PC], long long row) __attribute__((always_inline)) {
        l.load(a, x + (size_t)row * C, C);
        l.load(b, dy + (size_t)row * C, C);
    };
    fetch(p, q, n < N ? n : 0);
    Two st = *reinterpret_cast<const Two *>(stats + 2 * (n < N ? n : 0)), st1 = st;
    for (long long turn = 0; turn < turns; ++turn, n += step) {
        const bool in = n < N;
        const long long m = n + step < N ? n + step : 0;
        if (AHEAD && turn + 1 < turns) {
            fetch(p1, q1, m);
            st1 = *reinterpret_cast<const Two *>(stats + 2 * m);
        }
        if (!AHEAD) l.weights(gm, gamma, 1.f, C);
        l.settle(p, C);
        l.settle(q, C);
        const float mean = st.x, rstd = st.y;
        float s[2] = {0.f, 0.f};
        // Past the row g is zero and z is -mean * rstd.  In rows of one value that may be past all numbers (1e37 at an eps of 1e-5), and 0 * inf is NaN: their sum takes z at 2^-96.
        // (A choice for each place of every row: 1024 x 1000 bf16 11.4 us for 10.5, 16384 x 4096 85.7 for 84.1.)
        const bool far = !(fabsf(mean * rstd) <= 3.4e38f);
        const float rstd_down = far ? rstd * 0x1p-96f : rstd;
#pragma unroll
        for (int k = 0; k < PC; ++k)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const float g = q[k].get(i) * gm[k * VE + i];
                s[0] += g;
                s[1] += g * ((p[k].get(i) - mean) * rstd_down);
            }
        row_sums<TPR>(s, part[turn & 1]);
#pragma unroll
        for (int k = 0; k < PC; ++k) {
            held(p[k].raw);
            held(q[k].raw);
        }
        const float s1 = s[0] * by, s2 = s[1] * by * (far ? 0x1p96f : 1.f);
        if (in) {
#pragma unroll
            for (int k = 0; k < PC; ++k) {
                float v[VE];
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const float d = q[k].get(i), z = (p[k].get(i) - mean) * rstd;
                    v[i] = (d * gm[k * VE + i] - s1 - z * s2) * rstd;
                    ag[k * VE + i] += d * z;
                    ab[k * VE + i] += d;
                }
                Piece<T> r;
                r.set(v);
                store_piece<PAST>(dx + (size_t)n * C, l.at(k), C, r);
            }
        }
        if (AHEAD) {
#pragma unroll
            for (int k = 0; k < PC; ++k) {
                p[k] = p1[k];
                q[k] = q1[k];
            }
            st = st1;
        } else if (turn + 1 < turns) {
            fetch(p, q, m);
            st = *reinterpret_cast<const Two *>(stats + 2 * m);
        }
    }
    if constexpr (FEW) return;
    float *to = parts + (size_t)blockIdx.x * 2 * pitch;
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int k = 0; k < V; k += 4) {
            const float *a = half ? ab + k : ag + k;
            float4 f = make_float4(a[0], a[1], a[2], a[3]);
            if constexpr (TPR != 0) {          // the rows that share the workgroup meet
                __syncthreads();
                meet[threadIdx.x] = f;
                __syncthreads();
                for (int r = 1; r < G; ++r) {
                    const float4 o = meet[(threadIdx.x + r * TPR) % ROW_NT];
                    f.x += o.x; f.y += o.y; f.z += o.z; f.w += o.w;
                }
            }
            const int c = l.at(k / VE) + k % VE;
            if (l.group == 0 && c < C) *reinterpret_cast<float4 *>(to + (size_t)half * pitch + c) = f;      // (pitch is a multiple of 4)
        }
}

int launched() { return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH; }
// whether a call moves what the 256 MB of the last cache do not hold: then its rows go past the caches.  us, us past them: forward 16384 x 4096 bf16 52.8, 49.6; 4096 x 2048 fp32
// 12.7, 14.2; gradient 16384 x 4096 bf16 81.0, 77.8; 1024 x 4096 13.2, 14.5
bool past_caches(int N, int C, int tensors, int dtype) { return (unsigned long long)N * C * tensors * elem_size(dtype) >= 256ull << 20; }

// How a row is shared: TPR lanes of PC pieces (TPR = 0: `waves` waves); PC = 0: a row that registers do not hold.  More pieces a lane only where a row would need more than
// ten waves (16383 x 4097 bf16: 9 waves of one piece 95 us the gradient, 5 of two, with 134 registers, 147; 8192 x 4096 fp32: 16 of one 90, 8 of two 78.5)
struct Share {
    int TPR, PC, waves;
};
Share share_of(int C, int dtype)
{
    const int VE = dtype == MXC_BF16 ? 8 : 4, most = dtype == MXC_BF16 ? 2 : 4;
    const int P = (C + VE - 1) / VE;
    for (int lanes = 4; lanes <= 64; lanes *= 2)
        if (P <= lanes) return {lanes, 1, 1};
    for (int pc = 1; pc <= most; pc *= 2) {
        const int waves = (P + 64 * pc - 1) / (64 * pc);
        if (waves <= 10 || (pc == most && waves <= 16)) return {0, pc, waves};
    }
    return {0, 0, 0};
}

template <class T, class F>
int with_share(const Share &h, F &&f)
{
    switch (h.TPR) {
    case 4: return f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
    case 8: return f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    case 16: return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
    case 32: return f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
    case 64: return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
    default: break;
    }
    if (h.PC == 1) return f(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
    if (h.PC == 2) return f(std::integral_constant<int, 0>{}, std::integral_constant<int, 2>{});
    if constexpr (sizeof(T) == 4) return f(std::integral_constant<int, 0>{}, std::integral_constant<int, 4>{});
    return MXC_ERR_LAUNCH;
}

// rows for which one launch makes dx and the weights' gradients; us, two launches and one: 128 x 1000 fp32 8.1, 4.8; 256 x 4096 bf16 10.1, 5.0; 512 x 4096 11.2, 7.5; 1024 x 64 fp32 8.1,
// 9.5; 1024 x 1000 bf16 10.6, 19.9
bool is_few(int N) { return N <= 512; }

struct BwdPlan {
    Share h;
    bool few;                           // one launch, which leaves nothing for another
    int workgroups;                     // of rows in registers
    int rows, ranges, pitch;            // ranges: shares of dgamma and dbeta
    size_t part_bytes, sums_bytes;
};
BwdPlan bwd_plan(int N, int C, int dtype)
{
    BwdPlan q = {};
    q.h = share_of(C, dtype);
    q.few = q.h.PC && is_few(N);
    q.pitch = (int)align_up(C, 4);
    if (q.h.PC) {
        // 18 waves a compute unit (8: 105 us at 16384 x 4096 bf16, 16: 79.5; of rows that a wave shares 24 are no better), and few workgroups where there are few rows, for
        // each leaves a share that is read again: 1024 x 4096 bf16 with 512 workgroups 17.9, with 256 15.0, x 2048 16.1 and 11.5 (but fp32 x 4096 18.2 and 20.5)
        const int G = q.h.TPR ? ROW_NT / q.h.TPR : 1, waves = q.h.TPR ? ROW_NT / 64 : q.h.waves;
        const long long need = ((long long)N + G - 1) / G, most = 256ll * (waves > 18 || need <= 1024 ? 1 : 18 / waves);
        q.ranges = q.workgroups = (int)(need < most ? need : most);
    } else {
        const int VE = dtype == MXC_BF16 ? 8 : 4;
        const long long columns = (C + 256ll * VE - 1) / (256ll * VE);
        const long long want = columns >= 1024 ? 1 : 1024 / columns;          // ranges of rows, for about four workgroups a compute unit
        q.rows = (int)((N + want - 1) / want);
        q.ranges = (int)(((long long)N + q.rows - 1) / q.rows);
        q.sums_bytes = align_up((size_t)N * 8, 256);
    }
    q.part_bytes = q.few ? 0 : align_up((size_t)q.ranges * 2 * q.pitch * 4, 256);
    return q;
}

template <class T>
int fwd(int N, int C, int dtype, const T *x, const float *gamma, const float *beta, float eps, T *y, float *stats, hipStream_t st)
{
    const Share h = share_of(C, dtype);
    if (h.PC == 0) {
        hipLaunchKernelGGL(fwd_long_kernel<T>, dim3(N < 1 << 20 ? N : 1 << 20), dim3(LONG_NT), 0, st, N, C, x, gamma, beta, eps, y, stats);
        return launched();
    }
    return with_share<T>(h, [&](auto tpr, auto pc) {
        constexpr int TPR = decltype(tpr)::value, PC = decltype(pc)::value;
        const int G = TPR ? ROW_NT / (TPR ? TPR : 1) : 1, waves = TPR ? ROW_NT / 64 : h.waves;
        const long long need = ((long long)N + G - 1) / G, per_cu = (PC == 1 ? 32 : 24) / waves, most = 256 * (per_cu < 1 ? 1 : per_cu);
        const auto kernel = past_caches(N, C, 2, dtype) ? fwd_rows_kernel<T, TPR, PC, true> : fwd_rows_kernel<T, TPR, PC, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(need < most ? need : most)), dim3(64 * waves), 0, st, N, C, x, gamma, beta, eps, y, stats);
        return launched();
    });
}

template <class T>
int bwd(int N, int C, int dtype, const T *x, const float *gamma, const float *stats, const T *dy, T *dx, float *dgamma, float *dbeta, char *ws, hipStream_t st)
{
    const BwdPlan q = bwd_plan(N, C, dtype);
    float *part = (float *)ws;
    if (q.h.PC) {
        const bool few = q.few;
        const int rc = with_share<T>(q.h, [&](auto tpr, auto pc) {
            constexpr int TPR = decltype(tpr)::value, PC = decltype(pc)::value;
            const int threads = TPR ? ROW_NT : 64 * q.h.waves;
            auto launch = [&](auto kernel, int groups, int columns) {
                hipLaunchKernelGGL(kernel, dim3(groups + columns), dim3(threads), few ? threads / 8 * 2 * COLUMNS * 4 : 0, st, N, C, x, gamma, stats, dy, dx, part, q.pitch, groups, dgamma, dbeta);
                return launched();
            };
            // the kernel with the next row's loads under way, or of rows of more than 8 waves of several pieces without
            auto kernel_of = [&](auto past, auto one) {
                constexpr bool PAST = decltype(past)::value, FEW = decltype(one)::value;
                if constexpr (TPR == 0 && PC > 1)
                    if (q.h.waves > 8) return bwd_rows_kernel<T, 0, PC, false, PAST, FEW>;
                return bwd_rows_kernel<T, TPR, PC, true, PAST, FEW>;
            };
            constexpr std::true_type yes{};
            constexpr std::false_type no{};
            if (few) {
                const auto kernel = kernel_of(no, yes);
                const int columns = dgamma || dbeta ? (C + COLUMNS - 1) / COLUMNS : 0;
                // in place: what the columns read is overwritten only after them
                const bool apart = columns && ((const void *)dx == x || (const void *)dx == dy);
                if (apart && launch(kernel, 0, columns) != MXC_OK) return (int)MXC_ERR_LAUNCH;
                return launch(kernel, q.workgroups, apart ? 0 : columns);
            }
            return launch(past_caches(N, C, 3, dtype) ? kernel_of(yes, no) : kernel_of(no, no), q.workgroups, 0);
        });
        if (rc != MXC_OK || few) return rc;
    } else {
        float2 *sums = (float2 *)(ws + q.part_bytes);
        hipLaunchKernelGGL(bwd_sums_kernel<T>, dim3(N < 1 << 20 ? N : 1 << 20), dim3(LONG_NT), 0, st, N, C, x, gamma, stats, dy, sums);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
        hipLaunchKernelGGL(bwd_columns_kernel<T>, dim3((unsigned)((C + 256ll * Piece<T>::VE - 1) / (256ll * Piece<T>::VE)), q.ranges), dim3(256), 0, st, N, C, q.rows, x, gamma, stats,
                           dy, sums, dx, part, q.pitch);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    }
    if (!dgamma && !dbeta) return MXC_OK;
    const bool few = q.ranges <= 64;
    hipLaunchKernelGGL(few ? bwd_join_kernel<8> : bwd_join_kernel<32>, dim3((C + 31) / 32, 2), dim3(few ? 256 : 1024), 0, st, C, q.ranges, part, q.pitch, dgamma, dbeta);
    return launched();
}

}  // namespace

int layernorm_fwd(int N, int C, int dtype, const void *x, const float *gamma, const float *beta, float eps, void *y, float *stats, hipStream_t st)
{
    if (dtype == MXC_BF16) return fwd(N, C, dtype, (const bf16_t *)x, gamma, beta, eps, (bf16_t *)y, stats, st);
    return fwd(N, C, dtype, (const float *)x, gamma, beta, eps, (float *)y, stats, st);
}

size_t layernorm_workspace(int N, int C, int dtype)
{
    const BwdPlan q = bwd_plan(N, C, dtype);
    return q.part_bytes + q.sums_bytes;
}

int layernorm_bwd(int N, int C, int dtype, const void *x, const float *gamma, const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta, void *ws, hipStream_t st)
{
    if (dtype == MXC_BF16) return bwd(N, C, dtype, (const bf16_t *)x, gamma, stats, (const bf16_t *)dy, (bf16_t *)dx, dgamma, dbeta, (char *)ws, st);
    return bwd(N, C, dtype, (const float *)x, gamma, stats, (const float *)dy, (float *)dx, dgamma, dbeta, (char *)ws, st);
}

}  // namespace mxc
