// Orthogonal update directions by Newton-Schulz steps, X <- a X + (b A + c A A) X with A = X X^T, over many matrices at once, and the weight update that
// uses them.  A step is three launches of matrix products that all read their operands along rows: A and B = b A + c A A, which are symmetric (the tiles on
// and above the diagonal are computed, each stored twice), and the third product.  X lies there in both orientations, Z [rows][cols] and its transpose, so
// that every operand's reduction runs along memory; sides are padded to 64 with zeros, which every product keeps zero.
//
// Numbers.  Singular values of X stay below 1.2025 (the largest a s + b s^3 + c s^5 of any s up to there), so no entry of X leaves +-1.2025, none of A off its
// diagonal +-0.73 (half the spread of its eigenvalues), none of B off its diagonal +-1.41: fp16 at fixed powers of two holds all of them with 11 bits, three more than bf16 has.  What would cost most digits is kept out of fp16: with A = diag(d) + O and
// B = diag(e) + P,
//     A A = diag(d d) + (d_i + d_j) O + O O,   B X = diag(e) X + P X,
// so that d and e live in fp32 and the matrix instructions multiply O and P alone; and X is carried as two fp16 (22 bits) whose first part is the operand, the sum a X + diag(e) X
// being formed from both.  Errors against 64 bits after 5 steps, of a Gaussian 512 x 512: 7e-4 of the norm, where rounding X, A and B to fp16 gives 2.5e-3 and to bf16 1.0e-2; of a matrix
// of rank 4, whose rounding errors the first steps would blow up by a^5, 6e-4, 7e-2 and 0.6.
#include <math.h>

#include <algorithm>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "pieces.h"

namespace mxc {
namespace {

typedef _Float16 f16_t;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
// powers of two: X at 2^15, the rest of X at 2^26, O and P at 2^14
constexpr float X_UP = 32768.f, X_DOWN = 1.f / 32768.f, LO_UP = 2048.f, LO_DOWN = 1.f / 2048.f, S_UP = 16384.f, S_DOWN = 1.f / 16384.f;

constexpr int BK = 64;                      // reduction of a stage, and what sides are padded to
constexpr int NORM_MOST = 1024, NORM_CHUNK = 2048;
constexpr int KINDS = 3, SHAPE_COUNT = 5;   // products of a step, shapes of their tiles
constexpr int SMALL_M = 64, SMALL_N = 576;
__host__ __device__ inline bool is_small(int R, int C) { return (R < C ? R : C) <= SMALL_M && (R < C ? C : R) <= SMALL_N; }

// Longer matrices whose shorter side is one tile of 64: A is split over the reduction, and what adds its parts makes B at once
__host__ __device__ inline bool is_flat(int R, int C) { return (R < C ? R : C) <= BK && !is_small(R, C); }

// The work items of a matrix in the launches of a product
struct Items {
    unsigned first, count;                  // tiles, the last of them in `split` ranges of the reduction each
    unsigned whole, split;                  // tiles that are not split
    unsigned part_first, finish_first, finish_count;            // of the split ones: the first one's first partial sums; workgroups that add them
    unsigned short shape, side;             // of the tiles: a launch each
};
// One matrix of a call: what the host knows
struct Given {
    int R, C;
    const void *u;                          // x, or the gradient
    bf16_t *y;                              // y, or the bf16 copy of w
    float *w, *m;
    char *room;                             // its part of the workspace
    float step;                             // w' = keep w - step O
    unsigned prep_first;                    // among the tiles of prepare_kernel
    Items items[KINDS];
};
constexpr int GROUP = 22;
struct Group {
    Given t[GROUP];
    unsigned first[GROUP + 1];
    int count, base;
};
struct Sizes {
    int Rp, Cp, mp;                         // rows, columns and the shorter side, padded to BK
    int norm_count, norm_parts;             // workgroups that sum the squares, and what they leave
    size_t mat, sq, side;                   // bytes of one orientation of X, of A, of a diagonal
    unsigned prep;                          // tiles of prepare_kernel
    bool flat;
    size_t bytes;
};
// and what the kernels read.  Z is ping-ponged where the third product reads it (tall), its transpose where it does not (wide); the other pair of pointers is one buffer.
struct Entry {
    int R, C, Rp, Cp, mp, tall, norm_parts;
    float step;
    const void *u;
    bf16_t *y;
    float *w, *m;
    f16_t *z[2], *zt[2], *lo, *O, *P;
    float *d, *e;
    double *norm;
    unsigned prep_first;
    Items items[KINDS];
};
struct Common {
    float momentum, grad_scale, keep;
    int nesterov, muon, bf16;
};

// The arithmetic of each value, the same wherever it is done: a product and a sum that the compiler may or may not join, or a sum that it may round to 16 bits without
// rounding to 32 first, would differ from kernel to kernel.
__device__ __forceinline__ float b_of(float o, float di, float dj, float sum) { return in_32_bits(__builtin_fmaf(NS_C, __builtin_fmaf(di + dj, o, sum), NS_B * o)); }        // off the diagonal
__device__ __forceinline__ float e_of(float d, float sum) { return __builtin_fmaf(NS_C, __builtin_fmaf(d, d, sum), NS_B * d); }                                  // on it
__device__ __forceinline__ float x_of(float e, f16_t hi, f16_t lo, float sum) { return in_32_bits(__builtin_fmaf(NS_A + e, __builtin_fmaf((float)lo, LO_DOWN, (float)hi), sum * S_DOWN)); }
__device__ __forceinline__ f16_t rest_of(float x, f16_t hi) { return (f16_t)((x - (float)hi) * LO_UP); }
__device__ __forceinline__ float w_of(float w, float x, float keep, float step) { return __builtin_fmaf(-step, x * X_DOWN, w * keep); }

// Four values of the matrix that is made orthogonal, from column c of a row of len: x, or of the gradient and the momentum.  In two steps, so that the loads of many stay under way.
// FRESH: the momentum is still to be made of the gradient; it goes back to where it was.
template <bool BF16, bool FRESH>
struct Values {
    typedef typename std::conditional<BF16, bf16_t, float>::type T;
    decltype(begin_quad((const T *)nullptr, 0, 0)) u;
    Piece<float> m;
    __device__ __forceinline__ void begin(const Common &f, const void *from, const float *mom, int c, int len)
    {
        if (FRESH || !f.muon || f.nesterov) u = begin_quad((const T *)from, c, len);
        if (f.muon) m = begin_quad(mom, c, len);
    }
    __device__ __forceinline__ void end(const Common &f, float *mom, int c, int len, float (&v)[4])
    {
        if (FRESH || !f.muon || f.nesterov) {
            settle_quad(u, c, len);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = u.get(i);
        }
        if (f.muon) {
            settle_quad(m, c, len);
            float n[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float g = v[i] * f.grad_scale;
                n[i] = FRESH ? __builtin_fmaf(m.get(i), f.momentum, g) : m.get(i);
                v[i] = f.nesterov ? __builtin_fmaf(n[i], f.momentum, g) : n[i];
            }
            if (FRESH) {
                m.set(n);
                store_piece(mom, c, len, m);
            }
        }
    }
};

// Matrices of up to SMALL_M by SMALL_N (either way), which a compute unit holds: X, its shorter side as rows, in blocks of 32 x 32, the b-th at row 32 * (b % 2) and column
// 32 * (b / 2), block b belonging to wave b % 16; a lane has row lane % 32 and of the columns 8 g + 4 (lane / 32) + 0 .. 3.  Their squares are added in this order wherever it is
// done.
constexpr int SMALL_BLOCKS = (SMALL_N / 32 * 2 + 15) / 16;
// Block b's values, zeros outside of the matrix; the momentum is made of the gradient on the way.
template <bool BF16>
__device__ __forceinline__ void block_values(const Common &f, int R, int C, const void *u, float *mom, int b, int lane, float (&v)[4][4])
{
    typedef typename std::conditional<BF16, bf16_t, float>::type T;
    const int m = min(R, C), n = max(R, C), r = b % 2 * 32 + lane % 32, c0 = b / 2 * 32 + lane / 32 * 4;
    // (loads first, outside of branches and with addresses inside of the matrix: they are under way together)
    if (R <= C) {
        const int at = min(r, m - 1) * n;
        Values<BF16, true> q[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) q[g].begin(f, (const T *)u + at, mom + at, c0 + 8 * g, n);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const bool in = r < m && c0 + 8 * g < n;
            if (in) q[g].end(f, mom + at, c0 + 8 * g, n, v[g]);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[g][i] = in && c0 + 8 * g + i < n ? v[g][i] : 0.f;
        }
    } else {
        float o[4][4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = min(c0 + 8 * g + i, n - 1) * m + min(r, m - 1);
                v[g][i] = load_f32((const T *)u + at);
                o[g][i] = f.muon ? mom[at] : 0.f;
            }
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = r < m && c0 + 8 * g + i < n;
                if (f.muon) {
                    const float grad = v[g][i] * f.grad_scale, next = __builtin_fmaf(o[g][i], f.momentum, grad);
                    v[g][i] = f.nesterov ? __builtin_fmaf(next, f.momentum, grad) : next;
                    if (in) mom[(c0 + 8 * g + i) * m + r] = next;
                }
                v[g][i] = in ? v[g][i] : 0.f;
            }
    }
}
__device__ __forceinline__ double squares_of(const float (&v)[4][4], double s)
{
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) s = __builtin_fma((double)v[g][i], (double)v[g][i], s);
    return s;
}
// s + that of the lane that DPP control CONTROL names
template <int CONTROL>
__device__ __forceinline__ double with_lane(double s)
{
    const long long bits = __double_as_longlong(s);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)bits, CONTROL, 0xF, 0xF, true), hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(bits >> 32), CONTROL, 0xF, 0xF, true);
    return s + __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
// sums over 16 lanes: pairs, fours, and the other half of eight and of sixteen, whose lanes have the same
__device__ __forceinline__ double sixteen_total(double s) { return with_lane<0x140>(with_lane<0x141>(with_lane<0x4E>(with_lane<0xB1>(s)))); }
__device__ __forceinline__ double wave_total(double s)
{
    s = sixteen_total(s);
    s += __shfl_xor(s, 16);
    return s + __shfl_xor(s, 32);
}

// ---- sums of squares, the momentum, and the table of the call's matrices ---------------------------------------------------------------------
//
// Memory bounds this one, which reads the gradient and reads and writes the momentum: 58 M values fp32 139 us, 5.0 TB/s; 8192 x 8192 bf16 without momentum 40 us, the gradient for the
// next kernel left in the last cache.  Its workgroups also lay out what those of the products do, once for all steps (derived in each product's workgroup: 42 filters 166 us, 158 so).

enum { SQUARE_X, SQUARE_A, THIRD };         // A, then P and e, then the next X

// (i, j), i <= j, of the t-th tile of the upper triangle of T x T, row by row
__device__ __forceinline__ void triangle(unsigned t, unsigned T, unsigned &i, unsigned &j)
{
    const float b = 2.f * T + 1.f;
    unsigned k = (unsigned)fmaxf(0.f, (b - sqrtf(b * b - 8.f * (float)t)) * 0.5f);
    auto start = [&](unsigned r) { return r * T - r * (r - 1) / 2; };       // (for r = 0: 0 - 0)
    while (k > 0 && start(k) > t) --k;
    while (start(k + 1) <= t) ++k;
    i = k;
    j = k + t - start(k);
}

// where tile `tile` of a matrix lies, of side x side: its first row and column
__device__ __forceinline__ void place(int Rp, int Cp, int mp, int kind, unsigned side, unsigned tile, int &m0, int &n0)
{
    unsigned ti, tj;
    if (kind == THIRD) {
        // in bands of 8 rows of tiles, column by column
        const unsigned across = (Cp + side - 1) / side, down = (Rp + side - 1) / side;
        const unsigned band = tile / (8 * across), rows = min(8u, down - band * 8), in = tile - band * 8 * across;
        ti = band * 8 + in % rows;
        tj = in / rows;
    } else {
        triangle(tile, (mp + side - 1) / side, ti, tj);
    }
    m0 = ti * side;
    n0 = tj * side;
}

// What a workgroup of a product's launch does
struct Work {
    unsigned matrix;
    int m0, n0;                             // its tile
    int part;                               // which of the matrix's partial sums, or -1: a whole tile
};
__host__ __device__ inline Sizes sizes_of(int R, int C)
{
    auto up = [](size_t bytes, size_t to) { return (bytes + to - 1) / to * to; };
    Sizes s;
    s.Rp = (int)up(R, BK);
    s.Cp = (int)up(C, BK);
    s.mp = R <= C ? s.Rp : s.Cp;
    const unsigned chunks = ((unsigned)R * (unsigned)C + NORM_CHUNK - 1) / NORM_CHUNK;
    s.norm_count = is_small(R, C) ? 4 : chunks < NORM_MOST ? (int)chunks : NORM_MOST;
    s.norm_parts = is_small(R, C) ? 16 : s.norm_count;
    s.mat = up((size_t)s.Rp * s.Cp * 2, 256);
    s.sq = up((size_t)s.mp * s.mp * 2, 256);
    s.side = up((size_t)s.mp * 4, 256);
    s.prep = (unsigned)(s.Rp / BK) * (s.Cp / BK);
    s.flat = is_flat(R, C);
    s.bytes = 4 * s.mat + 2 * s.sq + 2 * s.side + up((size_t)s.norm_parts * 8, 256);
    return s;
}
__device__ __forceinline__ Entry entry_of(const Given &g, const Sizes &s)
{
    Entry t;
    t.R = g.R; t.C = g.C; t.Rp = s.Rp; t.Cp = s.Cp; t.mp = s.mp; t.tall = g.R > g.C; t.norm_parts = s.norm_parts; t.step = g.step;
    t.u = g.u; t.y = g.y; t.w = g.w; t.m = g.m;
    char *at = g.room;
    auto take = [&](size_t bytes) { char *to = at; at += bytes; return to; };
    t.norm = (double *)at;                  // (first: norm_kernel finds it there)
    take(s.bytes - 4 * s.mat - 2 * s.sq - 2 * s.side);
    t.z[0] = (f16_t *)take(s.mat);
    t.zt[0] = (f16_t *)take(s.mat);
    f16_t *second = (f16_t *)take(s.mat);
    t.z[1] = t.tall ? second : t.z[0];
    t.zt[1] = t.tall ? t.zt[0] : second;
    t.lo = (f16_t *)take(s.mat);
    t.O = (f16_t *)take(s.sq);
    t.P = (f16_t *)take(s.sq);
    t.d = (float *)take(s.side);
    t.e = (float *)take(s.side);
    t.prep_first = g.prep_first;
#pragma unroll
    for (int k = 0; k < KINDS; ++k) t.items[k] = g.items[k];
    return t;
}
// which matrix each workgroup of the other launches belongs to
struct Maps {
    unsigned *prep, *flat, *finish[KINDS][SHAPE_COUNT];
    Work *items[KINDS][SHAPE_COUNT];
};
static_assert(sizeof(Group) + sizeof(Common) + sizeof(Maps) + 32 <= 4096, "kernel arguments");
__device__ __forceinline__ void fill(unsigned *map, unsigned first, unsigned count, unsigned value, unsigned at, unsigned step)
{
    for (unsigned k = at; k < count; k += step) map[first + k] = value;
}

template <bool BF16>
__global__ __launch_bounds__(256) void norm_kernel(Group q, Common f, Entry *table, Maps maps)
{
    // (its lanes look at all matrices at once)
    const int looked = min((int)(threadIdx.x & 63), q.count - 1), i = __builtin_amdgcn_readfirstlane(63 - __clzll(__ballot(blockIdx.x >= q.first[looked] && (int)(threadIdx.x & 63) < q.count)));
    const Given &t = q.t[i];
    const Sizes z = sizes_of(t.R, t.C);
    double *const norm = (double *)t.room;
    const unsigned part = blockIdx.x - q.first[i], at = part * 256 + threadIdx.x, step = z.norm_count * 256, me = q.base + i;
    if (at == 0) table[me] = entry_of(t, z);
    fill(maps.prep, t.prep_first, z.prep, me, at, step);
    if (at == 0 && is_flat(t.R, t.C)) maps.flat[t.items[SQUARE_A].first] = me;
    for (int k = 0; k < KINDS; ++k) {
        const Items &items = t.items[k];
        // workgroups go to the XCDs in turn: each XCD has items of the matrix that follow each other, so that its L2 serves several with what one reads
        auto spread = [](unsigned i, unsigned count) { return i % 8 * (count / 8) + min(i % 8, count % 8) + i / 8; };
        for (unsigned i = at; i < items.count; i += step) {
            const bool whole = i < items.whole;
            const unsigned piece = whole ? 0 : spread(i - items.whole, items.count - items.whole);
            Work w = {me, 0, 0, whole ? -1 : (int)piece};
            place(z.Rp, z.Cp, z.mp, k, items.side, whole ? spread(i, items.whole) : items.whole + piece / items.split, w.m0, w.n0);
            maps.items[k][items.shape][items.first + i] = w;
        }
        fill(maps.finish[k][items.shape], items.finish_first, items.finish_count, me, at, step);
    }
    if (is_small(t.R, t.C)) {               // a wave's blocks
        const int wave = part * 4 + (threadIdx.x >> 6), blocks = (max(t.R, t.C) + BK - 1) / BK * BK / 32 * 2;
        double s = 0.0;
        for (int b = wave; b < blocks; b += 16) {
            float v[4][4];
            block_values<BF16>(f, t.R, t.C, t.u, t.m, b, threadIdx.x & 63, v);
            s = squares_of(v, s);
        }
        s = wave_total(s);
        if ((threadIdx.x & 63) == 0) norm[wave] = s;
        return;
    }
    const int n = t.R * t.C;                // (2^30 at most)
    const void *u = t.u;
    float *m = t.m;
    double s = 0.0;
    constexpr int AHEAD = 4;
    const long long every = (long long)z.norm_count * 1024;
    for (long long k0 = (long long)(part * 256 + threadIdx.x) * 4; k0 < n; k0 += AHEAD * every) {
        Values<BF16, true> q[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) q[a].begin(f, u, m, (int)min(k0 + a * every, (long long)n), n);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const long long k = k0 + a * every;
            if (k >= n) break;
            float v[4];
            q[a].end(f, m, (int)k, n, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) s = k + j < n ? __builtin_fma((double)v[j], (double)v[j], s) : s;
        }
    }
    __shared__ double wave_sum[4];
    s = wave_total(s);
    if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) norm[part] = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
}

// 1 / norm, at X's power of two, as a power of two and a factor of ordinary size.  A value that is not finite makes NaN of the whole matrix; zeros stay zeros
__device__ __forceinline__ float over_norm(double squares, int &up)
{
    up = 0;
    const double norm = frexp(sqrt(squares), &up);
    return !(squares < 1e300) ? __builtin_nanf("") : squares > 0.0 ? (float)((double)X_UP / norm) : 0.f;
}

// ---- X over its norm, in both orientations: a workgroup for 64 x 64 values -----------------------------------------------------------------------
//
// Memory: 8192 x 8192 bf16 122 us, 512 MB at 4.2 TB/s; the transpose goes through LDS.

template <bool BF16>
__global__ __launch_bounds__(256) void prepare_kernel(Common f, const Entry *table, const unsigned *map)
{
    const Entry &t = table[map[blockIdx.x]];
    const unsigned tile = blockIdx.x - t.prep_first, across = t.Cp / 64;
    const int r0 = tile / across * 64, c0 = tile % across * 64;
    __shared__ f16_t turned[64][68];
    __shared__ double wave_sum[4];
    const int c = threadIdx.x % 16 * 4, row = threadIdx.x / 16;
    Values<BF16, false> q[4];
    // (rows and columns past the matrix: the last row's, not used)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const size_t at = (size_t)min(r0 + k * 16 + row, t.R - 1) * t.C;
        q[k].begin(f, BF16 ? (const void *)((const bf16_t *)t.u + at) : (const void *)((const float *)t.u + at), t.m + at, c0 + c, t.C);
    }
    double s = 0.0;
    for (int k = threadIdx.x; k < t.norm_parts; k += 256) s += t.norm[k];
    s = wave_total(s);
    if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
    __syncthreads();
    s = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    int up;
    const float by = over_norm(s, up);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        f16x4 hi, lo;
        float v[4];
        q[k].end(f, nullptr, c0 + c, t.C, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = r0 + k * 16 + row < t.R && c0 + c + i < t.C;
            const float x = in ? in_32_bits(ldexpf(v[i], -up) * by) : 0.f;
            hi[i] = (f16_t)x;
            lo[i] = rest_of(x, hi[i]);
            turned[c + i][k * 16 + row] = hi[i];
        }
        const size_t to = (size_t)(r0 + k * 16 + row) * t.Cp + c0 + c;
        *reinterpret_cast<f16x4 *>(t.z[0] + to) = hi;
        *reinterpret_cast<f16x4 *>(t.lo + to) = lo;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 64; k += 16) *reinterpret_cast<f16x4 *>(t.zt[0] + (size_t)(c0 + k + row) * t.Rp + r0 + c) = *reinterpret_cast<const f16x4 *>(&turned[k + row][c]);
}

// ---- products -----------------------------------------------------------------------------------------------------------------------------------

template <int N> __device__ __forceinline__ void wait_vmcnt() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_lgkmcnt0() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }
// the bare barrier: what it publishes has been waited for by hand (a fence would wait for every load of the ring)
__device__ __forceinline__ void ring_barrier() { pin(); __builtin_amdgcn_s_barrier(); pin(); }
template <int I> using IC = std::integral_constant<int, I>;
template <class F, int... I> __device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, I...>) { (f(IC<I>{}), ...); }
template <int N, class F> __device__ __forceinline__ void static_for(F &&f) { static_for_impl(f, std::make_integer_sequence<int, N>{}); }
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What becomes of the sums of 32 rows by NI * 32 columns, a wave's: through LDS, as fp32, in rows and then, for the other orientation, in columns.
template <int MODE, int NI>
struct Results {
    static constexpr int WN = NI * 32, PITCH = WN + 4, CPR = WN / 8, ROWS = 64 / CPR, KI = 32 / ROWS;      // chunks of 8 columns in a row; rows that 64 lanes cover; turns
    static constexpr int WITH = MODE == THIRD ? 2 : MODE == SQUARE_A ? 1 : 0, BYTES = 32 * PITCH * 4;
    // what results are made with besides the sums: X, or O, and a value of the diagonal for each row
    struct With {
        f16x8 v[KI][WITH ? WITH : 1];
        float of_row[KI];
    };
    const Entry &t;
    const Common &f;
    const int cur, last, rows, cols, mp, lane, my_row, my_col, col0, col;
    const bool tall, turned;                // turned: the other orientation is stored too
    const float *const diagonal;
    float *const stage;
    float of_col[8];                        // the diagonal at this lane's columns

    __device__ __forceinline__ Results(const Entry &t_, const Common &f_, int cur_, int last_, int m0, int n0, int col0_, float *stage_)
        : t(t_), f(f_), cur(cur_), last(last_), rows(MODE == THIRD ? t.Rp : t.mp), cols(MODE == THIRD ? t.Cp : t.mp), mp(t.mp), lane(threadIdx.x & 63), my_row(lane / CPR),
          my_col(lane % CPR * 8), col0(col0_), col(col0 + my_col), tall(t.tall != 0), turned(MODE == THIRD ? !last_ : m0 != n0), diagonal(MODE == THIRD ? t.e : t.d), stage(stage_)
    {
        if constexpr (WITH != 0)
#pragma unroll
            for (int q = 0; q < 8; q += 4) {
                const float4 f4 = *reinterpret_cast<const float4 *>(diagonal + min(col, mp - 8) + q);
                of_col[q] = f4.x; of_col[q + 1] = f4.y; of_col[q + 2] = f4.z; of_col[q + 3] = f4.w;
            }
    }
    __device__ __forceinline__ void fetch(With &w, int row0) const
    {
        if constexpr (WITH != 0) {
#pragma unroll
            for (int k = 0; k < KI; ++k) {
                const int row = row0 + k * ROWS + my_row;
                const size_t at = (size_t)min(row, rows - 1) * cols + min(col, cols - 8);
                w.v[k][0] = *reinterpret_cast<const f16x8 *>((MODE == THIRD ? t.z[cur] : t.O) + at);
                if constexpr (WITH == 2) w.v[k][WITH - 1] = *reinterpret_cast<const f16x8 *>(t.lo + at);
                w.of_row[k] = diagonal[min(row, mp - 1)];
            }
        }
    }
    __device__ __forceinline__ void put(const f32x16 (&acc)[NI], const With &with, int row0) const
    {
        const int frag_row = lane & 31, frag_k = lane >> 5;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(stage + frag_row * PITCH + j * 32 + 8 * g + 4 * frag_k) =
                    make_float4(acc[j][4 * g], acc[j][4 * g + 1], acc[j][4 * g + 2], acc[j][4 * g + 3]);
        wave_sync();
#pragma unroll
        for (int turn = 0; turn < KI; ++turn) {
            const int r = turn * ROWS + my_row, c = my_col, row = row0 + r;
            float v[8];
            *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(stage + r * PITCH + c);
            *reinterpret_cast<float4 *>(v + 4) = *reinterpret_cast<const float4 *>(stage + r * PITCH + c + 4);
            f16x8 out;
            if (row < rows && col < cols) {
                if constexpr (MODE == SQUARE_X) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        v[q] *= X_DOWN * X_DOWN;
                        if (col + q == row) {
                            t.d[row] = v[q];
                            v[q] = 0.f;
                        }
                        out[q] = (f16_t)(v[q] * S_UP);
                    }
                    *reinterpret_cast<f16x8 *>(t.O + (size_t)row * mp + col) = out;
                } else if constexpr (MODE == SQUARE_A) {
                    const f16x8 o = with.v[turn][0];
                    const float di = with.of_row[turn];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float s = v[q] * (S_DOWN * S_DOWN);
                        v[q] = b_of((float)o[q] * S_DOWN, di, of_col[q], s);
                        if (col + q == row) {
                            t.e[row] = e_of(di, s);
                            v[q] = 0.f;
                        }
                        out[q] = (f16_t)(v[q] * S_UP);
                    }
                    *reinterpret_cast<f16x8 *>(t.P + (size_t)row * mp + col) = out;
                } else {
                    const size_t at = (size_t)row * t.Cp + col;
                    const f16x8 hi = with.v[turn][0], lo = with.v[turn][WITH ? WITH - 1 : 0];
                    const float er = with.of_row[turn];
                    f16x8 low;
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float e = tall ? of_col[q] : er;
                        v[q] = x_of(e, hi[q], lo[q], v[q]);       // at 2^15, as X is
                        out[q] = (f16_t)v[q];
                        low[q] = rest_of(v[q], out[q]);
                    }
                    if (!last) {
                        *reinterpret_cast<f16x8 *>(t.z[cur ^ 1] + at) = out;
                        *reinterpret_cast<f16x8 *>(t.lo + at) = low;
                    } else if (row < t.R && col < t.C) {
                        Piece<bf16_t> copy;
                        if (f.muon) {
                            float *w = t.w + (size_t)row * t.C;
#pragma unroll
                            for (int h = 0; h < 8; h += 4) {
                                if (col + h >= t.C) break;
                                Piece<float> p = load_piece(w, col + h, t.C);
                                float n[4];
#pragma unroll
                                for (int q = 0; q < 4; ++q) n[q] = v[h + q] = w_of(p.get(q), v[h + q], f.keep, t.step);
                                p.set(n);
                                store_piece(w, col + h, t.C, p);
                            }
                        } else {
#pragma unroll
                            for (int q = 0; q < 8; ++q) v[q] *= X_DOWN;
                        }
                        copy.set(v);
                        if (t.y) store_piece(t.y + (size_t)row * t.C, col, t.C, copy);
                    }
                }
                if (turned) {               // the values as stored
                    *reinterpret_cast<float4 *>(stage + r * PITCH + c) = make_float4((float)out[0], (float)out[1], (float)out[2], (float)out[3]);
                    *reinterpret_cast<float4 *>(stage + r * PITCH + c + 4) = make_float4((float)out[4], (float)out[5], (float)out[6], (float)out[7]);
                }
            }
        }
        wave_sync();
        if (turned) {
            f16_t *to = MODE == THIRD ? t.zt[cur ^ 1] : MODE == SQUARE_X ? t.O : t.P;
#pragma unroll
            for (int k = 0; k < WN; k += 16) {
                const int c = k + lane / 4, r = lane % 4 * 8;
                f16x8 out;
#pragma unroll
                for (int q = 0; q < 8; ++q) out[q] = (f16_t)stage[(r + q) * PITCH + c];
                if (row0 + r < rows && col0 + c < cols) *reinterpret_cast<f16x8 *>(to + (size_t)(col0 + c) * rows + row0 + r) = out;
            }
            wave_sync();
        }
    }
};

// Tiles of BM x BN by WR x WC waves.  The reduction runs through a ring of NS stages of 64 values in LDS, filled by loads that go there directly and are issued
// NS stages ahead; 16-byte chunk k of a row lies at chunk k ^ (row / 2 % 8), which spreads the operand fetches over the banks.
// A tile that is split leaves its sums, in the order of the registers, for finish_kernel.
// Power and then the matrix pipe bound large ones: third products of 8192 x 8192 by tiles of 256 1000 us, 1.10 PFLOP/s, pipe busy 0.66 at 1.6 GHz; squares 485 to 500, of half the
// operations.  A tile of 256 has 18 us to begin and end beside 1.35 a stage, and thirds what they fetch and store, 10 bytes a value.
template <int BM, int BN, int NS, int WR, int WC, int MODE>
__global__ __launch_bounds__(64 * WR * WC) void product_kernel(const Entry *table, const Work *map, int cur, int last, Common f, float *partial)
{
    constexpr int NW = WR * WC, WM = BM / WR, WN = BN / WC, MI = WM / 32, NI = WN / 32, NMF = MI * NI;
    constexpr int RPL = 8, A_LD = BM / RPL / NW, B_LD = BN / RPL / NW, L = A_LD + B_LD, KS = BK / 16;
    constexpr int STAGE = (BM + BN) * BK * 2, STAGING = NW * Results<MODE, NI>::BYTES;
    static_assert(BM == BN && BM % (RPL * NW) == 0 && BN % (RPL * NW) == 0 && KS % 2 == 0 && L * (NS - 1) < 64, "tile");
    constexpr int LDS = STAGE * NS > STAGING ? STAGE * NS : STAGING;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];

    const Work me = map[blockIdx.x];
    const Entry &t = table[me.matrix];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave / WC * WM, wave_n = wave % WC * WN;
    const bool tall = t.tall != 0, whole = me.part < 0;
    const int mp = t.mp, m0 = me.m0, n0 = me.n0;

    const f16_t *a, *b;
    int K, a_rows, b_rows;
    if (MODE == THIRD) {
        a = tall ? t.z[cur] : t.P;
        b = tall ? t.P : t.zt[cur];
        K = mp;
        a_rows = t.Rp;
        b_rows = t.Cp;
    } else {
        a = MODE == SQUARE_A ? t.O : tall ? t.zt[cur] : t.z[cur];
        b = a;
        K = MODE == SQUARE_A ? mp : tall ? t.Rp : t.Cp;
        a_rows = b_rows = mp;
    }
    int k0 = 0, stages = K / BK;
    if (!whole) {
        const int split = (int)t.items[MODE].split, per = (stages + split - 1) / split;
        k0 = me.part % split * per;
        stages = max(0, min(per, stages - k0));
    }

    // rows past the operand's lie past the resource's end: their loads give zeros
    const buf_rsrc_t rs_a = make_buf_rsrc(a, (unsigned)a_rows * (unsigned)K * 2u), rs_b = make_buf_rsrc(b, (unsigned)b_rows * (unsigned)K * 2u);
    const int ld_row = lane / 8, ld_chunk = (lane % 8) ^ ((4 * wave + ld_row / 2) % 8);
    unsigned va[A_LD], vb[B_LD];
#pragma unroll
    for (int i = 0; i < A_LD; ++i) va[i] = (unsigned)(m0 + RPL * (wave + NW * i) + ld_row) * (unsigned)K * 2u + ld_chunk * 16 + k0 * (BK * 2);
#pragma unroll
    for (int i = 0; i < B_LD; ++i) vb[i] = (unsigned)(n0 + RPL * (wave + NW * i) + ld_row) * (unsigned)K * 2u + ld_chunk * 16 + k0 * (BK * 2);
    static_assert(NW % 2 == 0, "the chunk a lane loads is the same for all of its loads");
    auto load_task = [&](auto k, unsigned char *stage) __attribute__((always_inline)) {
        constexpr int Tk = decltype(k)::value;
        if constexpr (Tk < A_LD) {
            lds_dma16(rs_a, va[Tk], stage + (wave + NW * Tk) * 1024);
            va[Tk] += BK * 2;
        } else {
            lds_dma16(rs_b, vb[Tk - A_LD], stage + BM * BK * 2 + (wave + NW * (Tk - A_LD)) * 1024);
            vb[Tk - A_LD] += BK * 2;
        }
    };

    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int frag_row = lane & 31, frag_k = lane >> 5, frag_swz = frag_row / 2 % 8;
    struct Frags { f16x8 a[MI], b[NI]; } f0, f1;
    constexpr int N_READ = MI + NI;
    auto read_task = [&](auto k, Frags &to, const unsigned char *stage, int ks) __attribute__((always_inline)) {
        constexpr int Tk = decltype(k)::value;
        const int at = ((ks * 2 + frag_k) ^ frag_swz) * 16;
        if constexpr (Tk < MI) to.a[Tk] = *reinterpret_cast<const f16x8 *>(stage + (wave_m + Tk * 32 + frag_row) * 128 + at);
        else to.b[Tk - MI] = *reinterpret_cast<const f16x8 *>(stage + BM * BK * 2 + (wave_n + (Tk - MI) * 32 + frag_row) * 128 + at);
    };
    // the matrix instructions of 16 values of the reduction with side tasks between them, the first NFRONT of them (operand fetches) in the first half
    auto mfma_with = [&](const Frags &x, auto nfront, auto ntask, auto &&task) __attribute__((always_inline)) {
        constexpr int NFRONT = decltype(nfront)::value, NTASK = decltype(ntask)::value;
        constexpr int H1 = NMF > 1 ? NMF / 2 : 1, H2 = NMF - H1 > 0 ? NMF - H1 : 1;
        static_for<NMF>([&](auto s) __attribute__((always_inline)) {
            constexpr int S = decltype(s)::value;
            // the columns' fragment first: a lane then holds runs of four columns of one row
            acc[S / NI][S % NI] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x.b[S % NI], x.a[S / NI], acc[S / NI][S % NI], 0, 0, 0);
            static_for<NTASK>([&](auto k) __attribute__((always_inline)) {
                constexpr int Tk = decltype(k)::value;
                constexpr int slot = Tk < NFRONT ? Tk * H1 / NFRONT : NMF > 1 ? H1 + (Tk - NFRONT) * H2 / (NTASK - NFRONT > 0 ? NTASK - NFRONT : 1) : 0;
                if constexpr (slot == S) task(k);
            });
            pin();
        });
    };

    // Stage s lies in ring slot s % NS.  While it is multiplied the next NS - 1 are landing; the last 16 values of a stage are multiplied behind the barrier that
    // publishes the next one, while the slot is filled again.
    static_for<NS>([&](auto s) __attribute__((always_inline)) {
        static_for<L>([&](auto k) __attribute__((always_inline)) { load_task(k, lds + decltype(s)::value * STAGE); });
    });
    wait_vmcnt<L * (NS - 1)>();
    ring_barrier();
    static_for<N_READ>([&](auto k) __attribute__((always_inline)) { read_task(k, f0, lds, 0); });
    auto run_stage = [&](auto s) __attribute__((always_inline)) {
        constexpr int S = decltype(s)::value, S1 = (S + 1) % NS;
        unsigned char *here = lds + S * STAGE;
        static_for<KS - 1>([&](auto k) __attribute__((always_inline)) {
            constexpr int ks = decltype(k)::value;
            mfma_with((ks & 1) ? f1 : f0, IC<N_READ>{}, IC<N_READ>{}, [&](auto r) __attribute__((always_inline)) { read_task(r, (ks & 1) ? f0 : f1, here, ks + 1); });
        });
        wait_lgkmcnt0();                    // this slot has been read
        wait_vmcnt<L * (NS - 2)>();
        ring_barrier();
        mfma_with(f1, IC<N_READ>{}, IC<N_READ + L>{}, [&](auto r) __attribute__((always_inline)) {
            constexpr int Tk = decltype(r)::value;
            if constexpr (Tk < N_READ) read_task(r, f0, lds + S1 * STAGE, 0);
            else load_task(IC<Tk - N_READ>{}, here);
        });
    };
    int kt = 0;
    for (; kt + NS <= stages; kt += NS) static_for<NS>([&](auto s) __attribute__((always_inline)) { run_stage(s); });
    const int rest = stages - kt;
    if (rest >= 1) run_stage(IC<0>{});
    if constexpr (NS > 2) if (rest >= 2) run_stage(IC<1>{});
    if constexpr (NS > 3) if (rest >= 3) run_stage(IC<2>{});

    wait_vmcnt<0>();                        // loads past the end: nothing is under way any more
    wait_lgkmcnt0();
    if (!whole) {
        float4 *to = reinterpret_cast<float4 *>(partial + (size_t)(t.items[MODE].part_first + (unsigned)me.part) * BM * BN);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    to[(((wave * MI + i) * NI + j) * 4 + g) * 64 + lane] = make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
        return;
    }
    typedef Results<MODE, NI> Out;
    const Out out(t, f, cur, last, m0, n0, n0 + wave_n, reinterpret_cast<float *>(lds + wave * Out::BYTES));
    typename Out::With with[2];
    out.fetch(with[0], m0 + wave_m);
    ring_barrier();                         // every wave is done with the operands: their LDS is free
    static_for<MI>([&](auto block) __attribute__((always_inline)) {
        constexpr int i = decltype(block)::value;
        if constexpr (i + 1 < MI) out.fetch(with[(i + 1) % 2], m0 + wave_m + (i + 1) * 32);
        out.put(acc[i], with[i % 2], m0 + wave_m + i * 32);
    });
}

// The sums of split tiles, their pieces added in order: a wave for 32 rows of what was a wave's tile.  64 MB of the 16 split tiles' 256 pieces of 8192 x 8192: 16 us.
constexpr int FINISH = 2;                   // waves of a workgroup
template <int BM, int BN, int WR, int WC, int MODE>
__global__ __launch_bounds__(64 * FINISH) void finish_kernel(const Entry *table, const unsigned *map, int cur, int last, Common f, const float *partial)
{
    constexpr int NW = WR * WC, WM = BM / WR, WN = BN / WC, MI = WM / 32, NI = WN / 32;
    typedef Results<MODE, NI> Out;
    __shared__ __attribute__((aligned(16))) unsigned char lds[FINISH * Out::BYTES];
    const Entry &t = table[map[blockIdx.x]];
    const Items &items = t.items[MODE];
    const int lane = threadIdx.x & 63, half = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned unit = (blockIdx.x - items.finish_first) * FINISH + half, wave = unit / MI % NW, i = unit % MI, q = unit / (MI * NW);
    static_assert(NW * MI % FINISH == 0, "a tile's waves fill workgroups");
    int m0, n0;
    place(t.Rp, t.Cp, t.mp, MODE, BM, items.whole + q, m0, n0);
    const int row0 = m0 + (int)(wave / WC) * WM + (int)i * 32, col0 = n0 + (int)(wave % WC) * WN;
    const Out out(t, f, cur, last, m0, n0, col0, reinterpret_cast<float *>(lds + half * Out::BYTES));
    typename Out::With with;
    out.fetch(with, row0);
    f32x16 acc[NI];
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[j][e] = 0.f;
    const float4 *from = reinterpret_cast<const float4 *>(partial + (size_t)(items.part_first + q * items.split) * BM * BN) + (wave * MI + i) * NI * 256 + lane;
    for (unsigned p = 0; p < items.split; ++p, from += BM * BN / 4) {
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 v = from[(j * 4 + g) * 64];
                acc[j][4 * g] += v.x; acc[j][4 * g + 1] += v.y; acc[j][4 * g + 2] += v.z; acc[j][4 * g + 3] += v.w;
            }
    }
    out.put(acc, with, row0);
}

// Flat matrices: the parts of A, of four stages or more, added in order, and B = b A + c A A and its diagonal of them, a wave for each quarter.  Latency of a launch bounds it.  In place of
// A's sum by one workgroup, or of parts and their addition, and B's launch: 64 x 640 94 -> 81 us, 64 x 4096 137 -> 103, nine of up to 64 x 2304 122 -> 100.
__global__ __launch_bounds__(256) void flat_kernel(const Entry *table, const unsigned *map, const float *partial)
{
    __shared__ __attribute__((aligned(16))) unsigned char sq[8192];
    __shared__ __attribute__((aligned(16))) float diagonal[BK];
    const Entry &t = table[map[blockIdx.x]];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5, ti = wave >> 1, tj = wave & 1, row = ti * 32 + l32;
    auto at = [&](int r, int c) __attribute__((always_inline)) { return sq + r * 128 + ((c ^ (r >> 1 & 7)) << 4); };
    f32x16 acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
    const int parts = (int)t.items[SQUARE_X].split;
    const float4 *from = reinterpret_cast<const float4 *>(partial + (size_t)t.items[SQUARE_X].part_first * BK * BK) + wave * 256 + lane;
    constexpr int AHEAD = 4;
    for (int p0 = 0; p0 < parts; p0 += AHEAD) {
        float4 v[AHEAD][4];
#pragma unroll
        for (int p = 0; p < AHEAD; ++p)
#pragma unroll
            for (int g = 0; g < 4; ++g) v[p][g] = from[(size_t)min(p0 + p, parts - 1) * (BK * BK / 4) + g * 64];
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
            if (p0 + p >= parts) break;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                acc[4 * g] += v[p][g].x; acc[4 * g + 1] += v[p][g].y; acc[4 * g + 2] += v[p][g].z; acc[4 * g + 3] += v[p][g].w;
            }
        }
    }
    f16x4 o[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int c = tj * 32 + 8 * g + 4 * half;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = acc[4 * g + i] * (X_DOWN * X_DOWN);
            if (c + i == row) {
                diagonal[row] = x;
                x = 0.f;
            }
            o[g][i] = (f16_t)(x * S_UP);
        }
        *reinterpret_cast<f16x4 *>(at(row, c / 8) + half * 8) = o[g];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; c += 2) {
        const f16x8 a = *reinterpret_cast<const f16x8 *>(at(row, c + half)), b = *reinterpret_cast<const f16x8 *>(at(tj * 32 + l32, c + half));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(b, a, acc, 0, 0, 0);
    }
    const float di = diagonal[row];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int c = tj * 32 + 8 * g + 4 * half;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float s = acc[4 * g + i] * (S_DOWN * S_DOWN);
            float x = b_of((float)o[g][i] * S_DOWN, di, diagonal[c + i], s);
            if (c + i == row) {
                t.e[row] = e_of(di, s);
                x = 0.f;
            }
            o[g][i] = (f16_t)(x * S_UP);
        }
        *reinterpret_cast<f16x4 *>(t.P + row * BK + c) = o[g];
    }
}

// ---- matrices that a compute unit holds -----------------------------------------------------------------------------------------------------------
//
// All steps in one launch, a workgroup for a matrix of up to 64 by 576 (either way): X's first parts lie in LDS in both orientations, its second ones in the registers of
// the waves that form them; 16-byte chunks of a row are exchanged so that 16 rows of a fetch fall into different banks.  The same operations in the same order as in the
// kernels above, with the same bits.  One 64 x 363 matrix 31 us (95 by 17 launches of those), 4.2 a step and 10 to begin and end: latency of one unit's LDS,
// barriers and instructions, of which the third product and its results take half.

constexpr int SMALL_NT = 1024, SMALL_GROUP = 72;
struct SmallEntry {
    int R, C;
    float step;
    const void *u;
    bf16_t *y;
    float *w, *m;
};
struct SmallGroup {
    SmallEntry t[SMALL_GROUP];
};
static_assert(sizeof(SmallGroup) + sizeof(Common) + 16 <= 4096, "kernel arguments");
template <bool BF16>
__global__ __launch_bounds__(SMALL_NT) void small_kernel(SmallGroup q, Common f, int steps)
{
    constexpr int MOST = SMALL_BLOCKS;
    __shared__ __attribute__((aligned(256))) unsigned char lds[SMALL_M * SMALL_N * 4 + 8192];
    __shared__ __attribute__((aligned(16))) float diagonal[2][SMALL_M];       // d, e
    __shared__ double part_sum[SMALL_NT / 64];
    const SmallEntry &t = q.t[blockIdx.x];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int l32 = lane & 31, half = lane >> 5;
    const bool tall = t.R > t.C;
    const int m = tall ? t.C : t.R, n = tall ? t.R : t.C, np = (n + BK - 1) / BK * BK;
    const int blocks = np / 32 * 2;

    // the matrix's values, in the order of memory, to rows of X in LDS, fp32, 16-byte chunks exchanged so that both 16 rows and 16 fours of rows differ in their banks; and from there a wave's blocks (straight from and to memory, a lane a
    // row: 64 x 363 2 us more, 64 x 576 13)
    typedef typename std::conditional<BF16, bf16_t, float>::type T;
    auto at_x = [&](int r, int c) __attribute__((always_inline)) { return reinterpret_cast<float *>(lds + r * np * 4 + ((c / 4 ^ ((r >> 2 ^ r << 2) & 15)) << 4)) + c % 4; };
    if (!tall) {
        constexpr int PIECES = (SMALL_N + 255) / 256;
        for (int r = wave; r < m; r += 16) {
            Values<BF16, true> q[PIECES];
#pragma unroll
            for (int j = 0; j < PIECES; ++j) q[j].begin(f, (const T *)t.u + r * n, t.m + r * n, lane * 4 + 256 * j, n);
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                const int c = lane * 4 + 256 * j;
                float x[4];
                if (c >= n) continue;
                q[j].end(f, t.m + r * n, c, n, x);
                *reinterpret_cast<float4 *>(at_x(r, c)) = make_float4(x[0], x[1], x[2], x[3]);
            }
        }
    } else {
        const int r = lane % 16 * 4;
        constexpr int AHEAD = 3;
        for (int c0 = wave * 4 + lane / 16; c0 < n; c0 += 64 * AHEAD) {
            Values<BF16, true> q[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) q[j].begin(f, (const T *)t.u + min(c0 + 64 * j, n - 1) * m, t.m + min(c0 + 64 * j, n - 1) * m, r, m);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int c = c0 + 64 * j;
                float x[4];
                if (c >= n || r >= m) continue;
                q[j].end(f, t.m + c * m, r, m, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) *at_x(r + i, c) = x[i];
            }
        }
    }
    __syncthreads();
    float v[MOST][4][4];
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < MOST; ++k)
        if (wave + 16 * k < blocks) {
            const int b = wave + 16 * k, r = b % 2 * 32 + l32;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = b / 2 * 32 + 8 * g + 4 * half;
                const float4 x = *reinterpret_cast<const float4 *>(at_x(r, c));
#pragma unroll
                for (int i = 0; i < 4; ++i) v[k][g][i] = r < m && c + i < n ? (i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w) : 0.f;
            }
            s = squares_of(v[k], s);
        }
    s = wave_total(s);
    if (lane == 0) part_sum[wave] = s;
    __syncthreads();
    s = sixteen_total(part_sum[lane & 15]);
    int up;
    const float by = over_norm(s, up);

    // X [64][np], its transpose [np][64], A and B [64][64], in 16-byte chunks: chunk c of row r lies at chunk c ^ (r / 2 % 8), in X, where np / 64 is even, at c ^ r % 16.  A lane's addresses
    // of a block of 32 x 32 are a few sums and exclusive ors away from these:
    unsigned char *const z = lds, *const zt = lds + SMALL_M * 2 * np, *const sq = lds + SMALL_M * 4 * np;
    const bool odd = np / 64 % 2 != 0, upper = l32 & 1;
    int of_row = l32 * np * 2 + half * 8, swap = odd ? l32 >> 1 & 7 : l32 & 15;                        // X: its row, and what the chunks are exchanged by
    int operand = l32 * 128 + ((half ^ (l32 >> 1 & 7)) << 4);                                          // rows of 64: its chunk of the first 16 values; the others' differ in bits 5 and 6
    int turned = (4 * half + 2 * upper) * 128 + l32 % 8 / 2 * 4 + ((l32 / 8 ^ (2 * half + upper)) << 4);    // transpose: its row and column; bit 6 is that of the block's half and of g
    unsigned first = upper ? 0x01000504u : 0x05040100u, second = upper ? 0x03020706u : 0x07060302u;   // of its own two values and those of the lane beside: the lower row's first
    auto narrow_at = [](unsigned char *base, int r, int c) __attribute__((always_inline)) { return base + r * 128 + ((c ^ (r >> 1 & 7)) << 4); };
    f16x4 hi[MOST][4], lo[MOST][4];
    // 32 rows (upper ones, or the lower) by 8 columns, of which the lane has four of its row
    auto put_z = [&](int b, int g, const f16x4 &x) __attribute__((always_inline)) {
        *reinterpret_cast<f16x4 *>(z + ((of_row + b % 2 * (np * 64) + (((b / 2 * 4) ^ swap) << 4)) ^ (g << 4))) = x;
    };
    // the same turned, into rows of 64 at `to`, the first of them column 0: neighbouring lanes, which have neighbouring rows, give each other two columns, so that either stores two
    // of both rows
    auto put_turned = [&](unsigned char *to, int low, int g, const f16x4 &x) __attribute__((always_inline)) {
        const uint2 w = __builtin_bit_cast(uint2, x);
        const unsigned keep = upper ? w.y : w.x, give = upper ? w.x : w.y;
        const unsigned got = (unsigned)__builtin_amdgcn_update_dpp(0, (int)give, 0xB1, 0xF, 0xF, true);
        unsigned char *const at = to + (turned ^ ((low ^ (g & 1)) << 6)) + g * 1024;
        *reinterpret_cast<unsigned *>(at) = __builtin_amdgcn_perm(got, keep, first);
        *reinterpret_cast<unsigned *>(at + 128) = __builtin_amdgcn_perm(got, keep, second);
    };
    auto put_zt = [&](int b, int g, const f16x4 &x) __attribute__((always_inline)) { put_turned(zt + b / 2 * 4096, b % 2, g, x); };
    auto operand_at = [&](const unsigned char *rows, int c) __attribute__((always_inline)) { return *reinterpret_cast<const f16x8 *>(rows + (operand ^ (c << 4))); };
#pragma unroll
    for (int k = 0; k < MOST; ++k)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int b = wave + 16 * k, c = b / 2 * 32 + 8 * g + 4 * half;
            if (b >= blocks) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = b % 2 * 32 + l32 < m && c + i < n ? in_32_bits(ldexpf(v[k][g][i], -up) * by) : 0.f;       // (zeros outside, also where the norm is NaN)
                hi[k][g][i] = (f16_t)x;
                lo[k][g][i] = rest_of(x, hi[k][g][i]);
            }
            put_z(b, g, hi[k][g]);
            put_zt(b, g, hi[k][g]);
        }
    __syncthreads();

    for (int step = 0; step < steps; ++step) {
        // addresses are worked out of these in each step: all of them at once are more than the registers
        asm volatile("" : "+v"(l32), "+v"(half), "+v"(of_row), "+v"(swap), "+v"(operand), "+v"(turned));
        const bool last = step == steps - 1;
        // A, of which the lower left quarter is the upper right turned: a quarter a wave
        if (wave < 3) {
            const int ti = wave >> 1, tj = (wave + 1) >> 1, row = ti * 32 + l32, pairs = np / 32;
            f32x16 acc;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.f;
            // the operands of 32 values of the reduction are fetched while those before are multiplied
            f16x8 a[2][2], b[2][2];
            auto quarter = [&](auto off_diagonal) __attribute__((always_inline)) {
                constexpr bool OFF = decltype(off_diagonal)::value;
                auto fetch = [&](auto into, int pair) __attribute__((always_inline)) {
                    constexpr int I = decltype(into)::value;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const unsigned char *const at = z + (of_row - half * 8) + ti * (np * 64) + (((pair * 4 + 2 * j + half) ^ swap) << 4);
                        a[I][j] = *reinterpret_cast<const f16x8 *>(at);
                        if (OFF) b[I][j] = *reinterpret_cast<const f16x8 *>(at + np * 64);
                    }
                };
                auto multiply = [&](auto from) __attribute__((always_inline)) {
                    constexpr int I = decltype(from)::value;
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(OFF ? b[I][j] : a[I][j], a[I][j], acc, 0, 0, 0);
                };
                fetch(IC<0>{}, 0);
                for (int pair = 0; pair < pairs; pair += 2) {          // (an even number of them)
                    fetch(IC<1>{}, pair + 1);
                    multiply(IC<0>{});
                    if (pair + 2 < pairs) fetch(IC<0>{}, pair + 2);
                    multiply(IC<1>{});
                }
            };
            if (wave == 1) quarter(std::integral_constant<bool, true>{});
            else quarter(std::integral_constant<bool, false>{});
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = tj * 32 + 8 * g + 4 * half;
                f16x4 o;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = acc[4 * g + i] * (X_DOWN * X_DOWN);
                    if (c + i == row) {
                        diagonal[0][row] = x;
                        x = 0.f;
                    }
                    o[i] = (f16_t)(x * S_UP);
                }
                *reinterpret_cast<f16x4 *>(narrow_at(sq, row, tj * 4 + g) + half * 8) = o;
                if (wave == 1) put_turned(sq + 32 * 128, 0, g, o);
            }
        }
        __syncthreads();
        // B likewise: two waves for each of the three quarters, who multiply the same and finish half of the rows' values each
        const int part = wave & 1, ti = wave >> 2, tj = (wave / 2 + 1) >> 1, row = ti * 32 + l32;
        f16x4 out[2];
        if (wave < 6) {
            f32x16 acc;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll
            for (int c = 0; c < 8; c += 2) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(operand_at(sq + tj * 4096, c), operand_at(sq + ti * 4096, c), acc, 0, 0, 0);
            const float di = diagonal[0][row];
            auto finish = [&](auto from) __attribute__((always_inline)) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    constexpr int G = decltype(from)::value;
                    const int g = G + q, c = tj * 32 + 8 * g + 4 * half;
                    const f16x4 o = *reinterpret_cast<const f16x4 *>(narrow_at(sq, row, tj * 4 + g) + half * 8);
                    const float4 dj = *reinterpret_cast<const float4 *>(&diagonal[0][c]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float s = acc[4 * g + i] * (S_DOWN * S_DOWN);
                        float x = b_of((float)o[i] * S_DOWN, di, i == 0 ? dj.x : i == 1 ? dj.y : i == 2 ? dj.z : dj.w, s);
                        if (c + i == row) {
                            diagonal[1][row] = e_of(di, s);
                            x = 0.f;
                        }
                        out[q][i] = (f16_t)(x * S_UP);
                    }
                }
            };
            if (part) finish(IC<2>{});
            else finish(IC<0>{});
        }
        __syncthreads();                    // O has been read
        if (wave < 6)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                *reinterpret_cast<f16x4 *>(narrow_at(sq, row, tj * 4 + part * 2 + q) + half * 8) = out[q];
                if (ti != tj) put_turned(sq + 32 * 128 + part * 2048, 0, q, out[q]);
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            const int b = wave + 16 * k, r = b % 2 * 32 + l32;
            if (b >= blocks) continue;
            f32x16 acc;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll
            for (int c = 0; c < 8; c += 2) {
                acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(operand_at(zt + b / 2 * 4096, c), operand_at(sq + b % 2 * 4096, c), acc, 0, 0, 0);
            }
            const float e = diagonal[1][r];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = x_of(e, hi[k][g][i], lo[k][g][i], acc[4 * g + i]);
                if (last) {                 // the result stays as it is, in the registers of both parts
                    hi[k][g] = __builtin_bit_cast(f16x4, make_float2(x[0], x[1]));
                    lo[k][g] = __builtin_bit_cast(f16x4, make_float2(x[2], x[3]));
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    hi[k][g][i] = (f16_t)x[i];
                    lo[k][g][i] = rest_of(x[i], hi[k][g][i]);
                }
            }
        }
        __syncthreads();                    // X and B have been read
        if (last) break;
#pragma unroll
        for (int k = 0; k < MOST; ++k)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (wave + 16 * k < blocks) {
                    put_z(wave + 16 * k, g, hi[k][g]);
                    put_zt(wave + 16 * k, g, hi[k][g]);
                }
        __syncthreads();
    }

    // results back to the order of memory
#pragma unroll
    for (int k = 0; k < MOST; ++k)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int b = wave + 16 * k;
            const float2 x = __builtin_bit_cast(float2, hi[k][g]), y = __builtin_bit_cast(float2, lo[k][g]);
            if (b < blocks) *reinterpret_cast<float4 *>(at_x(b % 2 * 32 + l32, b / 2 * 32 + 8 * g + 4 * half)) = make_float4(x.x, x.y, y.x, y.y);
        }
    __syncthreads();
    // four results of a row of len values
    auto put_results = [&](const float (&x)[4], int row, int at, int len) __attribute__((always_inline)) {
        float o[4];
        if (f.muon) {
            Piece<float> w = load_piece(t.w + row * len, at, len);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = w_of(w.get(i), x[i], f.keep, t.step);
            w.set(o);
            store_piece(t.w + row * len, at, len, w);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = x[i] * X_DOWN;
        }
        if (t.y) store_quad(t.y + row * len, at, len, o);
    };
    if (!tall) {
        for (int r = wave; r < m; r += 16)
            for (int c = lane * 4; c < n; c += 256) {
                const float4 x = *reinterpret_cast<const float4 *>(at_x(r, c));
                put_results({x.x, x.y, x.z, x.w}, r, c, n);
            }
    } else if (lane % 16 * 4 < m) {
        const int r = lane % 16 * 4;
        for (int c = wave * 4 + lane / 16; c < n; c += 64) put_results({*at_x(r, c), *at_x(r + 1, c), *at_x(r + 2, c), *at_x(r + 3, c)}, c, r, m);
    }
}

// ---- a call -------------------------------------------------------------------------------------------------------------------------------------

// A shape of tiles
typedef void (*Product)(const Entry *, const Work *, int, int, Common, float *);
typedef void (*Finish)(const Entry *, const unsigned *, int, int, Common, const float *);
struct Shape {
    int bm, bn, threads, per_cu;
    double stage, alone, begin, store;      // us: a stage where all compute units are full, and where each has one workgroup at most; a tile's begin and end; what third ones store besides
    Product product[KINDS];
    Finish finish[KINDS];
    unsigned tiles(const Sizes &s, int kind) const
    {
        if (kind == THIRD) return (unsigned)((s.Rp + bm - 1) / bm) * ((s.Cp + bn - 1) / bn);
        const unsigned T = (s.mp + bm - 1) / bm;
        return T * (T + 1) / 2;
    }
    unsigned finish_groups() const { return (unsigned)(bm / 32) * (bn / wn()) / FINISH; }
    int wn() const { return bn == 64 ? 32 : 64; }
};
// Products whose tiles may be split, so that their parts are added.  The model splits those of X's square at every shape, of A's at 256 alone and thirds at 256 and, for six of all
// pairs of sides in steps of 64, at 128.
template <int...> constexpr Finish no_finish = nullptr;
#define TILES(BM, BN, NS, WR, WC, PER_CU, FINISH_A, FINISH_THIRD, ...)                                                                                               \
    {BM, BN, 64 * WR * WC, PER_CU, __VA_ARGS__,                                                                                                                        \
     {product_kernel<BM, BN, NS, WR, WC, SQUARE_X>, product_kernel<BM, BN, NS, WR, WC, SQUARE_A>, product_kernel<BM, BN, NS, WR, WC, THIRD>}, \
     {finish_kernel<BM, BN, WR, WC, SQUARE_X>, FINISH_A<BM, BN, WR, WC, SQUARE_A>, FINISH_THIRD<BM, BN, WR, WC, THIRD>}}
// (times measured on 512 x 512 to 8192 x 8192; the model is within a tenth of most launches, those of small tiles a quarter.  64 x 64 twice: four stages in LDS for few tiles, which
// wait for their loads, or two and twice the workgroups for many short ones.  42 filters of up to 512: 93 tiles of squares 9.6 and 13 us, 615 of thirds 14.8 and 10.8)
const Shape SHAPES[SHAPE_COUNT] = {TILES(64, 64, 4, 2, 2, 2, no_finish, no_finish, 0.38, 0.26, 4.5, 2), TILES(64, 64, 2, 2, 2, 4, no_finish, no_finish, 0.76, 0.45, 4.5, 2),
                                   TILES(128, 128, 2, 2, 2, 2, no_finish, finish_kernel, 1.0, 0.66, 10, 14), TILES(192, 192, 2, 2, 3, 1, no_finish, no_finish, 1.13, 1.13, 14, 18),
                                   TILES(256, 256, 2, 2, 4, 1, finish_kernel, finish_kernel, 1.35, 1.35, 18, 33)};

// tiles and stages of a reduction
struct Load {
    unsigned tiles;
    int stages;
};
int stages_of(const Sizes &s, int kind) { return (kind == SQUARE_X && s.Rp != s.mp ? s.Rp : kind == SQUARE_X ? s.Cp : s.mp) / BK; }
// Time of a launch of these loads, longest first, each going to the workgroup slots that are free first.  `busy` is for slots and the time they are free at, earliest first.
struct Busy {
    double us;
    unsigned slots;
};
double time_of(const Shape &h, int kind, const Load *loads, int count, std::vector<Busy> &busy)
{
    const unsigned slots = 256 * h.per_cu;
    unsigned total = 0;
    for (int k = 0; k < count; ++k) total += loads[k].tiles;
    const double fill = total < slots ? (double)total / slots : 1.0;
    busy.assign(1, Busy{0.0, slots});
    double last = 0.0;
    for (int k = 0; k < count;) {
        const int stages = loads[k].stages;
        unsigned tiles = 0;
        for (; k < count && loads[k].stages == stages; ++k) tiles += loads[k].tiles;
        while (tiles) {
            const Busy b = busy.front();
            const unsigned n = std::min(tiles, b.slots);
            const double us = b.us + stages * (total > 256 && (b.us == 0.0 || tiles > 256) ? h.stage : h.alone) + h.begin + (kind == THIRD ? h.store * fill : 0.0);
            if (n == b.slots) busy.erase(busy.begin());
            else busy.front().slots -= n;
            size_t at = 0;
            while (at < busy.size() && busy[at].us < us) ++at;
            busy.insert(busy.begin() + at, Busy{us, n});
            last = std::max(last, us);
            tiles -= n;
        }
    }
    return last;
}
// The tiles that a matrix's launch leaves for a last round, or all of few, may be split over the reduction.  This goes by the matrix alone, for it decides the order of sums: a call's
// results do not depend on its other matrices.  8192 x 8192: 528 tiles of 256 on 256 compute units, 620 us; the last 16 of them in 16 pieces each 505.
struct Split {
    int shape;                              // or -1
    unsigned whole, by;
};
Split split_of(const Sizes &s, int kind, std::vector<Busy> &busy)
{
    Split best = {-1, 0, 1};
    double least = 1e30, unsplit = 1e30;
    const int stages = stages_of(s, kind);
    if (s.flat && kind == SQUARE_X) return {0, 0, (unsigned)std::min(16, std::max(1, stages / 4))};
    if (s.flat && kind == SQUARE_A) return {0, 1, 1};
    for (int i = 0; i < SHAPE_COUNT; ++i) {
        const Shape &h = SHAPES[i];
        const Load all = {h.tiles(s, kind), stages};
        const unsigned slots = 256 * h.per_cu, rest = all.tiles % slots;
        unsplit = std::min(unsplit, time_of(h, kind, &all, 1, busy));
        unsigned by = rest ? std::min(slots / rest, 16u) : 1;
        by = std::min(by, (unsigned)stages / 8);
        if (by < 2 || !h.finish[kind]) continue;
        const Load rounds = {all.tiles - rest, stages}, pieces = {rest * by, (int)((stages + by - 1) / by)};
        // the pieces' sums are written and read at some 5 TB/s
        const double us = (rounds.tiles ? time_of(h, kind, &rounds, 1, busy) : 0.0) + time_of(h, 0, &pieces, 1, busy) + 6.0 + pieces.tiles * (h.bm * h.bn * 8.0 / 5e6) + (kind == THIRD ? h.store * rest / slots : 0.0);
        if (us < least) {
            least = us;
            best = {i, all.tiles - rest, by};
        }
    }
    if (unsplit - least < 10.0) best.shape = -1;
    return best;
}

// What a call of these matrices launches
struct Plan {
    std::vector<Items> items[KINDS];
    unsigned count[KINDS][SHAPE_COUNT], finish[KINDS][SHAPE_COUNT], prep, flat;
    size_t parts, bytes;                    // bytes of partial sums; of the workspace
};
Plan plan_of(int count, const int *rows, const int *cols)
{
    Plan p = {};
    std::vector<Sizes> sizes(count);
    std::vector<Split> split(count);
    std::vector<int> order(count);
    std::vector<Load> loads(count);
    std::vector<Busy> busy;
    p.bytes = align_up((size_t)count * sizeof(Entry), 256);
    for (int i = 0; i < count; ++i) {
        sizes[i] = sizes_of(rows[i], cols[i]);
        p.bytes += sizes[i].bytes;
        p.prep += sizes[i].prep;
    }
    p.bytes += align_up((size_t)p.prep * 4, 256);
    for (int kind = 0; kind < KINDS; ++kind) {
        // longest reductions first
        for (int i = 0; i < count; ++i) order[i] = i;
        std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return stages_of(sizes[a], kind) > stages_of(sizes[b], kind); });
        for (int i = 0; i < count; ++i) split[i] = split_of(sizes[i], kind, busy);
        // the others have one shape, that of the least time
        int shape = 0;
        double least = 1e30;
        for (int i = 0; i < SHAPE_COUNT; ++i) {
            int n = 0;
            for (int k = 0; k < count; ++k)
                if (split[order[k]].shape < 0) loads[n++] = {SHAPES[i].tiles(sizes[order[k]], kind), stages_of(sizes[order[k]], kind)};
            const double us = n ? time_of(SHAPES[i], kind, loads.data(), n, busy) : 0.0;
            if (us < least) {
                least = us;
                shape = i;
            }
        }
        p.items[kind].resize(count);
        size_t parts[SHAPE_COUNT] = {};
        for (int k = 0; k < count; ++k) {
            const int i = order[k], at = split[i].shape < 0 ? shape : split[i].shape;
            const Shape &h = SHAPES[at];
            Items &t = p.items[kind][i];
            t = Items{};
            if (sizes[i].flat && kind == SQUARE_A) {        // flat_kernel does it
                t.first = p.flat++;
                continue;
            }
            const unsigned tiles = h.tiles(sizes[i], kind);
            t.first = p.count[kind][at];
            t.whole = split[i].shape < 0 ? tiles : split[i].whole;
            t.split = split[i].by;
            t.count = t.whole + (tiles - t.whole) * t.split;
            t.part_first = (unsigned)parts[at];
            t.finish_first = p.finish[kind][at];
            t.finish_count = sizes[i].flat && kind == SQUARE_X ? 0 : (tiles - t.whole) * h.finish_groups();
            t.shape = (unsigned short)at;
            t.side = (unsigned short)h.bm;
            parts[at] += (tiles - t.whole) * t.split;
            p.finish[kind][at] += t.finish_count;
            p.count[kind][at] += t.count;
        }
        for (int i = 0; i < SHAPE_COUNT; ++i) {
            p.parts = std::max(p.parts, align_up(parts[i] * SHAPES[i].bm * SHAPES[i].bn * 4, 256));
            p.bytes += align_up((size_t)p.count[kind][i] * sizeof(Work), 256) + align_up((size_t)p.finish[kind][i] * 4, 256);
        }
    }
    p.bytes += p.parts + align_up((size_t)p.flat * 4, 256);
    return p;
}
// whether every matrix of a call fits a compute unit: then the call is one launch for SMALL_GROUP of them, without a workspace.  (Beside larger ones they are
// less than a round of the tiles' launches.)
bool all_small(int count, const int *rows, const int *cols)
{
    for (int i = 0; i < count; ++i)
        if (!is_small(rows[i], cols[i])) return false;
    return true;
}
float step_of(const MuonArgs &q, int R, int C) { return (float)(q.lr * (q.rms > 0.0 ? q.rms * sqrt((double)std::max(R, C)) : R > C ? sqrt((double)R / C) : 1.0)); }
int launched() { return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH; }

}  // namespace

// (the plan's lists are the library's only memory of its own; a call that has none is refused)
int muon_workspace(int count, const int *rows, const int *cols, size_t *bytes)
{
    try {
        *bytes = all_small(count, rows, cols) ? 0 : plan_of(count, rows, cols).bytes;
        return MXC_OK;
    } catch (const std::bad_alloc &) {
        return MXC_ERR_LAUNCH;
    }
}

static int run_small(const MuonArgs &q, hipStream_t st)
{
    const Common f = {q.momentum, q.grad_scale, q.keep, q.nesterov, q.w != nullptr, q.dtype == MXC_BF16};
    for (int base = 0; base < q.count; base += SMALL_GROUP) {
        SmallGroup g;
        const int count = std::min(SMALL_GROUP, q.count - base);
        for (int k = 0; k < count; ++k) {
            const int i = base + k;
            g.t[k] = SmallEntry{q.rows[i], q.cols[i], step_of(q, q.rows[i], q.cols[i]), q.u[i], (bf16_t *)(q.w ? (q.w_bf16 ? q.w_bf16[i] : nullptr) : q.y[i]), q.w ? q.w[i] : nullptr,
                                q.w ? q.m[i] : nullptr};
        }
        hipLaunchKernelGGL(f.bf16 ? small_kernel<true> : small_kernel<false>, dim3(count), dim3(SMALL_NT), 0, st, g, f, q.steps);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    }
    return MXC_OK;
}

static int run(const MuonArgs &q, void *ws, size_t ws_bytes, hipStream_t st)
{
    if (all_small(q.count, q.rows, q.cols)) return run_small(q, st);
    const Plan p = plan_of(q.count, q.rows, q.cols);
    if (!ws || ws_bytes < p.bytes) return MXC_ERR_WORKSPACE;
    char *at = (char *)ws;
    auto take = [&](size_t bytes) { char *to = at; at += align_up(bytes, 256); return to; };
    Entry *table = (Entry *)take((size_t)q.count * sizeof(Entry));
    Maps maps;
    maps.prep = (unsigned *)take((size_t)p.prep * 4);
    maps.flat = (unsigned *)take((size_t)p.flat * 4);
    for (int kind = 0; kind < KINDS; ++kind)
        for (int i = 0; i < SHAPE_COUNT; ++i) {
            maps.items[kind][i] = (Work *)take((size_t)p.count[kind][i] * sizeof(Work));
            maps.finish[kind][i] = (unsigned *)take((size_t)p.finish[kind][i] * 4);
        }
    float *partial = (float *)take(p.parts);
    const Common f = {q.momentum, q.grad_scale, q.keep, q.nesterov, q.w != nullptr, q.dtype == MXC_BF16};
    unsigned prep_at = 0;
    for (int base = 0; base < q.count; base += GROUP) {
        Group g;
        g.base = base;
        g.count = q.count - base < GROUP ? q.count - base : GROUP;
        unsigned blocks = 0;
        for (int k = 0; k < g.count; ++k) {
            const int i = base + k, R = q.rows[i], C = q.cols[i];
            const Sizes s = sizes_of(R, C);
            Given &t = g.t[k];
            t.R = R; t.C = C;
            t.step = step_of(q, R, C);
            t.u = q.u[i];
            t.y = (bf16_t *)(q.w ? (q.w_bf16 ? q.w_bf16[i] : nullptr) : q.y[i]);
            t.w = q.w ? q.w[i] : nullptr;
            t.m = q.w ? q.m[i] : nullptr;
            t.room = take(s.bytes);
            t.prep_first = prep_at;
            prep_at += s.prep;
            for (int kind = 0; kind < KINDS; ++kind) t.items[kind] = p.items[kind][i];
            g.first[k] = blocks;
            blocks += s.norm_count;
        }
        g.first[g.count] = blocks;
        hipLaunchKernelGGL(f.bf16 ? norm_kernel<true> : norm_kernel<false>, dim3(blocks), dim3(256), 0, st, g, f, table, maps);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    }
    hipLaunchKernelGGL(f.bf16 ? prepare_kernel<true> : prepare_kernel<false>, dim3(prep_at), dim3(256), 0, st, f, table, maps.prep);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    for (int k = 0; k < q.steps; ++k) {
        const int cur = k & 1, last = k == q.steps - 1;
        for (int mode = SQUARE_X; mode < KINDS; ++mode) {
            for (int i = 0; i < SHAPE_COUNT; ++i) {
                if (!p.count[mode][i]) continue;
                const Shape &h = SHAPES[i];
                hipLaunchKernelGGL(h.product[mode], dim3(p.count[mode][i]), dim3(h.threads), 0, st, table, maps.items[mode][i], cur, last, f, partial);
                if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
                if (mode == SQUARE_X && i == 0 && p.flat) {
                    hipLaunchKernelGGL(flat_kernel, dim3(p.flat), dim3(256), 0, st, table, maps.flat, partial);
                    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
                }
                if (!p.finish[mode][i]) continue;
                hipLaunchKernelGGL(h.finish[mode], dim3(p.finish[mode][i]), dim3(64 * FINISH), 0, st, table, maps.finish[mode][i], cur, last, f, partial);
                if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
            }
        }
    }
    return MXC_OK;
}

int muon_run(const MuonArgs &q, void *ws, size_t ws_bytes, hipStream_t st)
{
    try {
        return run(q, ws, ws_bytes, st);
    } catch (const std::bad_alloc &) {
        return MXC_ERR_LAUNCH;
    }
}

}  // namespace mxc
