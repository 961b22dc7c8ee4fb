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

#include <type_traits>
#include <utility>

#include "mxc_internal.h"

namespace mxc {
namespace {

typedef _Float16 f16_t;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
// powers of two: X at 2^15, the rest of X at 2^26, O and P at 2^14
constexpr float X_UP = 32768.f, X_DOWN = 1.f / 32768.f, LO_UP = 2048.f, LO_DOWN = 1.f / 2048.f, S_UP = 16384.f, S_DOWN = 1.f / 16384.f;

constexpr int BK = 64;                      // reduction of a stage, and what sides are padded to
constexpr int NORM_MOST = 256, NORM_CHUNK = 8192;

// One matrix of a call.  Z is ping-ponged where the third product reads it (tall), its transpose where it does not (wide); the other pair of pointers is one buffer.
struct Entry {
    int R, C, Rp, Cp;                       // rows, columns, and padded to BK
    int mp, tall;                           // the padded shorter side; rows > cols
    int norm_count;                         // workgroups that sum the squares
    float step;                             // w' = keep w - step O
    const void *u;                          // x, or the gradient
    bf16_t *y;                              // y, or the bf16 copy of w
    float *w, *m;
    f16_t *z[2], *zt[2], *lo, *O, *P;
    float *d, *e;
    double *norm;
    unsigned sym_first, prod_first, prep_first, sym_count, prod_count, prep_count;      // tiles of the three kinds of launches
};
constexpr int GROUP = 20;
struct Group {
    Entry t[GROUP];
    unsigned first[GROUP + 1];
    int count, base;
};
struct Common {
    float momentum, grad_scale, keep;
    int nesterov, muon, bf16;
};
static_assert(sizeof(Group) + sizeof(Common) + 64 <= 4096, "kernel arguments");

__device__ __forceinline__ float value_of(const void *p, size_t i, int bf16) { return bf16 ? bf16_to_f32(((const bf16_t *)p)[i]) : ((const float *)p)[i]; }

// ---- sums of squares, the momentum, and the table of the call's matrices ---------------------------------------------------------------------

__global__ __launch_bounds__(256) void norm_kernel(Group q, Common f, Entry *table, unsigned *sym_map, unsigned *prod_map, unsigned *prep_map)
{
    int i = 0;
    while (i + 1 < q.count && blockIdx.x >= q.first[i + 1]) ++i;
    const Entry &t = q.t[i];
    const unsigned part = blockIdx.x - q.first[i];
    if (part == 0 && threadIdx.x == 0) table[q.base + i] = t;
    for (unsigned k = part * 256 + threadIdx.x; k < t.sym_count; k += t.norm_count * 256) sym_map[t.sym_first + k] = q.base + i;
    for (unsigned k = part * 256 + threadIdx.x; k < t.prod_count; k += t.norm_count * 256) prod_map[t.prod_first + k] = q.base + i;
    for (unsigned k = part * 256 + threadIdx.x; k < t.prep_count; k += t.norm_count * 256) prep_map[t.prep_first + k] = q.base + i;
    const size_t n = (size_t)t.R * t.C;
    double s = 0.0;
    for (size_t k = (size_t)part * 256 + threadIdx.x; k < n; k += (size_t)t.norm_count * 256) {
        float u = value_of(t.u, k, f.bf16);
        if (f.muon) {
            u *= f.grad_scale;
            const float m = t.m[k] * f.momentum + u;
            t.m[k] = m;
            u = f.nesterov ? u + m * f.momentum : m;
        }
        s += (double)u * (double)u;
    }
    __shared__ double wave_sum[4];
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) t.norm[part] = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
}

// ---- X over its norm, in both orientations: a workgroup for 64 x 64 values -----------------------------------------------------------------------

__global__ __launch_bounds__(256) void prepare_kernel(Common f, const Entry *table, const unsigned *map)
{
    const Entry &t = table[map[blockIdx.x]];
    const unsigned tile = blockIdx.x - t.prep_first, across = t.Cp / 64;
    const int r0 = tile / across * 64, c0 = tile % across * 64;
    __shared__ f16_t turned[64][66];
    __shared__ double wave_sum[4];
    double s = (int)threadIdx.x < t.norm_count ? t.norm[threadIdx.x] : 0.0;
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) wave_sum[threadIdx.x >> 6] = s;
    __syncthreads();
    s = wave_sum[0] + wave_sum[1] + wave_sum[2] + wave_sum[3];
    // a value that is not finite makes NaN of the whole matrix; zeros stay zeros
    const double by = !(s < 1e300) ? __builtin_nan("") : s > 0.0 ? (double)X_UP / sqrt(s) : 0.0;
    const int c = c0 + (threadIdx.x & 63);
    for (int k = threadIdx.x >> 6; k < 64; k += 4) {
        const int r = r0 + k;
        double x = 0.0;
        if (r < t.R && c < t.C) {
            const size_t at = (size_t)r * t.C + c;
            float u;
            if (f.muon && !f.nesterov) u = t.m[at];
            else {
                u = value_of(t.u, at, f.bf16);
                if (f.muon) {
                    u *= f.grad_scale;
                    u += t.m[at] * f.momentum;
                }
            }
            x = (double)u * by;
        }
        const f16_t hi = (f16_t)(float)x, lo = (f16_t)(float)((x - (double)(float)hi) * (double)LO_UP);
        const size_t to = (size_t)r * t.Cp + c;
        t.z[0][to] = hi;
        t.lo[to] = lo;
        turned[threadIdx.x & 63][k] = hi;
    }
    __syncthreads();
    for (int k = threadIdx.x >> 6; k < 64; k += 4) t.zt[0][(size_t)(c0 + k) * t.Rp + r0 + (threadIdx.x & 63)] = turned[k][threadIdx.x & 63];
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

// Tiles of BM x BN by WR x WC waves.  The reduction runs through a ring of NS stages of 64 values in LDS, filled by loads that go there directly and are issued
// NS stages ahead; 16-byte chunk k of a row lies at chunk k ^ (row / 2 % 8), which spreads the operand fetches over the banks.
template <int BM, int BN, int NS, int WR, int WC, int MODE>
__global__ __launch_bounds__(64 * WR * WC) void product_kernel(const Entry *table, const unsigned *map, int cur, int last, Common f)
{
    constexpr int NW = WR * WC, WM = BM / WR, WN = BN / WC, MI = WM / 32, NI = WN / 32, NMF = MI * NI;
    constexpr int RPL = 8, A_LD = BM / RPL / NW, B_LD = BN / RPL / NW, L = A_LD + B_LD, KS = BK / 16;
    constexpr int STAGE = (BM + BN) * BK * 2, PITCH = WN + 4, STAGING = NW * 32 * PITCH * 4;
    static_assert(BM % (RPL * NW) == 0 && BN % (RPL * NW) == 0 && KS % 2 == 0 && L * (NS - 1) < 64, "tile");
    constexpr int LDS = STAGE * NS > STAGING ? STAGE * NS : STAGING;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[LDS];

    const Entry &t = table[map[blockIdx.x]];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_m = wave / WC * WM, wave_n = wave % WC * WN;
    const bool tall = t.tall != 0;
    const int mp = t.mp;

    const f16_t *a, *b;
    int K, a_rows, b_rows;
    unsigned ti, tj;
    if (MODE == THIRD) {
        const unsigned tile = blockIdx.x - t.prod_first, across = (t.Cp + BN - 1) / BN;
        ti = tile / across;
        tj = tile % across;
        a = tall ? t.z[cur] : t.P;
        b = tall ? t.P : t.zt[cur];
        K = mp;
        a_rows = t.Rp;
        b_rows = t.Cp;
    } else {
        static_assert(MODE == THIRD || BM == BN, "a symmetric result has square tiles");
        triangle(blockIdx.x - t.sym_first, (mp + BM - 1) / BM, ti, tj);
        a = MODE == SQUARE_A ? t.O : tall ? t.zt[cur] : t.z[cur];
        b = a;
        K = MODE == SQUARE_A ? mp : tall ? t.Rp : t.Cp;
        a_rows = b_rows = mp;
    }
    const int m0 = ti * BM, n0 = tj * BN;

    // rows past the operand's lie past the resource's end: their loads give zeros
    const buf_rsrc_t rs_a = make_buf_rsrc(a, (unsigned)a_rows * (unsigned)K * 2u), rs_b = make_buf_rsrc(b, (unsigned)b_rows * (unsigned)K * 2u);
    const int ld_row = lane / 8, ld_chunk = (lane % 8) ^ ((4 * wave + ld_row / 2) % 8);
    unsigned va[A_LD], vb[B_LD];
#pragma unroll
    for (int i = 0; i < A_LD; ++i) va[i] = (unsigned)(m0 + RPL * (wave + NW * i) + ld_row) * (unsigned)K * 2u + ld_chunk * 16;
#pragma unroll
    for (int i = 0; i < B_LD; ++i) vb[i] = (unsigned)(n0 + RPL * (wave + NW * i) + ld_row) * (unsigned)K * 2u + ld_chunk * 16;
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
    const int stages = K / BK;
    int kt = 0;
    for (; kt + NS <= stages; kt += NS) static_for<NS>([&](auto s) __attribute__((always_inline)) { run_stage(s); });
    const int rest = stages - kt;
    if (rest >= 1) run_stage(IC<0>{});
    if constexpr (NS > 2) if (rest >= 2) run_stage(IC<1>{});
    if constexpr (NS > 3) if (rest >= 3) run_stage(IC<2>{});
    wait_vmcnt<0>();                        // loads past the end: nothing is under way any more
    wait_lgkmcnt0();
    __syncthreads();

    // ---- results: 32 rows of the wave's tile at a time through LDS, as fp32, in rows and then in columns ------------------------------------------------
    float *stage = reinterpret_cast<float *>(lds) + wave * 32 * PITCH;
    constexpr int CPR = WN / 8, ROWS = 64 / CPR;           // chunks of 8 columns in a row; rows that 64 lanes cover
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int row0 = m0 + wave_m + i * 32, col0 = n0 + wave_n;
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(stage + frag_row * PITCH + j * 32 + 8 * g + 4 * frag_k) =
                    make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
        wave_sync();
#pragma unroll
        for (int k = 0; k < 32; k += ROWS) {
            const int r = k + lane / CPR, c = lane % CPR * 8, row = row0 + r, col = col0 + c;
            float v[8];
            *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(stage + r * PITCH + c);
            *reinterpret_cast<float4 *>(v + 4) = *reinterpret_cast<const float4 *>(stage + r * PITCH + c + 4);
            const bool in = MODE == THIRD ? row < t.Rp && col < t.Cp : row < mp && col < mp;
            f16x8 out;
            if (in) {
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
                    const f16x8 o = *reinterpret_cast<const f16x8 *>(t.O + (size_t)row * mp + col);
                    const float di = t.d[row];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float s = v[q] * (S_DOWN * S_DOWN), dj = t.d[col + q], oq = (float)o[q] * S_DOWN;
                        v[q] = NS_B * oq + NS_C * ((di + dj) * oq + s);
                        if (col + q == row) {
                            t.e[row] = NS_B * di + NS_C * (di * di + s);
                            v[q] = 0.f;
                        }
                        out[q] = (f16_t)(v[q] * S_UP);
                    }
                    *reinterpret_cast<f16x8 *>(t.P + (size_t)row * mp + col) = out;
                } else {
                    const size_t at = (size_t)row * t.Cp + col;
                    const f16x8 hi = *reinterpret_cast<const f16x8 *>(t.z[cur] + at), lo = *reinterpret_cast<const f16x8 *>(t.lo + at);
                    const float er = tall ? 0.f : t.e[row];
                    f16x8 low;
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float e = tall ? t.e[col + q] : er;
                        v[q] = (NS_A + e) * ((float)hi[q] + (float)lo[q] * LO_DOWN) + v[q] * S_DOWN;       // at 2^15, as X is
                        out[q] = (f16_t)v[q];
                        low[q] = (f16_t)((v[q] - (float)out[q]) * LO_UP);
                    }
                    if (!last) {
                        *reinterpret_cast<f16x8 *>(t.z[cur ^ 1] + at) = out;
                        *reinterpret_cast<f16x8 *>(t.lo + at) = low;
                    } else if (row < t.R) {
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            if (col + q >= t.C) break;
                            const size_t to = (size_t)row * t.C + col + q;
                            if (f.muon) {
                                const float w = t.w[to] * f.keep - t.step * (v[q] * X_DOWN);
                                t.w[to] = w;
                                if (t.y) t.y[to] = (bf16_t)pack_bf16x2(w, 0.f);
                            } else {
                                t.y[to] = (bf16_t)pack_bf16x2(v[q] * X_DOWN, 0.f);
                            }
                        }
                    }
                }
                // the values as stored, for the other orientation
                if (MODE == THIRD ? !last : ti != tj) {
                    *reinterpret_cast<float4 *>(stage + r * PITCH + c) = make_float4((float)out[0], (float)out[1], (float)out[2], (float)out[3]);
                    *reinterpret_cast<float4 *>(stage + r * PITCH + c + 4) = make_float4((float)out[4], (float)out[5], (float)out[6], (float)out[7]);
                }
            }
        }
        wave_sync();
        if (MODE == THIRD ? !last : ti != tj) {
            f16_t *to = MODE == THIRD ? t.zt[cur ^ 1] : MODE == SQUARE_X ? t.O : t.P;
            const int pitch = MODE == THIRD ? t.Rp : mp, rows = MODE == THIRD ? t.Rp : mp, cols = MODE == THIRD ? t.Cp : mp;
#pragma unroll
            for (int k = 0; k < WN; k += 16) {
                const int c = k + lane / 4, r = lane % 4 * 8;
                f16x8 out;
#pragma unroll
                for (int q = 0; q < 8; ++q) out[q] = (f16_t)stage[(r + q) * PITCH + c];
                if (row0 + r < rows && col0 + c < cols) *reinterpret_cast<f16x8 *>(to + (size_t)(col0 + c) * pitch + row0 + r) = out;
            }
            wave_sync();
        }
    }
}

// ---- a call -------------------------------------------------------------------------------------------------------------------------------------

struct Sizes {
    int Rp, Cp, mp, norm_count;
    size_t mat, sq;                         // bytes of one orientation of X, of A
    unsigned sym, prod, prep;
    size_t bytes;
};
constexpr int TILE = 128;
Sizes sizes_of(int R, int C)
{
    Sizes s;
    s.Rp = (int)align_up(R, BK);
    s.Cp = (int)align_up(C, BK);
    s.mp = R <= C ? s.Rp : s.Cp;
    const size_t n = (size_t)R * C, chunks = (n + NORM_CHUNK - 1) / NORM_CHUNK;
    s.norm_count = chunks < NORM_MOST ? (int)chunks : NORM_MOST;
    s.mat = align_up((size_t)s.Rp * s.Cp * 2, 256);
    s.sq = align_up((size_t)s.mp * s.mp * 2, 256);
    const unsigned T = (s.mp + TILE - 1) / TILE;
    s.sym = T * (T + 1) / 2;
    s.prod = (unsigned)((s.Rp + TILE - 1) / TILE) * ((s.Cp + TILE - 1) / TILE);
    s.prep = (unsigned)(s.Rp / 64) * (s.Cp / 64);
    s.bytes = 4 * s.mat + 2 * s.sq + 2 * align_up((size_t)s.mp * 4, 256) + NORM_MOST * 8;
    return s;
}
int launched() { return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH; }

}  // namespace

size_t muon_workspace(int count, const int *rows, const int *cols)
{
    size_t bytes = align_up((size_t)count * sizeof(Entry), 256), sym = 0, prod = 0, prep = 0;
    for (int i = 0; i < count; ++i) {
        const Sizes s = sizes_of(rows[i], cols[i]);
        bytes += s.bytes;
        sym += s.sym;
        prod += s.prod;
        prep += s.prep;
    }
    return bytes + align_up(sym * 4, 256) + align_up(prod * 4, 256) + align_up(prep * 4, 256);
}

int muon_run(const MuonArgs &q, void *ws, hipStream_t st)
{
    char *at = (char *)ws;
    auto take = [&](size_t bytes) { char *p = at; at += align_up(bytes, 256); return p; };
    size_t sym = 0, prod = 0, prep = 0;
    for (int i = 0; i < q.count; ++i) {
        const Sizes s = sizes_of(q.rows[i], q.cols[i]);
        sym += s.sym;
        prod += s.prod;
        prep += s.prep;
    }
    Entry *table = (Entry *)take((size_t)q.count * sizeof(Entry));
    unsigned *sym_map = (unsigned *)take(sym * 4), *prod_map = (unsigned *)take(prod * 4), *prep_map = (unsigned *)take(prep * 4);
    const Common f = {q.momentum, q.grad_scale, q.keep, q.nesterov, q.w != nullptr, q.dtype == MXC_BF16};
    unsigned sym_at = 0, prod_at = 0, prep_at = 0;
    for (int base = 0; base < q.count; base += GROUP) {
        Group g;
        g.base = base;
        g.count = q.count - base < GROUP ? q.count - base : GROUP;
        unsigned blocks = 0;
        for (int k = 0; k < g.count; ++k) {
            const int i = base + k, R = q.rows[i], C = q.cols[i];
            const Sizes s = sizes_of(R, C);
            Entry &t = g.t[k];
            t.R = R; t.C = C; t.Rp = s.Rp; t.Cp = s.Cp; t.mp = s.mp; t.tall = R > C; t.norm_count = s.norm_count;
            t.step = (float)(q.lr * (q.rms > 0.0 ? q.rms * sqrt((double)(R > C ? R : C)) : R > C ? sqrt((double)R / C) : 1.0));
            t.u = q.u[i];
            t.y = (bf16_t *)(q.w ? (q.w_bf16 ? q.w_bf16[i] : nullptr) : q.y[i]);
            t.w = q.w ? q.w[i] : nullptr;
            t.m = q.w ? q.m[i] : nullptr;
            t.z[0] = (f16_t *)take(s.mat);
            t.zt[0] = (f16_t *)take(s.mat);
            f16_t *second = (f16_t *)take(s.mat);
            t.z[1] = t.tall ? second : t.z[0];
            t.zt[1] = t.tall ? t.zt[0] : second;
            t.lo = (f16_t *)take(s.mat);
            t.O = (f16_t *)take(s.sq);
            t.P = (f16_t *)take(s.sq);
            t.d = (float *)take((size_t)s.mp * 4);
            t.e = (float *)take((size_t)s.mp * 4);
            t.norm = (double *)take(NORM_MOST * 8);
            t.sym_first = sym_at; t.prod_first = prod_at; t.prep_first = prep_at;
            t.sym_count = s.sym; t.prod_count = s.prod; t.prep_count = s.prep;
            sym_at += s.sym; prod_at += s.prod; prep_at += s.prep;
            g.first[k] = blocks;
            blocks += s.norm_count;
        }
        g.first[g.count] = blocks;
        hipLaunchKernelGGL(norm_kernel, dim3(blocks), dim3(256), 0, st, g, f, table, sym_map, prod_map, prep_map);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    }
    hipLaunchKernelGGL(prepare_kernel, dim3(prep_at), dim3(256), 0, st, f, table, prep_map);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    for (int k = 0; k < q.steps; ++k) {
        const int cur = k & 1, last = k == q.steps - 1;
        hipLaunchKernelGGL((product_kernel<TILE, TILE, 2, 2, 2, SQUARE_X>), dim3(sym_at), dim3(256), 0, st, table, sym_map, cur, last, f);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
        hipLaunchKernelGGL((product_kernel<TILE, TILE, 2, 2, 2, SQUARE_A>), dim3(sym_at), dim3(256), 0, st, table, sym_map, cur, last, f);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
        hipLaunchKernelGGL((product_kernel<TILE, TILE, 2, 2, 2, THIRD>), dim3(prod_at), dim3(256), 0, st, table, prod_map, cur, last, f);
        if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    }
    return MXC_OK;
}

}  // namespace mxc
