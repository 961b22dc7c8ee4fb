// Embedding: y[n] = scale * w[tokens[n]], and the gradient of the table, dw[v] = scale * sum of dy[n] over the places n where tokens[n] == v.
// Memory bounds both: forward reads and writes each row once; the gradient reads dy once and writes a row of dw for every
// token of the vocabulary.  The gradient of more than a few places goes by the tokens' order, in three launches: the places are sorted by their token, each token's rows added, in
// parts, and the parts of a token that has several joined.  16384 rows of 4096 bf16 41.6 us, 6.5 TB/s (64 rows 3.9, a launch); gradient of 32768 places on 50257 x 2048, bf16,
// 137 us; of 500 places on 1000 x 512 fp32, added to it, in one launch, 5.2.
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

// four results: row[c, c + 4) = scale * s, or that added
template <bool PAST>
__device__ __forceinline__ void put(float *row, int c, int C, const float (&s)[4], float scale, bool add)
{
    Piece<float> p;
    float v[4];
    if (add) {
        p = load_piece(row, c, C);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = p.get(i) + s[i] * scale;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = s[i] * scale;
    }
    p.set(v);
    store_piece<PAST>(row, c, C, p);
}

// s += columns [c, c + 4) of rows places[0, count), in their order, AHEAD rows on their way at once
template <int AHEAD, class T>
__device__ __forceinline__ void add_rows(const T *dy, int c, int C, const int *places, int count, float (&s)[4])
{
    int k = 0;
    for (; k + AHEAD <= count; k += AHEAD) {
        decltype(begin_quad(dy, 0, 0)) p[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) p[j] = begin_quad(dy + (size_t)places[k + j] * C, c, C);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            settle_quad(p[j], c, C);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += p[j].get(i);
        }
    }
    if constexpr (AHEAD > 1) add_rows<AHEAD / 4>(dy, c, C, places + k, count - k, s);
}

// zeros for those of rows [v0, v0 + rows) of which clear() is true, by a workgroup: long rows one after the other, short ones together
template <bool PAST, class F>
__device__ __forceinline__ void clear_rows(float *dw, int v0, int rows, int C, F &&clear)
{
    const float zeros[4] = {0.f, 0.f, 0.f, 0.f};
    if (C > 256) {
        for (int r = 0; r < rows; ++r)
            if (clear(r))
                for (int c = threadIdx.x * 4; c < C; c += NT * 4) put<PAST>(dw + (size_t)(v0 + r) * C, c, C, zeros, 1.f, false);
    } else {
        const unsigned quads = (unsigned)(C + 3) / 4;
        for (int i = threadIdx.x; i < rows * (int)quads; i += NT) {
            const int r = (int)((unsigned)i / quads);
            if (clear(r)) put<PAST>(dw + (size_t)(v0 + r) * C, (i - r * (int)quads) * 4, C, zeros, 1.f, false);
        }
    }
}

// Groups of L = 1 << log_lanes threads hold sums of the same 4 L columns; those of the first group become the sums of all.
__device__ __forceinline__ void add_groups(float (&s)[4], float4 *room, int log_lanes)
{
    room[threadIdx.x] = make_float4(s[0], s[1], s[2], s[3]);
    __syncthreads();
    if (threadIdx.x >> log_lanes) return;
    for (unsigned k = threadIdx.x + (1 << log_lanes); k < NT; k += 1 << log_lanes) {
        const float4 o = room[k];
        s[0] += o.x; s[1] += o.y; s[2] += o.z; s[3] += o.w;
    }
}
// lanes of a group: 16 to 64, as the columns need
int group_lanes(int C) { return C <= 64 ? 4 : C <= 128 ? 5 : 6; }

// Few places, one launch: the workgroup of a place looks for its token among all places and, if the place is the first that has it, adds their rows,
// of which each group of L threads takes a run; workgroups behind them look which of ZERO_ROWS rows of dw have no place and clear these.
constexpr int FEW = 2048, ZERO_ROWS = 64;
template <class T, bool PAST>
__global__ __launch_bounds__(NT) void few_kernel(int N, int V, int C, int log_lanes, const int *tokens, const T *dy, float scale, int add, float *dw)
{
    __shared__ int places[FEW];
    __shared__ float4 room[NT];
    constexpr int TURNS = FEW / NT, nt = NT;
    __shared__ int wave_count[TURNS * (NT / 64)];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
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
        const int of = (ZERO_ROWS + (int)gridDim.y - 1) / (int)gridDim.y, r0 = (int)blockIdx.y * of, rows = (int)min((long long)min(of, ZERO_ROWS - r0), V - v0 - r0);
        clear_rows<PAST>(dw, (int)v0 + r0, rows, C, [&](int r) __attribute__((always_inline)) { return !found[r0 + r]; });
        return;
    }
    const int me = blockIdx.x;
    int other[TURNS];
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
        const int n = j * NT + threadIdx.x;
        other[j] = n < N ? tokens[n] : -1;
    }
    const int t = tokens[me];
    if ((unsigned)t >= (unsigned)V) return;
    bool earlier = false;
    unsigned long long same[TURNS];
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
        same[j] = __ballot(other[j] == t);
        earlier |= other[j] == t && j * NT + (int)threadIdx.x < me;
        if (lane == 0) wave_count[j * (NT / 64) + wave] = __popcll(same[j]);
    }
    if (__syncthreads_or(earlier)) return;
    int count = 0;
#pragma unroll
    for (int j = 0; j < TURNS; ++j) {
        int at = count;
        for (int k = 0; k < NT / 64; ++k) {
            at += k < wave ? wave_count[j * (NT / 64) + k] : 0;
            count += wave_count[j * (NT / 64) + k];
        }
        if (other[j] == t) places[at + __popcll(same[j] & ((1ull << lane) - 1))] = j * NT + threadIdx.x;
    }
    __syncthreads();
    const int L = 1 << log_lanes, c = ((int)blockIdx.y * L + (threadIdx.x & (L - 1))) * 4, share = (count + (NT >> log_lanes) - 1) / (NT >> log_lanes);
    const int k0 = min(count, (int)(threadIdx.x >> log_lanes) * share), k1 = min(count, k0 + share);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    add_rows<16>(dy, c < C ? c : 0, C, places + k0, k1 - k0, s);
    if (count > 1) add_groups(s, room, log_lanes);
    if (threadIdx.x < (unsigned)L && c < C) put<PAST>(dw + (size_t)t * C, c, C, s, scale, add);
}

// The places in the order of their tokens (of equal tokens in their own), and where each token's begin.  Workgroup (x, y) puts the places of segment y
// whose token is among the R tokens of range x; for where they go it counts all places first.  Each of its waves has a share of the segment and a counter of its own for each
// token, so that no wave waits for another on the way; lanes of one token find each other by the ballots of its bits.  LDS bounds it, where the common tokens are: 32768 places of 50257
// tokens 15.6 us, of which the range of the 786 most common ones takes all and another 8.
constexpr int ORDER_NT = 1024, ORDER_WAVES = ORDER_NT / 64, ORDER_MOST = 2048, BATCH = 16, OTHERS = 24;
template <int MOST>
__global__ __launch_bounds__(ORDER_NT) void order_kernel(int N, int V, int R, int segment, const int *tokens, int *order, int *start)
{
    __shared__ int counts[(ORDER_WAVES + 2) * MOST];         // [ORDER_WAVES][R] of this segment, [R] of earlier ones, [R] of later ones
    __shared__ int wave_sum[ORDER_WAVES], wave_before[ORDER_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    const int lo = blockIdx.x * R, here = min(R, V - lo);
    for (int i = threadIdx.x; i < (ORDER_WAVES + 2) * R; i += ORDER_NT) counts[i] = 0;
    __syncthreads();
    int *own = counts + wave * R;
    // places of a wave in its segment: a multiple of 64
    const int share = (segment + ORDER_NT - 1) / ORDER_NT * 64;
    const long long seg0 = (long long)blockIdx.y * segment, seg1 = min((long long)N, seg0 + segment);
    const long long n0 = min(seg1, seg0 + (long long)wave * share), n1 = min(seg1, n0 + share);
    int before = 0;
    auto count = [&](int t, int *into) __attribute__((always_inline)) {
        before += __popcll(__ballot((unsigned)t < (unsigned)lo));
        const unsigned d = (unsigned)t - (unsigned)lo;              // (a negative token is past every range: V - lo < 2^24)
        if (d < (unsigned)here) atomicAdd(into + d, 1);
    };
    // this wave's first places, which stay in registers, are on their way while those of the other segments are counted
    int mine[BATCH];
    auto load_mine = [&](long long m) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const long long n = m + 64 * j + lane;
            mine[j] = n < n1 ? tokens[n] : -1;
        }
    };
    load_mine(n0);
    const long long others = N - (seg1 - seg0);
    for (long long m0 = 0; m0 < others; m0 += (long long)ORDER_NT * OTHERS) {
        const long long m = m0 + threadIdx.x;
        int t[OTHERS];
#pragma unroll
        for (int j = 0; j < OTHERS; ++j) {
            const long long i = m + (long long)ORDER_NT * j;
            t[j] = i < others ? tokens[i < seg0 ? i : i + (seg1 - seg0)] : -1;
        }
#pragma unroll
        for (int j = 0; j < OTHERS; ++j) count(t[j], counts + (ORDER_WAVES + (m + (long long)ORDER_NT * j < seg0 ? 0 : 1)) * R);
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) count(mine[j], own);
    for (long long m = n0 + 64 * BATCH; m < n1; m += 64 * BATCH) {
        load_mine(m);
#pragma unroll
        for (int j = 0; j < BATCH; ++j) count(mine[j], own);
    }
    if (lane == 0) wave_before[wave] = before;
    __syncthreads();
    int base = 0;
    for (int k = 0; k < ORDER_WAVES; ++k) base += wave_before[k];
    // from counts to where a wave's places of a token go: OF tokens a thread
    constexpr int OF = MOST > ORDER_NT ? MOST / ORDER_NT : 1;
    const int t0 = threadIdx.x * OF;
    int total[OF], sum = 0;
#pragma unroll
    for (int j = 0; j < OF; ++j) {
        total[j] = 0;
        if (t0 + j < here)
#pragma unroll
            for (int k = 0; k < ORDER_WAVES + 2; ++k) total[j] += counts[k * R + t0 + j];
        sum += total[j];
    }
    int up = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(up, d);
        up += lane >= d ? v : 0;
    }
    if (lane == 63) wave_sum[wave] = up;
    __syncthreads();
    for (int k = 0; k < wave; ++k) base += wave_sum[k];
    base += up - sum;
#pragma unroll
    for (int j = 0; j < OF; ++j) {
        if (t0 + j >= here) break;
        if (blockIdx.y == 0) {
            start[lo + t0 + j] = base;
            if (lo + t0 + j == V - 1) start[V] = base + total[j];
        }
        int at = base + counts[ORDER_WAVES * R + t0 + j];
#pragma unroll
        for (int k = 0; k < ORDER_WAVES; ++k) {
            const int c = counts[k * R + t0 + j];
            counts[k * R + t0 + j] = at;
            at += c;
        }
        base += total[j];
    }
    __syncthreads();
    const int bits = 32 - __clz(R);
    for (long long m = n0; m < n1; m += 64 * BATCH) {
        if (n1 - n0 > 64 * BATCH) load_mine(m);
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            const unsigned d = (unsigned)mine[j] - (unsigned)lo;
            const bool in = d < (unsigned)here;
            unsigned long long same = __ballot(in);
            if (same == 0) continue;
            // the lanes that have the same token: those that agree in every bit
            for (int b = 0; b < bits; ++b) {
                const bool one = d >> b & 1;
                const unsigned long long ones = __ballot(one);
                same &= one ? ones : ~ones;
            }
            if (in) {
                const int to = own[d], rank = __popcll(same & ((1ull << lane) - 1));
                order[to + rank] = (int)(m + 64 * j) + lane;
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                if (rank == 0) own[d] = to + __popcll(same);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
}

// Sums of each token's rows: a wave for PART (16 to 64) places of the order and 256 columns.  Its lanes hold the places and their tokens, so that all control is the wave's; it loads the
// rows of 16 places at once and adds them one after the other, and where the token changes the sum is the token's row of dw, or, of a token that has places in other
// parts too, this part's share: slot 0 for the token of the part's first place, slot 1 for one that begins within it.  Workgroups behind the parts' clear the rows of
// tokens that stand nowhere (between the parts', 4 % slower).  32768 places on 50257 x 2048 from memory, bf16: 117 us of the gradient's 137, 4.7 TB/s.
constexpr int BLOCK = 256;
template <class T, bool PAST>
__global__ __launch_bounds__(NT) void rows_kernel(int V, int C, int PART, long long part_waves, unsigned part_groups, int empty_rows, const int *tokens,
                                                 const int *order, const int *start, const T *dy, float scale, int add, float *dw, float *parts)
{
    constexpr int AHEAD = 16;
    const int lane = threadIdx.x & 63;
    if (blockIdx.x >= part_groups) {
        const int v0 = (int)(blockIdx.x - part_groups) * empty_rows, rows = min(empty_rows, V - v0);
        const unsigned long long empty = __ballot(lane < rows && start[v0 + min(lane, rows - 1)] == start[v0 + min(lane, rows - 1) + 1]);
        clear_rows<PAST>(dw, v0, rows, C, [&](int r) __attribute__((always_inline)) { return (empty >> r & 1) != 0; });
        return;
    }
    const long long w = (long long)blockIdx.x * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= part_waves) return;
    const int blocks = (C + BLOCK - 1) / BLOCK, part = (int)(w / blocks), c = ((int)(w - (long long)part * blocks) * 64 + lane) * 4;
    const int all = __builtin_amdgcn_readfirstlane(start[V]), p0 = part * PART, count = min(PART, all - p0);
    if (count <= 0) return;
    // past the last place: the last one's row again, under a token of its own
    const int o = order[p0 + min(lane, count - 1)], t = lane < count ? tokens[o] : -1;
    const int ahead = p0 > 0 ? tokens[order[p0 - 1]] : -1, behind = p0 + count < all ? tokens[order[p0 + count]] : -1;
    const bool has = c < C;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    int now = __builtin_amdgcn_readlane(t, 0), slot = 0;
    bool whole = __builtin_amdgcn_readfirstlane(ahead) != now;          // the token's places begin in this part
    for (int k = 0; k < count; k += AHEAD) {
        decltype(begin_quad(dy, 0, 0)) p[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) p[j] = begin_quad(dy + (size_t)__builtin_amdgcn_readlane(o, k + j) * C, has ? c : 0, C);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            settle_quad(p[j], has ? c : 0, C);
            const int next = __builtin_amdgcn_readlane(t, k + j);
            if (next != now) {
                if (now >= 0 && has) {
                    if (whole) put<PAST>(dw + (size_t)now * C, c, C, s, scale, add);
                    else put<false>(parts + (size_t)(2 * part) * C, c, C, s, 1.f, false);
                }
                now = next;
                slot = 1;
                whole = true;
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += p[j].get(i);
        }
    }
    if (now >= 0 && has) {          // (a part of fewer places has ended its last token above)
        if (whole && __builtin_amdgcn_readfirstlane(behind) != now) put<PAST>(dw + (size_t)now * C, c, C, s, scale, add);
        else put<false>(parts + (size_t)(2 * part + slot) * C, c, C, s, 1.f, false);
    }
}

// A part in which a token begins that ends in another adds up that token's shares: a workgroup for 4 L columns, whose groups of L threads take a run of the shares each.
__global__ __launch_bounds__(NT) void join_kernel(int V, int C, int PART, int log_lanes, const int *tokens, const int *order, const int *start, const float *parts, float scale, int add,
                                                 float *dw)
{
    constexpr int AHEAD = 16;
    __shared__ float4 room[NT];
    const int all = start[V], part = blockIdx.x, p0 = part * PART, p1 = p0 + PART;
    if (p1 >= all) return;
    const int t = tokens[order[p1 - 1]], s0 = start[t], s1 = start[t + 1];
    if (s0 < p0 || s1 <= p1) return;
    const int L = 1 << log_lanes, groups = NT >> log_lanes, c = ((int)blockIdx.y * L + (threadIdx.x & (L - 1))) * 4, at = c < C ? c : 0;
    const int shares = (s1 - 1) / PART - part + 1, run = (shares + groups - 1) / groups, q0 = (int)(threadIdx.x >> log_lanes) * run, q1 = min(shares, q0 + run);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int q = q0; q < q1; q += AHEAD) {
        Piece<float> g[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int k = min(q + j, q1 - 1);
            g[j] = begin_piece(parts + (size_t)(2 * ((long long)part + k) + (k == 0 && s0 != p0 ? 1 : 0)) * C, at, C);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            settle_piece(g[j], at, C);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += q + j < q1 ? g[j].get(i) : 0.f;
        }
    }
    add_groups(s, room, log_lanes);
    if (threadIdx.x < (unsigned)L && c < C) put<false>(dw + (size_t)t * C, c, C, s, scale, add);
}

struct OrderPlan {
    int R, ranges, segment, segments, part;
    long long part_count;
    size_t order_bytes, start_bytes, part_bytes;
};
OrderPlan order_plan(int N, int V, int C)
{
    OrderPlan q = {};
    // some 256 workgroups, one a compute unit: 64 ranges of tokens where there are as many, by segments of the places
    q.ranges = V < 16 * 64 ? (V + 15) / 16 : 64;
    q.R = (V + q.ranges - 1) / q.ranges;
    if (q.R > ORDER_MOST) q.R = ORDER_MOST;
    q.ranges = (V + q.R - 1) / q.R;
    int segments = 256 / q.ranges;
    segments = segments < 1 ? 1 : segments > 16 ? 16 : segments;
    q.segment = (N + segments - 1) / segments;
    q.segments = (N + q.segment - 1) / q.segment;
    const int blocks = (C + BLOCK - 1) / BLOCK;
    // places of a part: as many as leave 2048 waves (65536 places of 256 columns: 64 places 81 us, 32 83, 16 93, for each part may leave shares that are read again)
    q.part = 64;
    while (q.part > 16 && (long long)N * blocks / q.part < 2048) q.part /= 2;
    q.part_count = ((long long)N + q.part - 1) / q.part;
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

// groups of the whole workgroup where those of a wave would make too many workgroups, each of which looks at all places
// One launch or three.  Up to 1024 places one; up to 2048 where the looking (each place among all, for each 256 columns) and the longest run of one workgroup cost less than two
// launches: us, one and three: 2048 places on 50257 x 512 bf16 8.1, 21.6; x 2048 17.7, 27.4; on 5000 x 4096 fp32 53, 33.5; on 2 x 512 30.6, 20.3; 4096 places on 10000 x 300 31, 21
bool is_few(int N, int V, int C) { return N <= 1024 || (N <= FEW && V >= 256 && (long long)N * C <= 1 << 22); }
int few_lanes(int N, int C) { return (long long)N * ((C + 255) / 256) <= 4096 ? group_lanes(C) : 8; }

template <class T>
int bwd(int N, int V, int C, const int *tokens, const T *dy, float scale, int add, float *dw, char *ws, hipStream_t st)
{
    const bool past = !add && (unsigned long long)V * C * 4 >= 256ull << 20;
    if (is_few(N, V, C)) {
        const int log_lanes = few_lanes(N, C), columns = 4 << log_lanes;
        const unsigned grid = (unsigned)(N + (add ? 0 : ((long long)V + ZERO_ROWS - 1) / ZERO_ROWS));
        hipLaunchKernelGGL(past ? (few_kernel<T, true>) : (few_kernel<T, false>), dim3(grid, (C + columns - 1) / columns), dim3(NT), 0, st, N, V, C, log_lanes, tokens, dy, scale, add, dw);
        return launched();
    }
    const OrderPlan q = order_plan(N, V, C);
    int *order = (int *)ws, *start = (int *)(ws + q.order_bytes);
    float *parts = (float *)(ws + q.order_bytes + q.start_bytes);
    hipLaunchKernelGGL(q.R <= 512 ? order_kernel<512> : q.R <= 1024 ? order_kernel<1024> : order_kernel<2048>, dim3(q.ranges, q.segments), dim3(ORDER_NT), 0, st, N, V, q.R, q.segment, tokens, order, start);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    const long long part_waves = q.part_count * ((C + BLOCK - 1) / BLOCK);
    const int empty_rows = C <= 256 ? 64 : 16;
    const unsigned part_groups = (unsigned)((part_waves + NT / 64 - 1) / (NT / 64)), empty_groups = add ? 0 : (unsigned)((V + empty_rows - 1) / empty_rows);
    hipLaunchKernelGGL(past ? (rows_kernel<T, true>) : (rows_kernel<T, false>), dim3(part_groups + empty_groups), dim3(NT), 0, st, V, C, q.part, part_waves, part_groups, empty_rows,
                       tokens, order, start, dy, scale, add, dw, parts);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    const int log_lanes = group_lanes(C);
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)q.part_count, (C + (4 << log_lanes) - 1) / (4 << log_lanes)), dim3(NT), 0, st, V, C, q.part, log_lanes, tokens, order, start, parts, scale, add, dw);
    return launched();
}

}  // namespace

int embedding_fwd(int N, int V, int C, int dtype, const int *tokens, const void *w, float scale, void *y, hipStream_t st)
{
    return dtype == MXC_BF16 ? fwd(N, V, C, tokens, (const bf16_t *)w, scale, (bf16_t *)y, st) : fwd(N, V, C, tokens, (const float *)w, scale, (float *)y, st);
}

size_t embedding_workspace(int N, int V, int C)
{
    if (is_few(N, V, C)) return 0;
    const OrderPlan q = order_plan(N, V, C);
    return q.order_bytes + q.start_bytes + q.part_bytes;
}

int embedding_bwd(int N, int V, int C, int dtype, const int *tokens, const void *dy, float scale, int add, float *dw, void *ws, hipStream_t st)
{
    return dtype == MXC_BF16 ? bwd(N, V, C, tokens, (const bf16_t *)dy, scale, add, dw, (char *)ws, st) : bwd(N, V, C, tokens, (const float *)dy, scale, add, dw, (char *)ws, st);
}

}  // namespace mxc
