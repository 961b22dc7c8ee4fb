// Embedding: y[n] = scale * w[tokens[n]], and the gradient of the table, dw[v] = scale * sum of dy[n] over the places n where tokens[n] == v.
// Memory bounds both: forward reads and writes each row once; the gradient reads dy once and writes a row of dw for every
// token of the vocabulary.  The gradient of more than a few places goes by the tokens' order, in three launches: the places are sorted by their token, each token's rows added, in
// parts, and the parts of a token that has several joined.  16384 rows of 4096 bf16 41.6 us, 6.5 TB/s (64 rows 3.9, a launch); gradient of 32768 places on 50257 x 2048, bf16,
// 130 us; of 500 places on 1000 x 512 fp32, added to it, in one launch, 5.2.
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

// The order of tokens that sorts the places: range by range, a range having every 2^log-th token, so that common tokens, whose numbers often lie close together, fall into different
// ranges (of contiguous ranges the one with a text's most common tokens took 15.6 us where the others took 8).
struct Ranges {
    int log, R;                             // ranges, as a power of two; tokens of a range
    __host__ __device__ int positions() const { return R << log; }
    __device__ __forceinline__ int position(int t) const { return (t & ((1 << log) - 1)) * R + (t >> log); }
};

// The places in the order of their tokens' positions (of equal tokens in their own), and where each position's begin.  Workgroup (x, y) puts the places of segment y
// whose token is among the R tokens of range x; for where they go it counts all places first.  Each of its waves has a share of the segment and a counter of its own for each
// token, so that no wave waits for another on the way; lanes of one token find each other by ballots.  The issue of instructions bounds it, for every workgroup looks at
// all tokens: 32768 places of 50257 tokens 13.2 us with 14 instructions for 64 tokens, 17.7 with 38.
constexpr int ORDER_NT = 1024, ORDER_WAVES = ORDER_NT / 64, ORDER_MOST = 2048, BATCH = 16, AT_ONCE = 12;
template <int MOST>
__global__ __launch_bounds__(ORDER_NT) void order_kernel(int N, int V, Ranges ranges, int segment, const int *tokens, int *order, int *start)
{
    __shared__ __attribute__((aligned(16))) int counts[(ORDER_WAVES + 2) * MOST];        // [ORDER_WAVES][R] of this segment, [R] of earlier ones, [R] of later ones
    __shared__ int wave_sum[ORDER_WAVES], wave_before[ORDER_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int R = ranges.R, log = ranges.log, range = blockIdx.x;
    for (int i = threadIdx.x * 4; i < (ORDER_WAVES + 2) * R; i += ORDER_NT * 4) *reinterpret_cast<int4 *>(counts + i) = make_int4(0, 0, 0, 0);
    __syncthreads();
    // a token rotated by `log` bits has its range at the top and its place in it below; one that is not in the table is past all ranges
    const unsigned lowest = log ? (unsigned)range << (32 - log) : 0u;
    auto key_of = [&](int t) __attribute__((always_inline)) {
        const unsigned key = __builtin_amdgcn_alignbit((unsigned)t, (unsigned)t, (unsigned)log);
        return (unsigned)t < (unsigned)V ? key : ~0u;
    };
    int before = 0;
    auto add = [&](unsigned key, int *into) __attribute__((always_inline)) {
        before += __popcll(__ballot(key < lowest));
        if (key - lowest < (unsigned)R) atomicAdd(into + (key - lowest), 1);
    };
    // tokens of places [from, to), 64 for each of the array; past them the last one's
    auto load = [&](auto &t, int from, int to) __attribute__((always_inline)) {
        constexpr int K = sizeof(t) / sizeof(t[0]);
        const int *at = tokens + from + lane;
        if (from + 64 * K <= to) {
#pragma unroll
            for (int j = 0; j < K; ++j) t[j] = at[64 * j];
        } else {
#pragma unroll
            for (int j = 0; j < K; ++j) t[j] = tokens[min(from + 64 * j + lane, to - 1)];
        }
    };
    // the places of this segment, and of these this wave's: multiples of 64 but the last
    const int share = (segment + ORDER_NT - 1) / ORDER_NT * 64;
    const int seg0 = blockIdx.y * segment, seg1 = min(N, seg0 + segment), n0 = min(seg1, seg0 + wave * share), n1 = min(seg1, n0 + share);
    int *own = counts + wave * R;
    // this wave's first places, which stay in registers, are on their way while those of the other segments are counted
    unsigned mine[BATCH];
    auto keys_of_mine = [&](int m) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < BATCH; ++j) mine[j] = m + 64 * j + lane < n1 ? key_of((int)mine[j]) : ~0u;
    };
    if (n0 < n1) load(mine, n0, n1);
    auto scan = [&](int from, int to, int *into) __attribute__((always_inline)) {
        const int part = (to - from + ORDER_NT - 1) / ORDER_NT * 64, end = min(to, from + (wave + 1) * part);
        for (int a = from + wave * part; a < end; a += 64 * AT_ONCE) {
            int t[AT_ONCE];
            load(t, a, end);
            if (a + 64 * AT_ONCE <= end) {
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j) add(key_of(t[j]), into);
            } else {
#pragma unroll
                for (int j = 0; j < AT_ONCE; ++j)
                    if (a + 64 * j < end) add(a + 64 * j + lane < end ? key_of(t[j]) : ~0u, into);
            }
        }
    };
    scan(0, seg0, counts + ORDER_WAVES * R);
    scan(seg1, N, counts + (ORDER_WAVES + 1) * R);
    for (int m = n0; m < n1; m += 64 * BATCH) {
        if (m != n0) load(mine, m, n1);
        keys_of_mine(m);
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
            if (m + 64 * j < n1) add(mine[j], own);
    }
    if (lane == 0) wave_before[wave] = before;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int k = 0; k < ORDER_WAVES; ++k) base += wave_before[k];
    // from counts to where a wave's places of a token go: OF tokens a thread
    constexpr int OF = MOST > ORDER_NT ? MOST / ORDER_NT : 1;
    const int t0 = threadIdx.x * OF;
    int has[OF][ORDER_WAVES + 2], sum = 0;
#pragma unroll
    for (int j = 0; j < OF; ++j)
#pragma unroll
        for (int k = 0; k < ORDER_WAVES + 2; ++k) {
            has[j][k] = t0 + j < R ? counts[k * R + t0 + j] : 0;
            sum += has[j][k];
        }
    int up = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int v = __shfl_up(up, d);
        up += lane >= d ? v : 0;
    }
    if (lane == 63) wave_sum[wave] = up;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ORDER_WAVES; ++k) base += k < wave ? wave_sum[k] : 0;
    base += up - sum;
#pragma unroll
    for (int j = 0; j < OF; ++j) {
        if (t0 + j >= R) break;
        if (blockIdx.y == 0) start[range * R + t0 + j] = base;
        int at = base + has[j][ORDER_WAVES];
#pragma unroll
        for (int k = 0; k < ORDER_WAVES; ++k) {
            counts[k * R + t0 + j] = at;
            at += has[j][k];
        }
        base = at + has[j][ORDER_WAVES + 1];
        if (blockIdx.y == 0 && t0 + j == R - 1 && range == (1 << log) - 1) start[ranges.positions()] = base;
    }
    __syncthreads();
    const int bits = 32 - __clz(R);
    for (int m = n0; m < n1; m += 64 * BATCH) {
        if (n1 - n0 > 64 * BATCH) {
            load(mine, m, n1);
            keys_of_mine(m);
        }
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            if (m + 64 * j >= n1) break;
            const unsigned d = mine[j] - lowest;
            const bool in = d < (unsigned)R;
            const unsigned long long all = __ballot(in);
            if (all == 0) continue;
            // the lanes that have the same token: of few one token after the other, of many those that agree in every bit (always the latter: 60000 places on 100000 x 16 28.9 us for 24.5)
            unsigned long long same = all;
            if (__popcll(all) <= 6) {
                for (unsigned long long left = all; left;) {
                    const unsigned long long of = __ballot(d == (unsigned)__builtin_amdgcn_readlane((int)d, __builtin_ctzll(left))) & all;
                    same = __builtin_amdgcn_inverse_ballot_w64(of) ? of : same;
                    left &= ~of;
                }
            } else {
                for (int b = 0; b < bits; ++b) {
                    const bool one = d >> b & 1;
                    const unsigned long long ones = __ballot(one);
                    same &= one ? ones : ~ones;
                }
            }
            if (in) {
                const int to = own[d], rank = __popcll(same & ((1ull << lane) - 1));
                order[to + rank] = m + 64 * j + lane;
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
// tokens that stand nowhere (between the parts', 4 % slower).  32768 places on 50257 x 2048 from memory, bf16: 110 us of the gradient's 130, 5 TB/s.
constexpr int BLOCK = 256;
template <class T, bool PAST>
__global__ __launch_bounds__(NT) void rows_kernel(int V, int C, int PART, long long part_waves, unsigned part_groups, int empty_rows, Ranges ranges, const int *tokens,
                                                 const int *order, const int *start, const T *dy, float scale, int add, float *dw, float *parts, int *joins)
{
    constexpr int AHEAD = 16;
    const int lane = threadIdx.x & 63;
    if (blockIdx.x >= part_groups) {
        const int v0 = (int)(blockIdx.x - part_groups) * empty_rows, rows = min(empty_rows, V - v0);
        const int at = ranges.position(v0 + min(lane, rows - 1));
        const unsigned long long empty = __ballot(lane < rows && start[at] == start[at + 1]);
        clear_rows<PAST>(dw, v0, rows, C, [&](int r) __attribute__((always_inline)) { return (empty >> r & 1) != 0; });
        return;
    }
    const long long w = (long long)blockIdx.x * (NT / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (w >= part_waves) return;
    const int blocks = (C + BLOCK - 1) / BLOCK, part = (int)(w / blocks), c = ((int)(w - (long long)part * blocks) * 64 + lane) * 4;
    const int all = __builtin_amdgcn_readfirstlane(start[ranges.positions()]), p0 = part * PART, count = min(PART, all - p0);
    const bool first = w == (long long)part * blocks && lane == 0;
    if (count <= 0) {
        if (first) joins[part] = -1;
        return;
    }
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
    const bool ends = __builtin_amdgcn_readfirstlane(behind) != now;
    if (first) joins[part] = now >= 0 && whole && !ends ? now : -1;
    if (now >= 0 && has) {          // (a part of fewer places has ended its last token above)
        if (whole && ends) put<PAST>(dw + (size_t)now * C, c, C, s, scale, add);
        else put<false>(parts + (size_t)(2 * part + slot) * C, c, C, s, 1.f, false);
    }
}

// A part in which a token begins that ends in another adds up that token's shares: a workgroup for 4 L columns, whose groups of L threads take a run of the shares each.
__global__ __launch_bounds__(NT) void join_kernel(int C, int PART, int log_lanes, Ranges ranges, const int *joins, const int *start, const float *parts, float scale, int add,
                                                 float *dw)
{
    constexpr int AHEAD = 8;
    __shared__ float4 room[NT];
    const int part = blockIdx.x, t = joins[part];
    if (t < 0) return;
    const int p = ranges.position(t), s0 = start[p], s1 = start[p + 1], p0 = part * PART;
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
    Ranges ranges;
    int segment, segments, part;
    long long part_count;
    size_t order_bytes, start_bytes, part_bytes, join_bytes;
};
OrderPlan order_plan(int N, int V, int C)
{
    OrderPlan q = {};
    // some 256 workgroups, one a compute unit: 16 to 64 ranges of tokens where there are as many, by segments of the places
    while (q.ranges.log < 6 && V >> q.ranges.log >= (q.ranges.log < 4 ? 2 : 32)) ++q.ranges.log;
    while ((V + (1 << q.ranges.log) - 1) >> q.ranges.log > ORDER_MOST) ++q.ranges.log;
    q.ranges.R = (V + (1 << q.ranges.log) - 1) >> q.ranges.log;
    int segments = 256 >> q.ranges.log;
    segments = segments < 1 ? 1 : segments > 16 ? 16 : segments;
    q.segment = (int)align_up((N + segments - 1) / segments, 64);
    q.segments = (N + q.segment - 1) / q.segment;
    const int blocks = (C + BLOCK - 1) / BLOCK;
    // places of a part: as many as leave 1024 waves, for each part may leave shares that are read again (us with 2048, 1024 and 512: 41282 places on 1713 x 192 fp32 43.8, 37.3, 37.0;
    // 60000 on 100000 x 16 bf16 36.4, 36.7, 42.1)
    q.part = 64;
    while (q.part > 16 && (long long)N * blocks / q.part < 1024) q.part /= 2;
    q.part_count = ((long long)N + q.part - 1) / q.part;
    q.order_bytes = align_up((size_t)N * 4, 256);
    q.start_bytes = align_up(((size_t)q.ranges.positions() + 1) * 4, 256);
    q.part_bytes = align_up((size_t)q.part_count * 2 * C * 4, 256);
    q.join_bytes = align_up((size_t)q.part_count * 4, 256);
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

// One launch or three.  Up to 1024 places one; up to 2048 where the looking (each place among all, for each 256 columns) and the longest run of one workgroup cost less than two
// launches: us, one and three: 2048 places on 50257 x 512 bf16 8.1, 18.9; x 2048 17.7, 23.7; on 5000 x 4096 fp32 53, 27.7; on 2 x 512 30.6, 17.9; 4096 places on 10000 x 300 31, 19.2
bool is_few(int N, int V, int C) { return N <= 1024 || (N <= FEW && V >= 256 && (long long)N * C <= 1 << 22); }
// groups of the whole workgroup where those of a wave would make too many workgroups, each of which looks at all places
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
    int *joins = (int *)(ws + q.order_bytes + q.start_bytes + q.part_bytes);
    hipLaunchKernelGGL(q.ranges.R <= 512 ? order_kernel<512> : q.ranges.R <= 1024 ? order_kernel<1024> : order_kernel<2048>, dim3(1 << q.ranges.log, q.segments), dim3(ORDER_NT), 0, st, N, V, q.ranges, q.segment, tokens, order, start);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    const long long part_waves = q.part_count * ((C + BLOCK - 1) / BLOCK);
    const int empty_rows = C <= 256 ? 64 : 16;
    const unsigned part_groups = (unsigned)((part_waves + NT / 64 - 1) / (NT / 64)), empty_groups = add ? 0 : (unsigned)((V + empty_rows - 1) / empty_rows);
    hipLaunchKernelGGL(past ? (rows_kernel<T, true>) : (rows_kernel<T, false>), dim3(part_groups + empty_groups), dim3(NT), 0, st, V, C, q.part, part_waves, part_groups, empty_rows,
                       q.ranges, tokens, order, start, dy, scale, add, dw, parts, joins);
    if (launched() != MXC_OK) return MXC_ERR_LAUNCH;
    const int log_lanes = group_lanes(C);
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)q.part_count, (C + (4 << log_lanes) - 1) / (4 << log_lanes)), dim3(NT), 0, st, C, q.part, log_lanes, q.ranges, joins, start, parts, scale, add, dw);
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
    return q.order_bytes + q.start_bytes + q.part_bytes + q.join_bytes;
}

int embedding_bwd(int N, int V, int C, int dtype, const int *tokens, const void *dy, float scale, int add, float *dw, void *ws, hipStream_t st)
{
    return dtype == MXC_BF16 ? bwd(N, V, C, tokens, (const bf16_t *)dy, scale, add, dw, (char *)ws, st) : bwd(N, V, C, tokens, (const float *)dy, scale, add, dw, (char *)ws, st);
}

}  // namespace mxc
