// Log probabilities of given tokens under softmax(scale*z), entropies, the most probable tokens, and the gradient of a weighted
// sum of log probabilities and entropies.  With d = scale*(z - max), S = sum exp(d), T = sum exp(d)*d:
//     logp = d[label] - log S,    entropy = log S - T/S,    dz = e*(A + B*d) + [k == label]*scale*dlogp,
//     e = exp(d), A = scale/S*(dentropy*T/S - dlogp), B = -scale/S*dentropy.
// fp32 arithmetic whatever the storage type, in powers of two: d2 = d/ln 2, so that an exponential is one instruction.
//
// A row is read once.  Workgroups of 64 to 1024 threads hold it in registers as 16-byte pieces (up to 256 KB: half of a compute
// unit's registers), meet for the maximum and for the sums, and write the gradient from what they hold.  Without a gradient, rows of more than
// 1024 pieces stream by.  Few rows, and rows that are longer than registers, are cut into chunks, each with its own maximum and sums, which a second
// launch joins (and reads again for the gradient).  4096 rows of 131072 bf16 with the gradient 433 us, 4.95 TB/s: one workgroup a compute unit, which loads nothing
// while it reduces and writes its row; the gradient from statistics, eight workgroups a unit, moves the same bytes in 367 us, 5.85 TB/s.  4096 of 50257 with the 8 best
// tokens 86 us, 4.8 TB/s: the vector units issue without a pause, 14.4 instructions a value (75 us and 11.3 without the best tokens; of fp32 151 us, 5.4 TB/s).
// One row of 131072 with the 20 best is latency, 11.3 us in two launches.
#include <type_traits>

#include "mxc_internal.h"

namespace mxc {
namespace {

constexpr float LOWEST = -3.402823466e38f, LN2 = 0.693147182464599609f, LOG2E = 1.442695021629333496f;
constexpr float NO_WEIGHT = -300.f;     // exp2 of this is 0: a term exp2(d)*d is 0 there, also at d = minus infinity
constexpr unsigned long long NO_KEY = 0;

// ordered as the values are; -0 and 0 are one value
__device__ __forceinline__ unsigned order(float z)
{
    const int b = __float_as_int(z + 0.f);
    return (unsigned)(b ^ ((b >> 31) & 0x7FFFFFFF)) ^ 0x80000000u;
}
__device__ __forceinline__ float unorder(unsigned o)
{
    const int b = (int)(o ^ 0x80000000u);
    return __int_as_float(b ^ ((b >> 31) & 0x7FFFFFFF));
}
// a larger key is a larger value, of equal ones the one of the lower index; NO_KEY is less than any
__device__ __forceinline__ unsigned long long key_of(unsigned o, unsigned index) { return ((unsigned long long)o << 32) | (0xFFFFFFFFu - index); }
__device__ __forceinline__ unsigned key_index(unsigned long long key) { return 0xFFFFFFFFu - (unsigned)key; }

// fmaxf takes an instruction more, for the sake of signalling NaNs
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

__device__ __forceinline__ float min3(float a, float b, float c)
{
    float r;
    asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

template <typename T>
struct Piece {      // 16 bytes of a row
    static constexpr int V = 16 / (int)sizeof(T);
    uint32_t w[4];
    __device__ __forceinline__ float at(int k) const
    {
        if constexpr (V == 8) return __uint_as_float(k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16);
        else return __uint_as_float(w[k]);
    }
    // The same for passes after the first: the compiler would keep both halves of each word as floats, or what the first pass made of
    // them, in twice the registers.
    __device__ __forceinline__ float again(int k) const
    {
        if constexpr (V == 8) {
            float r;
            if (k & 1) asm volatile("v_and_b32 %0, %1, %2" : "=v"(r) : "s"(0xFFFF0000u), "v"(w[k / 2]));
            else asm volatile("v_lshlrev_b32 %0, 16, %1" : "=v"(r) : "v"(w[k / 2]));
            return r;
        } else {
            uint32_t r;
            asm volatile("" : "=v"(r) : "0"(w[k]));
            return __uint_as_float(r);
        }
    }
    template <bool AGAIN>
    __device__ __forceinline__ float largest() const
    {
        auto v = [&](int k) { return AGAIN ? again(k) : at(k); };
        float m = v(0);
#pragma unroll
        for (int k = 1; k + 1 < V; k += 2) m = max3(m, v(k), v(k + 1));
        const float last = v(V - 1);
        return max3(m, last, last);
    }
    // minus infinities become `value`
    __device__ __forceinline__ void refill(float value)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (V == 8) {
                const uint32_t v = __float_as_uint(value) >> 16;
                if ((w[k] & 0xFFFFu) == 0xFF80u) w[k] = (w[k] & 0xFFFF0000u) | v;
                if (w[k] >> 16 == 0xFF80u) w[k] = (w[k] & 0xFFFFu) | (v << 16);
            } else if (w[k] == 0xFF800000u)
                w[k] = __float_as_uint(value);
        }
    }
    __device__ __forceinline__ void nothing()      // minus infinities: no weight in any sum
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = V == 8 ? 0xFF80FF80u : 0xFF800000u;
    }
};

// Lanes of a group of G (8 or a whole wave) meet: exchanges within rows of 16 lanes are part of an instruction (a shuffle through LDS has ten times the
// latency, and a row of few values is latency), the four rows meet as scalars.  The same order everywhere.
template <int CONTROL>
__device__ __forceinline__ float exchanged(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CONTROL, 0xF, 0xF, true)); }
template <int G, class F>
__device__ __forceinline__ float meet(float x, F f)
{
    x = f(x, exchanged<0xB1>(x));       // lanes 1 0 3 2
    x = f(x, exchanged<0x4E>(x));       // lanes 2 3 0 1
    x = f(x, exchanged<0x141>(x));      // the other half of eight
    if constexpr (G == 8) return x;
    x = f(x, exchanged<0x140>(x));      // the other half of sixteen
    auto of_row = [&](int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); };
    return f(f(of_row(0), of_row(16)), f(of_row(32), of_row(48)));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum(float a, float b) { return a + b; }

// What the first look at a row finds: its largest and its lowest value.  bf16 words are looked at as
// pairs of 16-bit integers, two values an instruction: of signed ones the largest is the largest value unless all are negative (then it
// is some value; `sure` is false), of unsigned ones the largest is the most negative value where there is one.  fp32 values are looked at as they are.
template <typename T>
struct Extent;
template <>
struct Extent<bf16_t> {
    typedef short i16x2 __attribute__((ext_vector_type(2)));
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    i16x2 hi = {(short)0x8000, (short)0x8000};
    u16x2 lo = {0, 0};
    __device__ __forceinline__ void look(const Piece<bf16_t> &p, bool whole)
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) hi = __builtin_elementwise_max(hi, __builtin_bit_cast(i16x2, p.w[k]));
        if (whole) {
#pragma unroll
            for (int k = 0; k < 4; ++k) lo = __builtin_elementwise_max(lo, __builtin_bit_cast(u16x2, p.w[k]));
        }
    }
    __device__ __forceinline__ void look(float low)
    {
        const unsigned short u = (unsigned short)(__float_as_uint(low) >> 16);
        lo.x = lo.x > u ? lo.x : u;
    }
    __device__ __forceinline__ void look(const Extent &e)
    {
        hi = __builtin_elementwise_max(hi, e.hi);
        lo = __builtin_elementwise_max(lo, e.lo);
    }
    __device__ __forceinline__ float largest() const { return __uint_as_float((unsigned)(uint16_t)(hi.x > hi.y ? hi.x : hi.y) << 16); }
    // one word for the lanes and waves to meet with: both maxima as signed numbers
    typedef i16x2 Word;
    __device__ __forceinline__ Word word() const
    {
        const unsigned short u = lo.x > lo.y ? lo.x : lo.y;
        return Word{hi.x > hi.y ? hi.x : hi.y, (short)(u ^ 0x8000u)};
    }
    static __device__ __forceinline__ Word join(Word a, Word b) { return __builtin_elementwise_max(a, b); }
    template <int G>
    static __device__ __forceinline__ Word meet_lanes(Word a)
    {
        return __builtin_bit_cast(Word, meet<G>(__builtin_bit_cast(float, a), [](float x, float y) {
            return __builtin_bit_cast(float, join(__builtin_bit_cast(Word, x), __builtin_bit_cast(Word, y)));
        }));
    }
    static __device__ __forceinline__ float most(Word a) { return __uint_as_float((unsigned)(uint16_t)a.x << 16); }
    static __device__ __forceinline__ bool sure(Word a) { return a.x >= 0; }
    static __device__ __forceinline__ float lowest(Word a) { return __uint_as_float(((uint16_t)a.y ^ 0x8000u) << 16); }
};
template <>
struct Extent<float> {
    float hi = -INFINITY, lo = INFINITY;
    __device__ __forceinline__ void look(const Piece<float> &p, bool whole)
    {
        hi = max3(max3(hi, p.at(0), p.at(1)), p.at(2), p.at(3));
        if (whole) lo = min3(min3(lo, p.at(0), p.at(1)), p.at(2), p.at(3));
    }
    __device__ __forceinline__ void look(float low) { lo = fminf(lo, low); }
    __device__ __forceinline__ void look(const Extent &e)
    {
        hi = fmaxf(hi, e.hi);
        lo = fminf(lo, e.lo);
    }
    __device__ __forceinline__ float largest() const { return hi; }
    typedef float2 Word;
    __device__ __forceinline__ Word word() const { return make_float2(hi, lo); }
    static __device__ __forceinline__ Word join(Word a, Word b) { return make_float2(fmaxf(a.x, b.x), fminf(a.y, b.y)); }
    template <int G>
    static __device__ __forceinline__ Word meet_lanes(Word a)
    {
        return make_float2(meet<G>(a.x, [](float x, float y) { return fmaxf(x, y); }), meet<G>(a.y, [](float x, float y) { return fminf(x, y); }));
    }
    static __device__ __forceinline__ float most(Word a) { return fmaxf(a.x, LOWEST); }
    static __device__ __forceinline__ bool sure(Word) { return true; }
    static __device__ __forceinline__ float lowest(Word a) { return a.y; }
};

// A row as pieces at 16-byte boundaries: the first and the last may be shared with what lies before and behind the row, which is
// neither read nor written.  NT: past the caches, for calls of more than they hold.
template <typename T, bool NT = false>
struct Row {
    static constexpr int V = Piece<T>::V;
    const T *z;         // element `head` elements before the row's first
    T *dz;
    int head, K, pieces;
    __device__ __forceinline__ Row(const LogprobArgs &a, size_t row)
    {
        const size_t first = row * a.ld;
        head = (int)(first % V);
        K = a.K;
        pieces = (a.K + head + V - 1) / V;
        z = (const T *)a.z + first - head;
        dz = a.dz ? (T *)a.dz + first - head : nullptr;
    }
    __device__ __forceinline__ bool whole(int piece) const { return whole(piece, 1); }
    // all pieces of [piece, piece + n) lie wholly in the row
    __device__ __forceinline__ bool whole(int piece, int n) const { return piece * V >= head && (piece + n) * V <= K + head; }
    // Places outside the row get minus infinity; low: the lowest value of pieces that are not whole.
    __device__ __forceinline__ Piece<T> load(int piece, float &low) const { return load(piece, low, pieces); }
    // as if the row ended before piece `end`
    __device__ __forceinline__ Piece<T> load(int piece, float &low, int end) const
    {
        Piece<T> p;
        if (whole(piece) && piece < end) {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            const u32x4 *from = reinterpret_cast<const u32x4 *>(z) + (unsigned)piece;
            const u32x4 u = NT ? __builtin_nontemporal_load(from) : *from;
            p.w[0] = u.x; p.w[1] = u.y; p.w[2] = u.z; p.w[3] = u.w;
        } else {
            p.nothing();
            if (piece < end) {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const int i = piece * V + k;
                    if (i < head || i >= K + head) continue;
                    low = fminf(low, load_f32(z + i));
                    if constexpr (V == 8) {
                        const uint32_t v = z[i];
                        p.w[k / 2] = k & 1 ? (p.w[k / 2] & 0xFFFFu) | (v << 16) : (p.w[k / 2] & 0xFFFF0000u) | v;
                    } else
                        p.w[k] = __float_as_uint(z[i]);
                }
            }
        }
        return p;
    }
    __device__ __forceinline__ void store(int piece, const float *g) const
    {
        if (whole(piece)) {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
            u32x4 u;
            if constexpr (V == 8) u = u32x4{pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]), pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7])};
            else u = u32x4{__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3])};
            u32x4 *to = reinterpret_cast<u32x4 *>(dz) + (unsigned)piece;
            if (NT) __builtin_nontemporal_store(u, to);
            else *to = u;
        } else if (piece < pieces) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const int i = piece * V + k;
                if (i < head || i >= K + head) continue;
                if constexpr (V == 8) dz[i] = (bf16_t)pack_bf16x2(g[k], g[k]);
                else dz[i] = g[k];
            }
        }
    }
};

// d2 of a logit.  Near: one fma, z*k2 + c with c = -max*k2 rounded once: the same for the whole row, so that it moves the
// reference point of d2 a little (by less than 2^-8) and cancels in every result.  Far from zero, where it would move it by more, and where the products
// overflow: the difference first.
struct Scale {
    float k, k2, m, c;
    bool near;
    __device__ __forceinline__ Scale(float scale, float most)
    {
        k = scale;
        k2 = scale * LOG2E;
        m = most;
        c = -(most * k2);
        near = fabsf(c) < 65536.f;
    }
    template <bool NEAR>
    __device__ __forceinline__ float d2(float z) const { return NEAR ? fmaf(z, k2, c) : (z - m) * k2; }
    __device__ __forceinline__ float any(float z) const { return near ? d2<true>(z) : d2<false>(z); }
    // the log probability of a logit whose d2 this is.  Very far from the maximum (a masked token) the product in powers of two may overflow where
    // the result does not, and ls is nothing (or NaN).
    __device__ __forceinline__ float log_prob(float d2, float z, float ls) const { return d2 > -0x1p100f ? (d2 - ls) * LN2 : (0.5f * z - 0.5f * m) * k * 2.f - ls; }
};

template <bool CLAMP>
__device__ __forceinline__ float weight(float d) { return CLAMP ? fmaxf(d, NO_WEIGHT) : d; }
// exp2(d)*(A + B*d), which is 0 where exp2(d) is, however low d and however large the factors are: without the clamp d may be -3.0e38 (see `masked`)
// and |B| 1; with it |B| 1e36; ANY takes what else 32 bits hold.  (It always would: 2 % of the time of masked rows, 4096 of 50257 bf16 155.6 -> 158.7 us.)
enum Slope { PLAIN, CLAMPED, ANY };
template <int S>
__device__ __forceinline__ float slope(float d, float A, float B)
{
    const float e = __builtin_amdgcn_exp2f(d), at = weight<S != PLAIN>(d);
    return S == ANY ? fmaf(e * at, B, e * A) : e * fmaf(at, B, A);
}
__device__ __forceinline__ bool moderate(float A, float B) { return fabsf(B) <= 1e36f && fabsf(A) <= 1e37f; }

// ---- the most probable tokens ---------------------------------------------------------------------------------------------
// Cells are sets of a wave's values, 64 or more of them, of which each lane knows one of the largest.  Where each of W waves has top/W cells that
// reach a bound, `top` values reach it; so they do where one wave has `top` cells that reach it.  What reaches the bound is collected in
// LDS and ranked by counting, which makes the order that of the keys whatever order they were collected in.
template <int CAP_>
struct TopShared {
    static constexpr int CAP = CAP_;
    unsigned long long list[CAP];
    unsigned bound[16];
    int count;
};

// the largest t that at least n of the wave's cells reach (t's lowest LOW bits are 0)
template <int S, int LOW>
__device__ __forceinline__ unsigned wave_bound(const unsigned *cell, int n)
{
    unsigned t = 0;
    for (int b = 31; b >= LOW; --b) {
        const unsigned trial = t | (1u << b);
        int c = 0;
#pragma unroll
        for (int s = 0; s < S; ++s) c += __popcll(__ballot(cell[s] >= trial));
        if (c >= n) t = trial;
    }
    return t;
}

template <int W, int CAP, class Emit>
__device__ __forceinline__ void rank_candidates(const TopShared<CAP> &sh, int n, int top, Emit emit)
{
    for (int i = threadIdx.x; i < n; i += 64 * W) {
        const unsigned long long key = sh.list[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) rank += sh.list[j] > key ? 1 : 0;
        if (rank < top) emit(rank, key);
    }
    for (int i = n + (int)threadIdx.x; i < top; i += 64 * W) emit(i, NO_KEY);
}

// Hands the i-th largest key of the row to emit(i, key); places past the last value get NO_KEY.  Called by a whole workgroup of W waves;
// cell: this lane's S cells.  each(from, f) calls f(order, index) for each of the thread's values that reaches `from`.
template <int W, int S, int LOW, int CAP, class Each, class Emit>
__device__ __forceinline__ void select_top(TopShared<CAP> &sh, const unsigned *cell, int top, Each each, Emit emit)
{
    const int wave = threadIdx.x >> 6;
    unsigned bound = wave_bound<S, LOW>(cell, (top + W - 1) / W);
    if (threadIdx.x == 0) sh.count = 0;
    if ((threadIdx.x & 63) == 0) sh.bound[wave] = bound;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) bound = min(bound, sh.bound[w]);
    if (bound <= order(-INFINITY)) {        // a wave has less than its share: what one wave holds alone
        __syncthreads();
        bound = wave_bound<S, LOW>(cell, top);
        if ((threadIdx.x & 63) == 0) sh.bound[wave] = bound;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) bound = max(bound, sh.bound[w]);
    }
    // Values above the bound, and equal ones up to index `tie`.  Where there are many equal ones (rows of one value, rows where few tokens are
    // allowed) a second turn takes only the lowest indices of those at the bound: each lane's first one is a cell again.
    unsigned tie = 0xFFFFFFFFu, first = 0xFFFFFFFFu;
    bool full = false;      // the list was, when this lane last had something for it
    int n;
    for (int turn = 0;; ++turn) {
        each(bound, [&](unsigned o, unsigned index) {
            const bool at_bound = o >> LOW == bound >> LOW;
            if (!full && (!at_bound || index <= tie)) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < CAP) sh.list[at] = key_of(o, index);
                full = at >= CAP;
            }
            if (at_bound) first = min(first, index);
        });
        __syncthreads();
        n = sh.count;
        if (n <= CAP || turn == 1) break;
        full = false;
        const unsigned cells[1] = {~first};
        tie = ~wave_bound<1, 0>(cells, top);        // (no less than top of them: those above the bound may be none)
        __syncthreads();
        if (threadIdx.x == 0) sh.count = 0;
        if ((threadIdx.x & 63) == 0) sh.bound[wave] = tie;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) tie = min(tie, sh.bound[w]);
    }
    if (n <= CAP) {
        rank_candidates<W>(sh, n, top, emit);
        return;
    }
    // the largest values crowd in a few threads' pieces: one after the other
    unsigned long long last = ~0ull;
    for (int i = 0; i < top; ++i) {
        unsigned long long best = NO_KEY;
        each(0, [&](unsigned o, unsigned index) {
            const unsigned long long key = key_of(o, index);
            if (key < last && key > best) best = key;
        });
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const unsigned long long other = __shfl_xor(best, d);
            best = other > best ? other : best;
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) sh.list[wave] = best;
        __syncthreads();
        for (int w = 0; w < W; ++w) best = sh.list[w] > best ? sh.list[w] : best;
        last = best;
        if (threadIdx.x == 0) emit(i, best);
    }
}

// Pieces with a value that may be among the most probable, set aside in LDS.  Minus infinities are left out: limit is LOWEST at least.  From there
// each thread looks at one value of one piece: short code counts here, for a kernel of few rows is mostly latency, that of fetching its code included.
template <typename T, int HELD>
struct Aside {
    static constexpr int V = Piece<T>::V;
    T value[HELD][V];
    int place[HELD], count;
    unsigned said[16];      // bounds of the waves

    __device__ __forceinline__ bool put(const Piece<T> &p, int piece)
    {
        const int at = atomicAdd(&count, 1);
        if (at >= HELD) return false;
        *reinterpret_cast<uint4 *>(value[at]) = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
        place[at] = piece;
        return true;
    }
    // the bound that all of W waves have reached
    template <int W>
    __device__ __forceinline__ unsigned hear() const
    {
        const volatile unsigned *w = said;
        unsigned b = w[0];
#pragma unroll
        for (int i = 1; i < W; ++i) b = min(b, w[i]);
        return b;
    }
    // Ranks what reaches the bound; false where that is not to be had: too many of them, or minus infinities are among the most probable ones of
    // `values`.  sh.count is 0.
    template <int W, int LOW, int CAP, class Emit>
    __device__ __forceinline__ bool rank(TopShared<CAP> &sh, unsigned bound, int head, int K, int top, int values, Emit emit) const
    {
        const int pieces = count;
        if (pieces > HELD) return false;
        const bool bounded = bound >> LOW > order(-INFINITY) >> LOW;
        for (int i = threadIdx.x; i < pieces * V; i += 64 * W) {
            const float z = load_f32(&value[0][0] + i);
            const int index = place[i / V] * V + i % V - head;
            if (!(z >= LOWEST) || order(z) < bound || (unsigned)index >= (unsigned)K) continue;
            const int at = atomicAdd(&sh.count, 1);
            if (at < CAP) sh.list[at] = key_of(order(z), (unsigned)index);
        }
        __syncthreads();
        const int n = sh.count;
        if (n > CAP || !(bounded || n >= top || n >= values)) return false;
        rank_candidates<W>(sh, n, top, emit);
        return true;
    }
};

// The values of a thread's pieces that reach `from`, and the row's index of each: f(order, index).  first: the index of value 0 of piece 0;
// held: pieces that any thread holds.  A whole wave goes on where no lane has a piece that may reach it (ordered: none of them is a NaN, which a piece's
// largest value passes over).
template <typename T, int P, class F>
__device__ __forceinline__ void each_value(const Piece<T> (&p)[P], int held, int first, int stride, int K, bool ordered, unsigned from, F f)
{
    const float limit = unorder(from);      // (NaN for the lowest bounds: then every value is looked at)
#pragma unroll
    for (int q = 0; q < P; ++q) {
        if (q >= held) continue;
        if (ordered && __ballot(!(p[q].template largest<true>() < limit)) == 0) continue;
        int index = first + q * stride;
        asm volatile("" : "+v"(index));     // (else the indices of all values are worked out ahead, and held)
#pragma unroll
        for (int k = 0; k < Piece<T>::V; ++k) {
            const float v = p[q].again(k);
            if (v < limit) continue;
            const int i = index + k;
            const unsigned o = order(v);
            if (o >= from && (unsigned)i < (unsigned)K) f(o, (unsigned)i);
        }
    }
}

// The most probable tokens of a row that one wave holds; cell: the largest value of each of the lane's P pieces, first: the index of value 0 of piece 0.
// The bound is the largest value that `top` pieces reach; what reaches it is collected and ranked.  Where that is many values (equal ones: rows in which few
// tokens are allowed), the second way: fewer than `top` pieces have values above the bound, all of which go on the list, and of those at the bound
// as many of the lowest indices as are missing.  Indices ascend with the piece, the lane and the place, so that their order is a count over ballots.
template <typename T, int P, int CAP, class Emit>
__device__ __forceinline__ void wave_top(TopShared<CAP> &sh, const Piece<T> (&p)[P], const unsigned (&cell)[P], int held, int first, int K, int top, Emit emit)
{
    constexpr int V = Piece<T>::V, LOW = sizeof(T) == 2 ? 16 : 0, FEW = 160;
    static_assert(CAP >= (MXC_LOGPROB_MAX_TOP - 1) * V, "room for all values of the pieces above the bound");
    auto value_of = [](unsigned o) { return o >> LOW <= order(-INFINITY) >> LOW ? -INFINITY : __uint_as_float(__float_as_uint(unorder(o)) >> LOW << LOW); };
    unsigned bound = wave_bound<P, LOW>(cell, top);
    float limit = value_of(bound);
    // f(index, value, in the row) for the places of piece q
    auto places = [&](int q, auto f) {
        int index = first + q * 64 * V;
        asm volatile("" : "+v"(index));
#pragma unroll
        for (int k = 0; k < V; ++k) f(index + k, p[q].again(k), (unsigned)(index + k) < (unsigned)K);
    };
    auto put = [&](float v, int index) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < CAP) sh.list[at] = key_of(order(v), (unsigned)index);
    };
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    if (limit > -INFINITY) {
#pragma unroll
        for (int q = 0; q < P; ++q)
            if (q < held && cell[q] >= bound)
                places(q, [&](int index, float v, bool in) {
                    if (v >= limit && in) put(v, index);
                });
        __syncthreads();
        const int n = sh.count;
        if (n <= FEW) {
            rank_candidates<1>(sh, n, top, emit);
            return;
        }
        __syncthreads();
        if (threadIdx.x == 0) sh.count = 0;
    } else if (K > 128) {       // fewer pieces than `top` have a value: the bound that as many values reach (of fewer values all are ranked)
        bound = 0;
#pragma unroll 1
        for (int b = 31; b >= LOW; --b) {
            const unsigned trial = bound | (1u << b);
            const float t = unorder(trial);     // (NaN below minus infinity)
            int c = 0;
#pragma unroll
            for (int q = 0; q < P; ++q)
                if (q < held) places(q, [&](int, float v, bool in) { c += __popcll(__ballot(in && v >= t)); });
            if (c >= top) bound = trial;
        }
        limit = value_of(bound);
    }
    int above = 0;
#pragma unroll
    for (int q = 0; q < P; ++q)
        if (q < held && __ballot(cell[q] >> LOW > bound >> LOW)) places(q, [&](int, float v, bool in) { above += __popcll(__ballot(in && v > limit)); });
    int need = top - above;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < P; ++q) {
        if (q >= held || !__ballot(cell[q] >= bound)) continue;
        int before = 0, all = 0;        // values at the bound in earlier lanes, in all
        if (need > 0)
            places(q, [&](int, float v, bool in) {
                const unsigned long long b = __ballot(in && v == limit);
                before = __builtin_amdgcn_mbcnt_hi((unsigned)(b >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)b, before));
                all += __popcll(b);
            });
        places(q, [&](int index, float v, bool in) {
            const bool equal = in && v == limit;
            if ((in && v > limit) || (equal && before < need)) put(v, index);
            if (equal) ++before;
        });
        need -= all;
    }
    __syncthreads();
    rank_candidates<1>(sh, min(sh.count, CAP), top, emit);
}

// G threads a row, P pieces a thread; rows of fewer than a wave's lanes share one.  TOP: with the most probable tokens, else
// the gradient where dz is given.
template <typename T, int G, int P, bool TOP, bool NT = false>
__global__ __launch_bounds__(G < 64 ? 256 : G, G == 512 && P == 16 ? 4 : 1) void logprob_row_kernel(LogprobArgs a)
{
    constexpr int W = G / 64;       // waves a row; 0: several rows a wave
    __shared__ float red[2][W > 1 ? W : 1];
    __shared__ typename Extent<T>::Word ext[W > 1 ? W : 1];
    const int lane = G < 64 ? threadIdx.x % G : threadIdx.x;
    const size_t row = G < 64 ? (size_t)blockIdx.x * (256 / G) + threadIdx.x / G : (size_t)blockIdx.x;
    if (G < 64 && row >= (size_t)a.N) return;
    const Row<T, NT> r(a, row);
    Piece<T> p[P];
    const int held = (r.pieces + G - 1) / G;        // pieces that any thread holds: what follows passes over the others
    float low = 0.f;        // (above nothing that matters)
#pragma unroll
    for (int q = 0; q < P; ++q) p[q] = r.load(q * G + lane, low);
    const int label = a.labels ? a.labels[row] : -1;
    const bool given = (unsigned)label < (unsigned)a.K;
    const float zl = given ? load_f32(r.z + r.head + label) : 0.f;      // (before the gradient is written: dz may be z)
    auto meet_row = [&](float x, int slot, auto f) {
        x = meet<(G < 64 ? G : 64)>(x, f);
        if constexpr (W > 1) {
            if ((threadIdx.x & 63) == 0) red[slot][threadIdx.x >> 6] = x;
        }
        return x;
    };
    auto joined = [&](float x, int slot, auto f) {
        if constexpr (W > 1) {
            x = red[slot][0];
#pragma unroll
            for (int w = 1; w < W; ++w) x = f(x, red[slot][w]);
        }
        return x;
    };
    constexpr int S = P < 4 ? P : 4;
    Extent<T> part[S];
#pragma unroll
    for (int q = 0; q < P; ++q) {
        if (q >= held) continue;
        if (r.whole(q * G, G)) part[q % S].look(p[q], true);        // (the same for all of the row's lanes)
        else part[q % S].look(p[q], r.whole(q * G + lane));
    }
    part[0].look(low);
    unsigned cell[S];
    if constexpr (TOP && W > 1) {
#pragma unroll
        for (int s = 0; s < S; ++s) cell[s] = s < held ? order(part[s].largest()) : 0u;     // (a part that has seen nothing has a value all the same)
    }
#pragma unroll
    for (int s = 1; s < S; ++s) part[0].look(part[s]);
    typename Extent<T>::Word e = part[0].word();
    e = Extent<T>::template meet_lanes<(G < 64 ? G : 64)>(e);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) ext[threadIdx.x >> 6] = e;
        __syncthreads();
        e = ext[0];
#pragma unroll
        for (int w = 1; w < W; ++w) e = Extent<T>::join(e, ext[w]);
    }
    // (where one wave selects, each piece's largest value, before the places outside the row get a number)
    unsigned most[TOP && W == 1 ? P : 1];
    if constexpr (TOP && W == 1) {
#pragma unroll
        for (int q = 0; q < P; ++q) most[q] = order(p[q].template largest<true>());
    }
    float m = Extent<T>::most(e);
    if (!Extent<T>::sure(e)) {      // all are negative
        m = LOWEST;
        float of[S];
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const float x = q < held ? p[q].template largest<true>() : -INFINITY;
            of[q % S] = q < S ? x : fmaxf(of[q % S], x);
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if constexpr (TOP && W > 1) cell[s] = order(of[s]);
            m = fmaxf(m, of[s]);
        }
        m = meet_row(m, 0, larger);
        if constexpr (W > 1) __syncthreads();
        m = joined(m, 0, larger);
        if constexpr (W > 1) __syncthreads();
    }
    const Scale sc(a.scale, m);
    // Some d2 may be minus infinity (a NaN comes here too).  Where none is, the places outside the row get a number that has no weight
    // either, and no product needs care.  (Under a scale so small that there is no such number they stay minus infinities.)
    const bool masked = !(Extent<T>::lowest(e) * sc.k2 > -3.0e38f) || sc.k2 < 0x1p-100f;
    const float fill = sc.near && !masked ? -0x1p20f / sc.k2 : -INFINITY;
#pragma unroll
    for (int q = 0; q < P; ++q)
        if (q < held && !r.whole(q * G, G)) p[q].refill(fill);
    float s = 0.f, t = 0.f;
    auto sums = [&](auto clamp) {
#pragma unroll
        for (int q = 0; q < P; ++q) {
            if (q >= held) continue;
#pragma unroll
            for (int k = 0; k < Piece<T>::V; ++k) {
                const float d = sc.d2<true>(p[q].again(k)), e = __builtin_amdgcn_exp2f(d);
                s += e;
                t = fmaf(e, weight<decltype(clamp)::value>(d), t);
            }
        }
    };
    if (!sc.near) {     // rare: the pieces once more from memory, one after the other
        for (int piece = lane; piece < r.pieces; piece += G) {
            const Piece<T> c = r.load(piece, low);
#pragma unroll
            for (int k = 0; k < Piece<T>::V; ++k) {
                const float d = sc.d2<false>(c.at(k)), e = __builtin_amdgcn_exp2f(d);
                s += e;
                t = fmaf(e, weight<true>(d), t);
            }
        }
    } else if (masked) sums(std::true_type());
    else sums(std::false_type());
    s = meet_row(s, 0, sum);
    t = meet_row(t, 1, sum);
    if constexpr (W > 1) __syncthreads();
    s = joined(s, 0, sum);
    t = joined(t, 1, sum);
    const bool empty = s == 0.f;
    const float ls = empty ? 0.f : log2f(s), mean = t / s;
    if (lane == 0) {
        if (a.logp) a.logp[row] = !given ? 0.f : empty ? -INFINITY : sc.log_prob(sc.any(zl), zl, ls);
        if (a.entropy) a.entropy[row] = empty ? 0.f : (ls - mean) * LN2;
        if (a.stats) {
            a.stats[2 * row] = empty ? -INFINITY : s == s ? m : s;
            a.stats[2 * row + 1] = empty ? 0.f : (ls - sc.any(m)) * LN2;
        }
    }
    if constexpr (TOP) {
        constexpr int CAP = 512, HELD = 256, LOW = sizeof(T) == 2 ? 16 : 0;
        __shared__ TopShared<CAP> sh;
        auto emit = [&](int i, unsigned long long key) {
            a.top_index[row * a.top + i] = key == NO_KEY ? -1 : (int)key_index(key);
            a.top_logp[row * a.top + i] = -INFINITY;
            if (key == NO_KEY || empty) return;
            const float z = unorder((unsigned)(key >> 32));
            a.top_logp[row * a.top + i] = sc.log_prob(sc.any(z), z, ls);
        };
        if (empty) {        // minus infinities alone
            if (lane < a.top) emit(lane, lane < a.K ? key_of(order(-INFINITY), (unsigned)lane) : NO_KEY);
            return;
        }
        // Not ordered: a row with a NaN or plus infinity, whose log probabilities are all NaN.  Maxima pass over NaNs and limits may be none; there the cells come from
        // the values' order as whole numbers, in which a NaN has its place.
        const bool ordered = s == s;
        auto each = [&](unsigned from, auto f) { each_value<T, P>(p, held, lane * Piece<T>::V - r.head, G * Piece<T>::V, a.K, ordered, from, f); };
        auto largest_order = [&]() {
            unsigned m = 0;
            each(0, [&](unsigned o, unsigned) { m = max(m, o); });
            return m;
        };
        if constexpr (W == 1) {
            if (ordered) wave_top<T, P>(sh, p, most, held, lane * Piece<T>::V - r.head, a.K, a.top, emit);
            else {
                const unsigned own[1] = {largest_order()};
                select_top<1, 1, LOW>(sh, own, a.top, each, emit);
            }
        } else {
            __shared__ Aside<T, HELD> aside;
            if (ordered) {
                const unsigned mine = wave_bound<S, LOW>(cell, (a.top + W - 1) / W);
                if ((lane & 63) == 0) aside.said[lane >> 6] = mine;
                if (lane == 0) aside.count = sh.count = 0;
                __syncthreads();
                const unsigned bound = aside.template hear<W>();
                const float limit = bound >> LOW > order(-INFINITY) >> LOW ? unorder(bound) : LOWEST;
#pragma unroll
                for (int q = 0; q < P; ++q)
                    if (q < held && p[q].template largest<true>() >= limit) aside.put(p[q], q * G + lane);
                __syncthreads();
                if (aside.template rank<W, LOW>(sh, bound, r.head, a.K, a.top, a.K, emit)) return;
                __syncthreads();
            } else {
#pragma unroll
                for (int c = 1; c < S; ++c) cell[c] = 0;
                cell[0] = largest_order();
            }
            select_top<W, S, LOW>(sh, cell, a.top, each, emit);
        }
    } else if (a.dz) {
        const float dl = a.dlogp && given ? a.dlogp[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f;
        // (the scale meets the weights first: divided by the sum it might be too small for a normal number where the product is not)
        const float part = empty ? 0.f : 1.f / s, A = empty ? 0.f : a.scale * (dh * (mean * LN2) - dl) * part, B = -(a.scale * dh) * LN2 * part;
        const int place = given && !empty ? label + r.head : -1;
        auto gradient = [&](int piece, auto how, auto d2_of) {
            float g[Piece<T>::V];
#pragma unroll
            for (int k = 0; k < Piece<T>::V; ++k) g[k] = slope<decltype(how)::value>(d2_of(k), A, B);
            const int at = place - piece * Piece<T>::V;
            if ((unsigned)at < (unsigned)Piece<T>::V) {
#pragma unroll
                for (int k = 0; k < Piece<T>::V; ++k)
                    if (k == at) g[k] += a.scale * dl;
            }
            r.store(piece, g);
            __builtin_amdgcn_sched_barrier(0);      // one piece at a time: several would cost the registers that hold the row
        };
        int again = lane;       // (else the places of all pieces are kept from the loads on, in registers)
        asm volatile("" : "+v"(again));
        auto all = [&](auto how) {
#pragma unroll
            for (int q = 0; q < P; ++q)
                if (q < held) gradient(q * G + again, how, [&](int k) { return sc.d2<true>(p[q].again(k)); });
        };
        auto reread = [&](auto near) {      // rare: the pieces once more from memory, as for the sums
            for (int piece = lane; piece < r.pieces; piece += G) {
                const Piece<T> c = r.load(piece, low);
                gradient(piece, std::integral_constant<int, ANY>(), [&](int k) { return sc.d2<decltype(near)::value>(empty ? -INFINITY : c.at(k)); });
            }
        };
        if (!sc.near) reread(std::false_type());
        else if (!moderate(A, B)) reread(std::true_type());
        else if (masked || fabsf(B) > 1.f) all(std::integral_constant<int, CLAMPED>());
        else all(std::integral_constant<int, PLAIN>());
    }
}

// what a row's sums say
struct Joined {
    float m, s, t;
};
__device__ __forceinline__ void write_row_results(const LogprobArgs &a, size_t row, int label, float zl, const Joined &j)
{
    const bool given = (unsigned)label < (unsigned)a.K, empty = j.s == 0.f;
    const float ls = empty ? 0.f : log2f(j.s);
    const Scale sc(a.scale, j.m);
    if (a.logp) a.logp[row] = !given ? 0.f : empty ? -INFINITY : sc.log_prob(sc.d2<false>(zl), zl, ls);
    if (a.entropy) a.entropy[row] = empty ? 0.f : (ls - j.t / j.s) * LN2;
    if (a.stats) {
        a.stats[2 * row] = empty ? -INFINITY : j.s == j.s ? j.m : j.s;
        a.stats[2 * row + 1] = ls * LN2;
    }
}
__device__ __forceinline__ void write_top(const LogprobArgs &a, size_t row, const Joined &j, int i, unsigned long long key)
{
    const bool none = key == NO_KEY;
    a.top_index[row * a.top + i] = none ? -1 : (int)key_index(key);
    const Scale sc(a.scale, j.m);
    const float z = unorder((unsigned)(key >> 32));
    a.top_logp[row * a.top + i] = none || j.s == 0.f ? -INFINITY : sc.log_prob(sc.d2<false>(z), z, log2f(j.s));
}

// ---- rows that stream by --------------------------------------------------------------------------------------------------
// Without a gradient nothing has to be held: a thread keeps a maximum, and the sums at it, as its pieces pass; four pieces at a time, whose
// values are unpacked once for the maximum and the sums.  Few registers, so that a compute unit has eight workgroups at different places
// of their rows, where rows held in registers leave it two that wait for each other's barriers (4096 rows of 50257: 134 us so).
// A row is one chunk, or several where there are few rows: chunks leave a Part each, which a second launch joins.

constexpr int CHUNK_THREADS = 256;

struct Part {       // of a chunk: its largest value, its sums, and the label's logit
    float m, s, t, zl;
};

// The values of a chunk once more, from memory, for the rare rows whose candidates do not fit their list: cells are every fourth of a
// thread's pieces.
template <typename T, int UNROLL, bool NT>
struct Streamed {
    const Row<T, NT> &r;
    int begin, end, K;
    const unsigned *cell;
    bool ordered;       // as in each_value
    template <class F>
    __device__ __forceinline__ void operator()(unsigned from, F f) const
    {
        constexpr int AHEAD = 4, STEP = UNROLL * CHUNK_THREADS;
        const float limit = unorder(from);      // (NaN for the lowest bounds: then every value is looked at)
        float low = 0.f;
        unsigned hits = 0;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) hits |= cell[u] >= from ? 1u << u : 0u;
        for (; hits; hits &= hits - 1)
            for (int at = begin + (__ffs(hits) - 1) * CHUNK_THREADS + (int)threadIdx.x; at < end; at += AHEAD * STEP) {
                Piece<T> p[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) p[i] = r.load(at + i * STEP, low, end);
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    if (at + i * STEP >= end || (ordered && p[i].template largest<true>() < limit)) continue;
                    int first = (at + i * STEP) * Piece<T>::V - r.head;
                    asm volatile("" : "+v"(first));
#pragma unroll
                    for (int k = 0; k < Piece<T>::V; ++k) {
                        const unsigned o = order(p[i].again(k));
                        if (o >= from && (unsigned)(first + k) < (unsigned)K) f(o, (unsigned)(first + k));
                    }
                }
            }
    }
};

template <typename T, bool TOP, int UNROLL, bool NT>
__global__ __launch_bounds__(CHUNK_THREADS) void logprob_stream_kernel(LogprobArgs a, int chunks, int chunk_pieces, Part *parts, unsigned long long *keys)
{
    constexpr int V = Piece<T>::V, LOW = sizeof(T) == 2 ? 16 : 0;
    __shared__ float red[3][4];
    const size_t row = blockIdx.x / (unsigned)chunks;
    const int chunk = blockIdx.x % (unsigned)chunks, wave = threadIdx.x >> 6;
    const Row<T, NT> r(a, row);
    const int begin = chunk * chunk_pieces, end = min(begin + chunk_pieces, r.pieces);
    const float k2 = a.scale * LOG2E;
    // (read first: two accesses that wait for each other)
    const int label = a.labels ? a.labels[row] : -1;
    const float zl = (unsigned)label < (unsigned)a.K ? load_f32(r.z + r.head + label) : 0.f;
    // the sums are those of exp2((z - m)*k2 + shift): shift is what the rounding of m*k2 moves them by (see Scale)
    float m = LOWEST, shift = 0.f, s = 0.f, t = 0.f, low = 0.f;

    // Candidates for the most probable tokens: pieces with a value that reaches a bound which `top` values have reached so far are set aside as they
    // pass.  The bound comes from what each wave says of its lanes' maxima: its share of `top` lanes have reached it, a quarter, or less of a wave that
    // has fewer lanes with a value, and more of the others.  They say so before the first turn and after 1, 2, 4, ...; a wave may read
    // an older word of another one, which is a bound too.  Minus infinities are never set aside.
    constexpr int CAP = 1024;
    __shared__ Aside<T, TOP ? 640 : 1> aside;
    float limit = LOWEST, seen = -INFINITY, of[UNROLL];
    int turn = 0, share = 0;        // share: less than 0 where there are not `top` lanes
    auto say = [&]() {
        const unsigned cells[1] = {order(seen)};
        const unsigned b = share > 0 ? wave_bound<1, LOW>(cells, share) : share == 0 ? 0xFFFFFFFFu : 0u;
        if ((threadIdx.x & 63) == 0) *(volatile unsigned *)&aside.said[wave] = b;
    };
    auto hear = [&]() {
        const unsigned b = aside.template hear<4>();
        limit = b >> LOW > order(-INFINITY) >> LOW ? unorder(b) : LOWEST;
    };
    if constexpr (TOP) {
        if (threadIdx.x == 0) aside.count = 0;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) of[u] = -INFINITY;
    }
    Piece<T> p[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) p[u] = r.load(begin + u * CHUNK_THREADS + (int)threadIdx.x, low, end);
    if constexpr (TOP) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) seen = fmaxf(seen, p[u].template largest<true>());
        const unsigned lanes = (unsigned)__popcll(__ballot(seen > -INFINITY));
        if ((threadIdx.x & 63) == 0) aside.said[4 + wave] = lanes;
        __syncthreads();
        unsigned most = (unsigned)(a.top + 3) / 4, total = 0;
        for (; most <= 64u; ++most) {
            total = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) total += min(aside.said[4 + w], most);
            if (total >= (unsigned)a.top) break;
        }
        share = total >= (unsigned)a.top ? (int)min(lanes, most) : -1;
        say();
        __syncthreads();
        hear();
    }
    for (int base = begin; base < end; base += UNROLL * CHUNK_THREADS) {
        Piece<T> c[UNROLL];
        const int next = base + UNROLL * CHUNK_THREADS;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            c[u] = p[u];
            if (next < end) p[u] = r.load(next + u * CHUNK_THREADS + (int)threadIdx.x, low, end);
        }
        float z[UNROLL][V], most = m;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
            for (int k = 0; k < V; ++k) z[u][k] = c[u].at(k);
            float x = z[u][0];
#pragma unroll
            for (int k = 1; k + 1 < V; k += 2) x = max3(x, z[u][k], z[u][k + 1]);
            x = max3(x, z[u][V - 1], z[u][V - 1]);
            most = fmaxf(most, x);
            if constexpr (TOP) {
                of[u] = fmaxf(of[u], x);
                if (x >= limit && !aside.put(c[u], base + u * CHUNK_THREADS + (int)threadIdx.x)) limit = INFINITY;     // too many: they are looked for once more below
            }
        }
        // the sums so far at the new maximum
        const Scale sc(a.scale, most);
        const bool near = __ballot(!sc.near) == 0;
        const float to = near ? fmaf(most, k2, sc.c) : 0.f;
        const float down = fmaxf(fmaf(m - most, k2, to - shift), NO_WEIGHT), by = __builtin_amdgcn_exp2f(down);
        t = fmaf(down, s, t) * by;
        s *= by;
        m = most;
        shift = to;
        auto sums = [&](auto near) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float d = sc.d2<decltype(near)::value>(z[u][k]), e = __builtin_amdgcn_exp2f(d);
                    s += e;
                    t = fmaf(e, weight<true>(d), t);
                }
            }
        };
        if (near) sums(std::true_type());
        else sums(std::false_type());
        if constexpr (TOP) {
            ++turn;
            if ((turn & (turn - 1)) == 0 && next < end && limit < INFINITY) {
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) seen = fmaxf(seen, of[u]);
                say();
                hear();
            }
        }
    }
    if constexpr (TOP) {
        if (end - begin > UNROLL * CHUNK_THREADS) {     // (else it has been said)
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) seen = fmaxf(seen, of[u]);
            say();
        }
    }
    float most = meet<64>(m, larger);
    if ((threadIdx.x & 63) == 0) red[0][wave] = most;
    __syncthreads();
    most = max3(max3(red[0][0], red[0][1], red[0][2]), red[0][3], LOWEST);
    const float down = fmaxf(fmaf(m - most, k2, -shift), NO_WEIGHT), by = __builtin_amdgcn_exp2f(down);
    t = meet<64>(fmaf(down, s, t) * by, sum);
    s = meet<64>(s * by, sum);
    if ((threadIdx.x & 63) == 0) {
        red[1][wave] = s;
        red[2][wave] = t;
    }
    __shared__ TopShared<TOP ? CAP : 1> sh;
    if (TOP && threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    const Joined j{most, red[1][0] + red[1][1] + red[1][2] + red[1][3], red[2][0] + red[2][1] + red[2][2] + red[2][3]};
    if (threadIdx.x == 0) {
        if (parts) parts[blockIdx.x] = Part{j.m, j.s, j.t, zl};
        else write_row_results(a, row, label, zl, j);
    }
    if constexpr (TOP) {
        auto emit = [&](int i, unsigned long long key) {
            if (parts) keys[(size_t)blockIdx.x * a.top + i] = key;
            else write_top(a, row, j, i, key);
        };
        const int first = max(begin * V - r.head, 0), values = min(end * V - r.head, a.K) - first;
        if (j.s == 0.f) {       // minus infinities alone
            if ((int)threadIdx.x < a.top) emit(threadIdx.x, (int)threadIdx.x < values ? key_of(order(-INFINITY), (unsigned)(first + (int)threadIdx.x)) : NO_KEY);
            return;
        }
        const bool ordered = j.s == j.s;        // (as in logprob_row_kernel)
        if (ordered && aside.template rank<4, LOW>(sh, aside.template hear<4>(), r.head, a.K, a.top, values, emit)) return;
        __syncthreads();
        unsigned cell[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) cell[u] = ordered && begin + u * CHUNK_THREADS + (int)threadIdx.x < end ? order(of[u]) : 0u;
        const Streamed<T, UNROLL, NT> each{r, begin, end, a.K, cell, ordered};
        if (!ordered) {
            unsigned largest[UNROLL] = {};
            each(0, [&](unsigned o, unsigned index) {
                const int turn = ((int)index + r.head) / V - begin;     // of pieces, in which u comes round
#pragma unroll
                for (int u = 0; u < UNROLL; ++u)
                    if (turn / CHUNK_THREADS % UNROLL == u) largest[u] = max(largest[u], o);
            });
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) cell[u] = largest[u];
        }
        select_top<4, UNROLL, LOW>(sh, cell, a.top, each, emit);
    }
}

// ---- chunks ---------------------------------------------------------------------------------------------------------------

// the chunks' sums at the row's maximum, in the chunks' order within each thread and the threads' in a fixed one
template <int W>
__device__ __forceinline__ Joined join_parts(const Part *parts, int chunks, float scale, float (*red)[W])
{
    const int wave = threadIdx.x >> 6;
    float m = LOWEST;
    for (int c = threadIdx.x; c < chunks; c += 64 * W) m = fmaxf(m, parts[c].m);
    m = meet<64>(m, larger);
    if ((threadIdx.x & 63) == 0) red[0][wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, red[0][w]);
    const Scale sc(scale, m);
    float s = 0.f, t = 0.f;
    for (int c = threadIdx.x; c < chunks; c += 64 * W) {
        const Part q = parts[c];
        const float d = sc.d2<false>(q.m), e = __builtin_amdgcn_exp2f(d);
        s = fmaf(q.s, e, s);
        t = fmaf(fmaf(fmaxf(d, NO_WEIGHT), q.s, q.t), e, t);
    }
    s = meet<64>(s, sum);
    t = meet<64>(t, sum);
    if ((threadIdx.x & 63) == 0) {
        red[1][wave] = s;
        red[2][wave] = t;
    }
    __syncthreads();
    Joined j{m, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
        j.s += red[1][w];
        j.t += red[2][w];
    }
    return j;
}

// What chunks found out about a row, joined by one wave.  A chunk's keys are in descending order: the first ones of each give the bound, and a lane goes
// down its chunks' lists as far as that.  Up to 64 chunks: the lanes hold the first 256 keys counted across the lists, which holds all that matters but for
// rare rows; more: the first four of each.
template <typename T, bool TOP>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a, int chunks, const Part *parts, const unsigned long long *keys)
{
    constexpr int DEPTH = 4, LOW = sizeof(T) == 2 ? 16 : 0;
    __shared__ float red[3][1];
    const size_t row = blockIdx.x;
    const int lane = threadIdx.x, top = a.top;
    parts += row * chunks;
    const int label = a.labels ? a.labels[row] : -1;
    const float zl = parts[0].zl;       // (every chunk has it)
    unsigned cell[DEPTH] = {};
    unsigned long long own[DEPTH] = {};
    const bool across = chunks <= 64;
    if constexpr (TOP) {
        keys += row * chunks * top;
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int e = lane + 64 * d, c = across ? e % chunks : lane, at = across ? e / chunks : d;
            own[d] = at < top ? keys[(size_t)c * top + at] : NO_KEY;
        }
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) cell[d] = (unsigned)(own[d] >> 32);
        for (int c = lane + 64; c < chunks; c += 64)
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) cell[d] = max(cell[d], d < top ? (unsigned)(keys[(size_t)c * top + d] >> 32) : 0u);
    }
    const Joined j = join_parts<1>(parts, chunks, a.scale, red);
    if (lane == 0) write_row_results(a, row, label, zl, j);
    if constexpr (TOP) {
        auto emit = [&](int i, unsigned long long key) { write_top(a, row, j, i, key); };
        if (j.s == 0.f) {       // minus infinities alone
            if (lane < top) emit(lane, lane < a.K ? key_of(order(-INFINITY), (unsigned)lane) : NO_KEY);
            return;
        }
        constexpr int CAP = 1024;
        __shared__ TopShared<CAP> sh;
        if (lane == 0) sh.count = 0;
        __syncthreads();
        const unsigned bound = wave_bound<DEPTH, LOW>(cell, top);
        // Many equal values: the index decides among those at the bound as well.
        unsigned long long least = (unsigned long long)bound << 32;
        int above = 0, reach = 0;
        unsigned low[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const bool equal = cell[d] >> LOW == bound >> LOW;
            above += __popcll(__ballot(cell[d] >= bound && !equal));
            reach += __popcll(__ballot(cell[d] >= bound));
            low[d] = equal ? (unsigned)own[d] : 0u;
        }
        if (across && reach > top + 32) {
            const unsigned index = wave_bound<DEPTH, 0>(low, top - above);
            least = (unsigned long long)(bound | (LOW ? (1u << LOW) - 1u : 0u)) << 32 | index;
        }
        auto take = [&](unsigned long long key) {       // whether to go on down the list
            // (keys at the bound differ in what lies below LOW only by their sign's fill: there all of them count as the largest)
            const unsigned o = (unsigned)(key >> 32);
            const unsigned long long as = o >> LOW == bound >> LOW ? (key | (unsigned long long)(LOW ? (1u << LOW) - 1u : 0u) << 32) : key;
            if (key == NO_KEY || as < least) return false;
            const int at = atomicAdd(&sh.count, 1);
            if (at < CAP) sh.list[at] = key;
            return at < CAP;
        };
        bool on = true;
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) on = (across || on) && take(own[d]);
        if (across) {       // what lies below the keys that were held
            if (lane < chunks)
                for (int i = (64 * DEPTH - lane + chunks - 1) / chunks; i < top && take(keys[(size_t)lane * top + i]); ++i) {}
        } else
            for (int c = lane, i = DEPTH; c < chunks; c += 64, i = 0, on = true)
                for (; on && i < top; ++i) on = take(keys[(size_t)c * top + i]);
        __syncthreads();
        const int n = sh.count;
        if (n <= CAP) {
            rank_candidates<1>(sh, n, top, emit);
            return;
        }
        __syncthreads();
        select_top<1, DEPTH, LOW>(
            sh, cell, top,
            [&](unsigned from, auto f) {
                for (int c = lane; c < chunks; c += 64)
                    for (int i = 0; i < top; ++i) {
                        const unsigned long long key = keys[(size_t)c * top + i];
                        if (key == NO_KEY || (unsigned)(key >> 32) < from) break;
                        f((unsigned)(key >> 32), key_index(key));
                    }
            },
            emit);
    }
}

// the gradient of a workgroup's 256*P pieces; mean: T/S in d2's units
template <typename T, int P>
__device__ __forceinline__ void block_gradient(const LogprobArgs &a, size_t row, int block, float m, float s, float mean, bool empty)
{
    constexpr int V = Piece<T>::V;
    const Row<T> r(a, row);
    const Scale sc(a.scale, m);
    const int label = a.labels ? a.labels[row] : -1;
    const bool given = (unsigned)label < (unsigned)a.K;
    const float dl = a.dlogp && given ? a.dlogp[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f;
    const float part = 1.f / s, A = a.scale * (dh * (mean * LN2) - dl) * part, B = -(a.scale * dh) * LN2 * part;        // (as in logprob_row_kernel)
    const int place = given ? label + r.head : -1;
    const int piece0 = block * (CHUNK_THREADS * P) + (int)threadIdx.x;
    Piece<T> p[P];
    float low = 0.f;        // (above nothing that matters)
#pragma unroll
    for (int q = 0; q < P; ++q) p[q] = r.load(piece0 + q * CHUNK_THREADS, low);
    auto all = [&](auto how) {
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int piece = piece0 + q * CHUNK_THREADS;
            float g[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                g[k] = slope<decltype(how)::value>(sc.d2<false>(p[q].at(k)), A, B) + (place == piece * V + k ? a.scale * dl : 0.f);
                if (empty) g[k] = 0.f;
            }
            r.store(piece, g);
        }
    };
    if (moderate(A, B)) all(std::integral_constant<int, CLAMPED>());
    else all(std::integral_constant<int, ANY>());
}

template <typename T, int P>
__global__ __launch_bounds__(CHUNK_THREADS) void logprob_gradient_kernel(LogprobArgs a, int blocks, int chunks, const Part *parts)
{
    __shared__ float red[3][4];
    const size_t row = blockIdx.x / (unsigned)blocks;
    const int block = blockIdx.x % (unsigned)blocks;
    parts += row * chunks;
    const int label = a.labels ? a.labels[row] : -1;
    const float zl = parts[0].zl;       // (the gradient may take z's place)
    const Joined j = join_parts<4>(parts, chunks, a.scale, red);
    if (block == 0 && threadIdx.x == 0) write_row_results(a, row, label, zl, j);
    block_gradient<T, P>(a, row, block, j.m, j.s, j.t / j.s, j.s == 0.f);
}

template <typename T, int P>
__global__ __launch_bounds__(CHUNK_THREADS) void logprob_bwd_kernel(LogprobArgs a, int blocks, const float *stats, const float *entropy)
{
    const size_t row = blockIdx.x / (unsigned)blocks;
    const float m = stats[2 * row], ls = stats[2 * row + 1];
    block_gradient<T, P>(a, row, blockIdx.x % (unsigned)blocks, m, expf(ls), entropy ? (ls - entropy[row]) * LOG2E : 0.f, m == -INFINITY);
}

// ---- host -----------------------------------------------------------------------------------------------------------------

// 16-byte pieces that a row of K values has where all rows begin on one (ld a multiple of a piece), or may have
int row_pieces(int K, int dtype, int ld)
{
    const int V = 16 / (int)elem_size(dtype);
    return (int)(((long long)K + (ld % V == 0 ? V - 1 : 2 * V - 2)) / V);
}
constexpr int ANY_LD = 1;

constexpr int ROW_PIECES = 16384;       // in registers: 16 of each of 1024 threads
constexpr int SHORT_PIECES = 1024;      // rows that are held in registers without a gradient too

// How a row is cut where it is not held: chunks, and pieces of each.
struct Cut {
    int chunks, pieces;     // chunks 0: rows are held
};
Cut cut_rows(int N, int pieces, bool gradient)
{
    // A gradient's rows are held, but for long ones where there are few: 131072 of bf16 took 20.4 us held and 13.9 in chunks at 64 rows, 23.3 and 21.2 at 128,
    // 29.4 and 31.5 at 192; 58262 of them 11.5 and 6.9 at 2, 12.7 and 12.6 at 64; 30000 7.4 and 6.2 at 2, 8.0 and 8.2 at 64.
    if (pieces <= SHORT_PIECES || (gradient && (pieces <= 2 * SHORT_PIECES || (pieces <= ROW_PIECES / 2 && N >= 64) || (pieces <= ROW_PIECES && N >= 160)))) return Cut{0, 0};
    // Without one, from 256 rows on a row is one workgroup and one launch: 4 (512 rows and more: 2) chunks each, 131072 of bf16 with 20 best tokens, 28.9 and 26.0 in
    // chunks at 256 rows, 35.1 and 36.9 at 400, 54.8 and 63.1 at 1000; without best tokens 16.8 and 16.7, 23.3 and 26.0, 49.1 and 55.2; 50257 18.0 and 19.8,
    // 20.6 and 24.9, 29.5 and 39.8; 20000 11.4 and 14.7, 13.3 and 16.6, 17.8 and 28.1.
    int chunks = N >= 256 ? 1 : (1024 + N - 1) / N;
    chunks = chunks < (pieces + CHUNK_THREADS - 1) / CHUNK_THREADS ? chunks : (pieces + CHUNK_THREADS - 1) / CHUNK_THREADS;
    Cut c;
    c.pieces = (pieces + chunks - 1) / chunks;
    c.chunks = (pieces + c.pieces - 1) / c.pieces;
    return c;
}
int block_count(int pieces, int per_thread) { return (int)((pieces + (long long)CHUNK_THREADS * per_thread - 1) / (CHUNK_THREADS * per_thread)); }

// Whether the logits alone fill the 256 MB of the last cache: then accesses go past the caches.  4096 rows of 50257 bf16: 90 -> 86 us with the top
// tokens, 161 -> 152 with the gradient; the gradient of 131072 does not gain.
bool past_caches(const LogprobArgs &a) { return (size_t)a.N * a.ld * elem_size(a.dtype) > (size_t)256 << 20; }

template <typename T, bool TOP>
void launch_row(const LogprobArgs &a, hipStream_t st)
{
    const int pieces = row_pieces(a.K, a.dtype, a.ld);
    const dim3 rows((unsigned)a.N);
    if (!TOP && pieces <= 8) {
        hipLaunchKernelGGL((logprob_row_kernel<T, 8, 1, false>), dim3((unsigned)((a.N + 31ll) / 32)), dim3(256), 0, st, a);
        return;
    }
    if (pieces <= 64) hipLaunchKernelGGL((logprob_row_kernel<T, 64, 1, TOP>), rows, dim3(64), 0, st, a);
    else if (pieces <= 256) hipLaunchKernelGGL((logprob_row_kernel<T, 64, 4, TOP>), rows, dim3(64), 0, st, a);
    else if (pieces <= 512) hipLaunchKernelGGL((logprob_row_kernel<T, 256, 2, TOP>), rows, dim3(256), 0, st, a);
    else if (TOP || pieces <= 1024) hipLaunchKernelGGL((logprob_row_kernel<T, 256, 4, TOP>), rows, dim3(256), 0, st, a);
    else if (pieces <= 2048) hipLaunchKernelGGL((logprob_row_kernel<T, 256, 8, false>), rows, dim3(256), 0, st, a);
    else {
        const bool past = past_caches(a);
        if (pieces <= 4096) hipLaunchKernelGGL((past ? logprob_row_kernel<T, 512, 8, false, true> : logprob_row_kernel<T, 512, 8, false>), rows, dim3(512), 0, st, a);
        else if (pieces <= 8192) hipLaunchKernelGGL((past ? logprob_row_kernel<T, 512, 16, false, true> : logprob_row_kernel<T, 512, 16, false>), rows, dim3(512), 0, st, a);
        else hipLaunchKernelGGL((logprob_row_kernel<T, 1024, 16, false>), rows, dim3(1024), 0, st, a);
    }
}

template <typename T>
int launch(const LogprobArgs &a, void *workspace, hipStream_t st)
{
    const int pieces = row_pieces(a.K, a.dtype, a.ld);
    const Cut cut = cut_rows(a.N, pieces, a.dz != nullptr);
    if (cut.chunks == 0) {
        if (!one_launch(a.N + 31ll, !a.top && pieces <= 8 ? 8 : pieces <= 256 ? 64 : pieces <= 2048 ? 256 : pieces <= 8192 ? 512 : 1024)) return MXC_ERR_SHAPE;
        if (a.top) launch_row<T, true>(a, st);
        else launch_row<T, false>(a, st);
        return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
    }
    const size_t grid = (size_t)a.N * cut.chunks;
    const int per = pieces <= 2048 || a.N < 160 ? 1 : 4, blocks = block_count(pieces, per);
    if (!one_launch(grid, CHUNK_THREADS) || (a.dz && !one_launch((size_t)a.N * blocks, CHUNK_THREADS))) return MXC_ERR_SHAPE;
    const bool alone = cut.chunks == 1 && !a.dz;
    Part *parts = alone ? nullptr : (Part *)workspace;
    unsigned long long *keys = (unsigned long long *)((char *)workspace + align_up(grid * sizeof(Part), 256));
    const dim3 g((unsigned)grid), b(CHUNK_THREADS);
    const bool past = !a.dz && past_caches(a);      // (what a gradient reads once more should stay)
    // a piece a thread: short code, whose fetching counts
    const bool once = cut.pieces <= CHUNK_THREADS;
    if (a.top && once) hipLaunchKernelGGL((logprob_stream_kernel<T, true, 1, false>), g, b, 0, st, a, cut.chunks, cut.pieces, parts, keys);
    else if (a.top && past) hipLaunchKernelGGL((logprob_stream_kernel<T, true, 4, true>), g, b, 0, st, a, cut.chunks, cut.pieces, parts, keys);
    else if (a.top) hipLaunchKernelGGL((logprob_stream_kernel<T, true, 4, false>), g, b, 0, st, a, cut.chunks, cut.pieces, parts, keys);
    else if (once) hipLaunchKernelGGL((logprob_stream_kernel<T, false, 1, false>), g, b, 0, st, a, cut.chunks, cut.pieces, parts, keys);
    else if (past) hipLaunchKernelGGL((logprob_stream_kernel<T, false, 4, true>), g, b, 0, st, a, cut.chunks, cut.pieces, parts, keys);
    else hipLaunchKernelGGL((logprob_stream_kernel<T, false, 4, false>), g, b, 0, st, a, cut.chunks, cut.pieces, parts, keys);
    if (hipGetLastError() != hipSuccess) return MXC_ERR_LAUNCH;
    if (alone) return MXC_OK;
    const dim3 gg((unsigned)((size_t)a.N * blocks));
    if (!a.dz && a.top) hipLaunchKernelGGL((logprob_join_kernel<T, true>), dim3((unsigned)a.N), dim3(64), 0, st, a, cut.chunks, parts, keys);
    else if (!a.dz) hipLaunchKernelGGL((logprob_join_kernel<T, false>), dim3((unsigned)a.N), dim3(64), 0, st, a, cut.chunks, parts, keys);
    else if (per == 1) hipLaunchKernelGGL((logprob_gradient_kernel<T, 1>), gg, b, 0, st, a, blocks, cut.chunks, parts);
    else hipLaunchKernelGGL((logprob_gradient_kernel<T, 4>), gg, b, 0, st, a, blocks, cut.chunks, parts);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

template <typename T>
int launch_bwd(const LogprobArgs &a, const float *stats, const float *entropy, hipStream_t st)
{
    const int pieces = row_pieces(a.K, a.dtype, a.ld), per = pieces <= CHUNK_THREADS ? 1 : 4, blocks = block_count(pieces, per);
    const size_t grid = (size_t)a.N * blocks;
    if (!one_launch(grid, CHUNK_THREADS)) return MXC_ERR_SHAPE;
    const dim3 g((unsigned)grid), b(CHUNK_THREADS);
    if (per == 1) hipLaunchKernelGGL((logprob_bwd_kernel<T, 1>), g, b, 0, st, a, blocks, stats, entropy);
    else hipLaunchKernelGGL((logprob_bwd_kernel<T, 4>), g, b, 0, st, a, blocks, stats, entropy);
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

}  // namespace

size_t logprob_workspace(int N, int K, int dtype, int top)
{
    size_t need = 0;
    for (int ld : {0, ANY_LD})      // whatever ld the call has
        for (bool gradient : {false, true}) {
            const Cut c = cut_rows(N, row_pieces(K, dtype, ld), gradient);
            const size_t grid = (size_t)N * c.chunks, bytes = c.chunks == 0 || (c.chunks == 1 && !gradient) ? 0 : align_up(grid * sizeof(Part), 256) + grid * top * sizeof(unsigned long long);
            need = bytes > need ? bytes : need;
        }
    return need;
}

int logprob_rows(const LogprobArgs &a, void *workspace, hipStream_t st)
{
    return a.dtype == MXC_BF16 ? launch<bf16_t>(a, workspace, st) : launch<float>(a, workspace, st);
}

int logprob_bwd(const LogprobArgs &a, const float *stats, const float *entropy, hipStream_t st)
{
    return a.dtype == MXC_BF16 ? launch_bwd<bf16_t>(a, stats, entropy, st) : launch_bwd<float>(a, stats, entropy, st);
}

}  // namespace mxc
