// FullyConnected on a filter in microscaled 4-bit floating point: y[n][k] = act( sum_c q(x)[n][c]*w[k][c] + bias[k] ).
// The matrix instructions take 4-bit operands as they are, 32 values of a row and their scale byte in each lane, multiply and add
// them in fp32.  The product is formed transposed (filter rows first), so that a lane holds four neighbouring columns of y.
//   token:  up to 8 rows of x.  One launch: every wave quantises the part of x that it multiplies.
//   skinny: some rows, or few filter rows: x is quantised once, then workgroups of eight waves that share out the columns.
//   tiled:  x quantised, both operands' scales brought into the order of the tiles, and tiles of LDS that a ring of loads fills.
#include <type_traits>

#include "mxfp4.h"

namespace mxc {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ i32x8 operand(uint4 u) { return i32x8{(int)u.x, (int)u.y, (int)u.z, (int)u.w, 0, 0, 0, 0}; }
constexpr int FP4 = 4;      // the instructions' code for the operands' format

// byte J of the scale words belongs to these operands
template <int J, int L>
__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), c, FP4, FP4, J, sa, L, sb);
}
template <int J>
__device__ __forceinline__ f32x16 mfma32(uint4 a, uint4 b, f32x16 c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a), operand(b), c, FP4, FP4, J, sa, J, sb);
}

template <typename T>
__device__ __forceinline__ void store_one(T *y, float v)
{
    if constexpr (sizeof(T) == 2) *y = (bf16_t)pack_bf16x2(v, v);
    else *y = v;
}
__device__ __forceinline__ float activated(float v, const float *bias, long long k, int relu)
{
    if (bias) v += bias[k];
    return relu && v < 0.f ? 0.f : v;
}

// ---- 16 rows of the filter straight from memory -----------------------------------------------------------------------------
// The instruction wants block l/16 of row l%16 in lane l.  Read so, neighbouring lanes are rows apart, and the 64 lanes' 16 bytes take 64 turns of the
// address unit; read as block l%4 of row l/4, four lanes a 64-byte piece, they take 16, and each word changes its lane through LDS.
__device__ __forceinline__ uint4 to_operand(uint4 v, int lane)
{
    const int from = (((lane & 15) << 2) | (lane >> 4)) << 2;       // byte address of the lane that has it
    return make_uint4((unsigned)__builtin_amdgcn_ds_bpermute(from, (int)v.x), (unsigned)__builtin_amdgcn_ds_bpermute(from, (int)v.y),
                      (unsigned)__builtin_amdgcn_ds_bpermute(from, (int)v.z), (unsigned)__builtin_amdgcn_ds_bpermute(from, (int)v.w));
}
__device__ __forceinline__ int to_operand(unsigned v, int lane) { return __builtin_amdgcn_ds_bpermute((((lane & 15) << 2) | (lane >> 4)) << 2, (int)v); }

struct FilterRows {
    const unsigned char *codes, *scales;        // of row l/4 of the 16
    int blocks, part;                           // part: l%4
    __device__ __forceinline__ FilterRows() {}
    __device__ __forceinline__ FilterRows(const unsigned char *wc, const unsigned char *ws, long long k0, int K, int blocks_, int scale_row, int lane)
        : blocks(blocks_), part(lane & 3)
    {
        const long long k = k0 + (lane >> 2), row = k < K ? k : K - 1;
        codes = wc + (size_t)row * blocks * 16;
        scales = ws + (size_t)row * scale_row;
    }
    // codes and scale of a step of 128 columns
    __device__ __forceinline__ uint4 load(int step) const
    {
        const int b = step * 4 + part;
        return b < blocks ? *reinterpret_cast<const uint4 *>(codes + (size_t)b * 16) : make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ unsigned load_scale(int step) const { return scales[step * 4 + part]; }
};

// ---- up to 8 rows of x ----------------------------------------------------------------------------------------------------
// 16 filter rows a workgroup; its WAVES waves take every WAVES-th group of 512 columns in four steps of 128.  A wave brings its columns of x into
// 4 bits by itself, eight values a lane, and passes the codes through LDS to the lanes that multiply them: lane l holds a block of
// filter row l%16 and one of row l%16 of x.  1 row of 4096 by 4096 4.2 us, of which most is a launch and one chain of load, quantise, multiply, join;
// of 16384 by 16384 30 us, 4.7 TB/s.

constexpr int TOKEN_ROWS = 8;

struct TokenRow {       // of x: the codes and scales of a group, and room that spreads rows over the banks
    unsigned codes[64];
    unsigned char scales[16];
};

template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mxfp4_token_kernel(int N, int C, int K, int blocks, int scale_row, const T *x, const unsigned char *wc,
                                                                       const unsigned char *ws, const float *bias, int relu, T *y)
{
    constexpr int BATCH = 4;        // rows of x whose loads are under way together
    __shared__ f32x4 part[WAVES][64];
    __shared__ __align__(16) TokenRow rows[WAVES][TOKEN_ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, quarter = lane >> 4;
    const long long k0 = (long long)blockIdx.x * 16;
    const FilterRows filter(wc, ws, k0, K, blocks, scale_row, lane);
    const int groups = scale_row / 16;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    uint4 next[4];
    unsigned next_scale[4];
    auto ahead = [&](int group) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            next[j] = filter.load(group * 4 + j);
            next_scale[j] = filter.load_scale(group * 4 + j);
        }
    };
    if (wave < groups) ahead(wave);
    for (int group = wave; group < groups; group += WAVES) {
        uint4 w[4];
        unsigned sw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = next[j];
            sw[j] = next_scale[j];
        }
        const int column = group * 512 + lane * 8;
#pragma unroll 1
        for (int n0 = 0; n0 < N; n0 += BATCH) {
            float v[BATCH][8];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (n0 + i >= N) break;
                load8_edge(x + (size_t)(n0 + i) * C + column, C - column, v[i]);
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (n0 + i >= N) break;
                const unsigned byte = mxfp4_scale_byte(max_quad(largest8(v[i])));
                TokenRow &to = rows[wave][n0 + i];
                to.codes[lane] = mxfp4_codes8(v[i], byte);
                if ((lane & 3) == 0) to.scales[lane >> 2] = (unsigned char)byte;
            }
        }
        if (group + WAVES < groups) ahead(group + WAVES);       // (after x, whose arrival would be waited for behind it)
        // (a wave's own accesses to LDS keep their order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const TokenRow &from = rows[wave][r % TOKEN_ROWS];
        const bool live = r < N;
        const uint4 scales = *reinterpret_cast<const uint4 *>(from.scales);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 c = *reinterpret_cast<const uint4 *>(from.codes + (4 * j + quarter) * 4);
            unsigned sx = j == 0 ? scales.x : j == 1 ? scales.y : j == 2 ? scales.z : scales.w;
            if (!live) {
                c = make_uint4(0, 0, 0, 0);
                sx = 0;
            }
            acc = mfma16<0, 0>(to_operand(w[j], lane), c, acc, to_operand(sw[j], lane), (int)(sx >> (8 * quarter)));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    part[wave][lane] = acc;
    __syncthreads();
    // thread t: column t/16 of the tile's sixteen, row t%16 of x
    const int t = threadIdx.x;
    const int n = t & 15, kk = t >> 4;
    if (t >= 256 || n >= N || k0 + kk >= K) return;
    const float *p = reinterpret_cast<const float *>(&part[0][(kk >> 2) * 16 + n]) + (kk & 3);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += p[w * 256];
    store_one(y + (size_t)n * K + k0 + kk, activated(sum, bias, k0 + kk, relu));
}

// ---- some rows of x -------------------------------------------------------------------------------------------------------
// x in the order in which the waves read it: [16 rows][step of 128 columns][lane] of 16 bytes of codes, lane l: row l%16, block l/16 of the step, and
// the same of bytes of scales.  Rows past N are zeros.
template <typename T>
__global__ __launch_bounds__(256) void mxfp4_order_kernel(int N, int C, int groups, const T *x, unsigned *xc, unsigned *xs)
{
    __shared__ unsigned char bytes[4][64];
    const int group = (int)(blockIdx.x % (unsigned)groups), tile = (int)(blockIdx.x / (unsigned)groups);
    const int quarter = threadIdx.x & 3, row = threadIdx.x >> 4, at = (threadIdx.x >> 2) & 3;       // four lanes a block, the step's block `at`
    const int n = tile * 16 + row, lane = row + 16 * at;
    float v[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int column = group * 512 + j * 128 + at * 32 + quarter * 8;
        load8_edge(x + (n < N ? (size_t)n * C + column : 0), n < N ? C - column : 0, v[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const unsigned byte = mxfp4_scale_byte(max_quad(largest8(v[j])));
        if (quarter == 0) bytes[j][lane] = (unsigned char)byte;
        xc[(((size_t)blockIdx.x * 4 + j) * 64 + lane) * 4 + quarter] = mxfp4_codes8(v[j], byte);
    }
    __syncthreads();
    if (threadIdx.x < 64) xs[(size_t)blockIdx.x * 64 + threadIdx.x] = reinterpret_cast<const unsigned *>(bytes)[threadIdx.x];
}

// 16*WF filter rows and 16*NF rows of x a workgroup, both straight from the caches into registers; its eight waves take every eighth step of
// 128 columns, and their sums meet in LDS.  A step is under way while one is multiplied (two were no faster).
// What a compute unit reads through its L2 bounds the steps: 128 rows by 4096 take 6.6, 10.6 and 17.1 us for 4608, 9216 and 18432 columns, so 0.7 to 0.9 us for each
// step of 52 KB a workgroup, and 3 us to begin and to join; with steps of 26 KB (32 rows of x) 9216 columns take 6.5 us.  Ordering x is another 3 to 4 us.
template <typename T, int WF, int NF>
__global__ __launch_bounds__(512) void mxfp4_skinny_kernel(int N, int K, int blocks, int scale_row, const unsigned char *xc, const unsigned char *xs,
                                                           const unsigned char *wc, const unsigned char *ws, const float *bias, int relu, T *y)
{
    constexpr int WAVES = 8;
    __shared__ f32x4 part[WAVES][WF * NF][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int groups = scale_row / 16, tiles = (N + 15) / 16, tile0 = blockIdx.y * NF, all = (blocks + 3) / 4;
    const long long k0 = (long long)blockIdx.x * (16 * WF);
    FilterRows filter[WF];
#pragma unroll
    for (int i = 0; i < WF; ++i) filter[i] = FilterRows(wc, ws, k0 + 16 * i, K, blocks, scale_row, lane);
    // first steps of each tile of x (the last tile again where there are fewer); places are counted in 32 bits: at most 2^14 rows of 2^23 columns
    // are 2^32 lanes' pieces
    unsigned first[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) first[i] = (unsigned)min(tile0 + i, tiles - 1) * (unsigned)groups * 4u;
    f32x4 acc[WF][NF] = {};
    struct Step {
        uint4 w[WF], x[NF];
        unsigned sw[WF];
        int sx[NF];
    } place[2];
    auto load = [&](Step &s, int step) {
#pragma unroll
        for (int i = 0; i < WF; ++i) {
            s.w[i] = filter[i].load(step);
            s.sw[i] = filter[i].load_scale(step);
        }
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const unsigned at = (first[i] + (unsigned)step) * 64u + (unsigned)lane;
            s.x[i] = reinterpret_cast<const uint4 *>(xc)[at];
            s.sx[i] = xs[at];
        }
    };
    auto multiply = [&](const Step &s) {
#pragma unroll
        for (int i = 0; i < WF; ++i) {
            const uint4 w = to_operand(s.w[i], lane);
            const int sw = to_operand(s.sw[i], lane);
#pragma unroll
            for (int q = 0; q < NF; ++q) acc[i][q] = mfma16<0, 0>(w, s.x[q], acc[i][q], sw, s.sx[q]);
        }
    };
    if (wave < all) load(place[0], wave);
    for (int step = wave; step < all; step += 2 * WAVES) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int now = step + u * WAVES;
            if (now >= all) break;
            if (now + WAVES < all) load(place[1 - u], now + WAVES);
            multiply(place[u]);
        }
    }
#pragma unroll
    for (int i = 0; i < WF; ++i)
#pragma unroll
        for (int q = 0; q < NF; ++q) part[wave][i * NF + q][lane] = acc[i][q];
    __syncthreads();
    // a thread: four neighbouring columns of a row, in ascending order of waves
    for (int u = threadIdx.x; u < WF * NF * 64; u += 512) {
        const int f = u >> 6, l = u & 63;
        f32x4 v = part[0][f][l];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += part[w][f][l];
        const long long k = k0 + (f / NF) * 16 + (l >> 4) * 4, n = (tile0 + f % NF) * 16ll + (l & 15);
        if (n >= N) continue;
        T *to = y + (size_t)n * K + k;
        if (k + 4 <= K) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = activated(v[e], bias, k + e, relu);
            if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_any *>(to) = u32x2_any{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
            else *reinterpret_cast<f32x4_any *>(to) = f32x4_any{v[0], v[1], v[2], v[3]};
        } else
            for (int e = 0; k + e < K; ++e) store_one(to + e, activated(v[e], bias, k + e, relu));
    }
}

// ---- many rows of x -------------------------------------------------------------------------------------------------------
// Scales in the tiles' order: for 32 rows and 256 columns one word a lane, lane l: row l%32 and of the 8 blocks those of l/32's parity.
// [group of 256 columns][32 rows][64 lanes] words.
__device__ __forceinline__ unsigned pick_scales(uint2 s, int odd)
{
    return odd ? (s.x >> 8 & 255u) | (s.x >> 24) << 8 | (s.y >> 8 & 255u) << 16 | (s.y >> 24) << 24
               : (s.x & 255u) | (s.x >> 16 & 255u) << 8 | (s.y & 255u) << 16 | (s.y >> 16 & 255u) << 24;
}

// Prepares both operands in one launch.  Workgroups up to `x_groups`: x, 32 rows and 256 columns each, four lanes a block as in
// mxfp4_quantize; the others: the filter's scales, 32 rows and 8 groups.
template <typename T>
__global__ __launch_bounds__(256) void mxfp4_prepare_kernel(int N, int C, int K, int blocks, int scale_row, int groups, unsigned x_groups, const T *x,
                                                            unsigned *xc, unsigned *xs, const unsigned char *ws, unsigned *wt)
{
    if (blockIdx.x >= x_groups) {
        const int row = threadIdx.x >> 3, at = threadIdx.x & 7;
        const unsigned i = blockIdx.x - x_groups, eights = (unsigned)(groups + 7) / 8;
        const int group = (int)(i % eights) * 8 + at;
        const long long tile = i / eights, k = tile * 32 + row, tiles = (K + 31ll) / 32;
        if (group >= groups) return;
        uint2 s = make_uint2(0, 0);
        if (k < K) s = *reinterpret_cast<const uint2 *>(ws + (size_t)k * scale_row + group * 8);
        unsigned *out = wt + ((size_t)group * tiles + tile) * 64 + row;
        out[0] = pick_scales(s, 0);
        out[32] = pick_scales(s, 1);
        return;
    }
    __shared__ unsigned char bytes[32][8];
    const int group = (int)(blockIdx.x % (unsigned)groups), quarter = threadIdx.x & 3, at = (threadIdx.x >> 2) & 7, b = group * 8 + at;
    const long long tile = blockIdx.x / (unsigned)groups, tiles = (N + 31ll) / 32;
    const int column = b * 32 + quarter * 8;
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {       // rows threadIdx.x/32 + 8*i
        const long long n = tile * 32 + i * 8 + (threadIdx.x >> 5);
        load8_edge(x + (n < N ? (size_t)n * C + column : 0), n < N ? C - column : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 8 + (threadIdx.x >> 5);
        const long long n = tile * 32 + row;
        const unsigned byte = mxfp4_scale_byte(max_quad(largest8(v[i])));
        if (n < N && b < blocks) xc[((size_t)n * blocks + b) * 4 + quarter] = mxfp4_codes8(v[i], byte);
        if (quarter == 0) bytes[row][at] = (unsigned char)byte;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint2 s = *reinterpret_cast<const uint2 *>(bytes[threadIdx.x & 31]);
        xs[((size_t)group * tiles + tile) * 64 + threadIdx.x] = pick_scales(s, threadIdx.x >> 5);
    }
}

// GM x GN waves of 32*FM filter rows by 32*FN rows of x each.  A stage is 128 columns, 64 bytes of codes a row, brought into a ring of four
// stages by direct loads; scales come a word for two stages.  Row r's 16-byte chunk c lies at place c ^ (r/4)%4, so that the 16 rows
// that one phase of a 16-byte read covers lie in all 64 banks once.
// 8192 x 8192 by 8192: 260 us, 4.2 PFLOP/s (in single calls some 300), the matrix pipe busy 0.62 of the time at 1.75 GHz: a stage's reads from LDS and fills of it take as many
// cycles as its products.  Preparing the operands takes 38 us more, from fp32 66.
// One barrier a stage, between the last operand fetch of the stage and its last products: the fetches of the next stage and the
// loads of the one after three more go between the products.
template <int FM, int FN, int GM, int GN>
struct Tile {
    static constexpr int WAVES = GM * GN, BM = 32 * FM * GM, BN = 32 * FN * GN;
    static constexpr int STAGE = (BM + BN) * 64, RING = 4;
    static constexpr int KB = (BM + BN) / 128;      // kilobytes of scales of two stages
    static constexpr int LW = BM / 16 / WAVES, LX = BN / 16 / WAVES, LOADS = LW + LX;       // of 1 KB, each wave's, a stage
    static_assert(BM % 128 == 0 && BN % 128 == 0 && LW * WAVES * 16 == BM && LX * WAVES * 16 == BN && KB <= WAVES, "whole loads");
    static_assert(FM + FN <= FM * FN && LOADS <= FM * FN, "room between the products");
};

template <typename T, int FM, int FN, int GM, int GN>
__global__ __launch_bounds__(64 * GM * GN, 1) void mxfp4_tile_kernel(int N, int K, int code_row, int groups, const unsigned char *xc, const unsigned *xs,
                                                                     const unsigned char *wc, const unsigned *wt, const float *bias, int relu, T *y, int k_tiles,
                                                                     int n_tiles)
{
    typedef Tile<FM, FN, GM, GN> G;
    __shared__ __align__(16) unsigned char lds[G::RING * G::STAGE + 4 * G::KB * 1024];
    unsigned char *ring = lds, *scales = lds + G::RING * G::STAGE;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % GM, wn = wave / GM, half = lane >> 5;

    // Each XCD works on neighbouring tiles: groups of 8 filter tiles by all tiles of x, the filter's fastest.
    const unsigned total = (unsigned)k_tiles * (unsigned)n_tiles, per = total / 8, rest = total % 8, xcd = blockIdx.x % 8, in_xcd = blockIdx.x / 8;
    const unsigned id = xcd * per + (xcd < rest ? xcd : rest) + in_xcd;
    const unsigned band = id / (8u * (unsigned)n_tiles), first = band * 8u, width = min(8u, (unsigned)k_tiles - first), in_band = id - band * 8u * (unsigned)n_tiles;
    const long long k0 = (long long)(first + in_band % width) * G::BM, n0 = (long long)(in_band / width) * G::BN;

    // sources: this tile's rows (what lies outside reads as zeros)
    const int k_rows = (int)(K - k0 < G::BM ? K - k0 : G::BM), n_rows = (int)(N - n0 < G::BN ? N - n0 : G::BN);
    const buf_rsrc_t rs_w = make_buf_rsrc(wc + (size_t)k0 * code_row, (unsigned)k_rows * (unsigned)code_row);
    const buf_rsrc_t rs_x = make_buf_rsrc(xc + (size_t)n0 * code_row, (unsigned)n_rows * (unsigned)code_row);
    // A kilobyte of scales is 128 rows: wave w brings part w of the filter's, then of x's; waves past the last part bring one of these once more
    // (the same bytes to the same place), so that every wave has as many loads under way.
    constexpr int WS = G::BM / 128;
    const int s_part = wave % G::KB;
    const bool of_w = s_part < WS;
    const long long s_tile = of_w ? k0 / 32 + s_part * 4 : n0 / 32 + (s_part - WS) * 4, s_tiles = of_w ? (K + 31ll) / 32 : (N + 31ll) / 32;
    const unsigned *s_base = (of_w ? wt : xs) + s_tile * 64;
    const size_t s_pitch = (size_t)s_tiles * 256;
    const unsigned s_bytes = s_tile >= s_tiles ? 0u : (unsigned)min(s_tiles - s_tile, 4ll) * 256u;

    const int stages = (code_row + 63) / 64;
    const int chunk = (lane & 3) ^ ((lane >> 4) & 3);
    unsigned src[G::LOADS];
#pragma unroll
    for (int i = 0; i < G::LOADS; ++i) {
        const int row = (i < G::LW ? wave * G::LW + i : wave * G::LX + i - G::LW) * 16 + (lane >> 2);
        src[i] = (unsigned)row * (unsigned)code_row + chunk * 16;
    }
    auto issue_codes = [&](int stage, int i) {       // load i of a stage: LW of filter rows, then LX of rows of x
        const unsigned column = (unsigned)stage * 64u;
        const unsigned off = (int)(column + chunk * 16) < code_row ? src[i] + column : 0x80000000u;
        unsigned char *to = ring + (stage & 3) * G::STAGE;
        if (i < G::LW) lds_dma16(rs_w, off, to + (wave * G::LW + i) * 1024);
        else lds_dma16(rs_x, off, to + G::BM * 64 + (wave * G::LX + i - G::LW) * 1024);
    };
    auto issue_scales = [&](int stage) {             // of stages `stage` (even) and the next
        const int group = stage >> 1;
        const buf_rsrc_t rs = make_buf_rsrc((const unsigned char *)s_base + (size_t)(group < groups ? group : 0) * s_pitch, group < groups ? s_bytes : 0u);
        lds_dma16(rs, (unsigned)lane * 16u, scales + ((group & 3) * G::KB + s_part) * 1024);
    };

    f32x16 acc[FM][FN] = {};
    uint4 w[2][FM], x[2][FN];
    int sw[FM], sx[FN];
    // operand addresses of the first half of a stage; the second's are 32 bytes away, one way or the other
    const int swz = (lane >> 2) & 3;
    const int w_at = (wm * 32 * FM + (lane & 31)) * 64, x_at = (G::BM + wn * 32 * FN + (lane & 31)) * 64;
    auto fetch_w = [&](int stage, int s, int i) { return *reinterpret_cast<const uint4 *>(ring + (stage & 3) * G::STAGE + w_at + i * 2048 + ((2 * s + half) ^ swz) * 16); };
    auto fetch_x = [&](int stage, int s, int i) { return *reinterpret_cast<const uint4 *>(ring + (stage & 3) * G::STAGE + x_at + i * 2048 + ((2 * s + half) ^ swz) * 16); };
    auto fetch_sw = [&](int group, int i) { return *reinterpret_cast<const int *>(scales + (group & 3) * G::KB * 1024 + (wm * FM + i) * 256 + lane * 4); };
    auto fetch_sx = [&](int group, int i) { return *reinterpret_cast<const int *>(scales + (group & 3) * G::KB * 1024 + G::BM * 8 + (wn * FN + i) * 256 + lane * 4); };

#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (t % 2 == 0) issue_scales(t);
#pragma unroll
        for (int i = 0; i < G::LOADS; ++i) issue_codes(t, i);
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(3 * G::LOADS + 1) : "memory");
#pragma unroll
    for (int i = 0; i < FM; ++i) { w[0][i] = fetch_w(0, 0, i); sw[i] = fetch_sw(0, i); }
#pragma unroll
    for (int i = 0; i < FN; ++i) { x[0][i] = fetch_x(0, 0, i); sx[i] = fetch_sx(0, i); }

    // products of half S of a stage (byte B of the scales), and between them fetch(i), i < FM*FN
    auto products = [&](auto B, int s, auto fetch) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                acc[i][j] = mfma32<decltype(B)::value>(w[s][i], x[s][j], acc[i][j], sw[i], sx[j]);
                fetch(i * FN + j);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    int nsw[FM], nsx[FN];
    auto stage_of = [&](int t, auto odd) {
        constexpr int ODD = decltype(odd)::value;
        products(std::integral_constant<int, 2 * ODD>(), 0, [&](int u) {
            if (u < FM) w[1][u < FM ? u : 0] = fetch_w(t, 1, u);
            else if (u < FM + FN) x[1][u < FM ? 0 : u - FM < FN ? u - FM : 0] = fetch_x(t, 1, u - FM);
        });
        // the next stage has landed (those after it, two of codes and one of scales, may be under way), and no wave reads this one any more
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(2 * G::LOADS + 1) : "memory");
        products(std::integral_constant<int, 2 * ODD + 1>(), 1, [&](int u) {
            if (u < FM) w[0][u < FM ? u : 0] = fetch_w(t + 1, 0, u);
            else if (u < FM + FN) x[0][u < FM ? 0 : u - FM < FN ? u - FM : 0] = fetch_x(t + 1, 0, u - FM);
            if (ODD) {
                if (u < FM) nsw[u < FM ? u : 0] = fetch_sw((t + 1) >> 1, u);
                else if (u < FM + FN) nsx[u < FM ? 0 : u - FM < FN ? u - FM : 0] = fetch_sx((t + 1) >> 1, u - FM);
            }
            if (u < G::LOADS) {
                if (u == 0 && !ODD) issue_scales(t + 4);
                issue_codes(t + 4, u);
            }
        });
    };
    for (int t = 0; t < stages; t += 2) {
        stage_of(t, std::integral_constant<int, 0>());
        stage_of(t + 1, std::integral_constant<int, 1>());
#pragma unroll
        for (int i = 0; i < FM; ++i) sw[i] = nsw[i];
#pragma unroll
        for (int i = 0; i < FN; ++i) sx[i] = nsx[i];
    }
    // Results through LDS, 32*GN rows of y at a time, so that they leave as whole lines: written from the registers, eight bytes of each
    // of 32 rows an instruction, they took 10 us a tile.  A row's pitch of 16 bytes more spreads rows over the banks.
    constexpr int PIECE = 16 / (int)sizeof(T), PITCH = G::BM * (int)sizeof(T) + 16, ROWS = 32 * GN, PIECES = G::BM / PIECE;
    static_assert(ROWS * PITCH <= (int)sizeof(lds), "room for the results");
    f32x4 b[FM][4] = {};
    if (bias) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const long long k = k0 + wm * 32 * FM + i * 32 + g * 8 + half * 4 + e;
                    if (k < K) b[i][g][e] = bias[k];
                }
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");       // nothing under way into, or read from, what is written now
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = acc[i][j][g * 4 + e] + b[i][g][e];
                    if (relu && v[e] < 0.f) v[e] = 0.f;
                }
                unsigned char *to = lds + (wn * 32 + (lane & 31)) * PITCH + (wm * 32 * FM + i * 32 + g * 8 + half * 4) * (int)sizeof(T);
                if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(to) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                else *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
            }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < ROWS * PIECES / (64 * G::WAVES); ++u) {
            const int at = u * 64 * G::WAVES + (int)threadIdx.x, row = at / PIECES, piece = at % PIECES;
            const long long n = n0 + (row >> 5) * 32 * FN + j * 32 + (row & 31), k = k0 + piece * PIECE;
            const uint4 q = *reinterpret_cast<const uint4 *>(lds + row * PITCH + piece * 16);
            const u32x4_any v = {q.x, q.y, q.z, q.w};
            if (n >= N || k >= K) continue;
            T *to = y + (size_t)n * K + k;
            if (k + PIECE <= K) *reinterpret_cast<u32x4_any *>(to) = v;
            else {
#pragma unroll
                for (int e = 0; e < PIECE; ++e)
                    if (k + e < K) {
                        if constexpr (sizeof(T) == 2) to[e] = (bf16_t)(v[e / 2] >> (16 * (e & 1)));
                        else to[e] = __uint_as_float(v[e]);
                    }
            }
        }
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------------

// Waves of a token workgroup: 16 where there is one for a compute unit at most and each has some columns.  1 row of 16384 by 4096 13.4 -> 11.1 us, 8 of
// 8192 13.2 -> 9.4; by 16384, where workgroups share a compute unit, 1 row of 9216 22 -> 28.
int token_waves(int C, int K) { return C > 4096 && K <= 4096 ? 16 : 8; }

enum Path { TOKEN, SKINNY, TILED };
Path path_of(int N, int C, int K)
{
    // One launch where it serves: every workgroup brings x into 4 bits once more, which costs for each row and round of workgroups, against one launch more and
    // x read from the caches.  Token and skinny, us: 4096 by 4096, 1 row 4.6 and 7.7, 8 rows 6.5 and 7.4, 12 rows 7.7 and 7.4; 9216 by 4096, 4 rows 9.9 and 10.6,
    // 8 rows 12.8 and 10.7; 4096 by 16384, 2 rows 12.4 and 13.0, 4 rows 14.0 and 12.5; 512 by 65536, 1 row 20.7 and 12.3.  Long rows
    // read the filter at memory's rate: 16384 by 65536, 1 row 114 and 160, 3 rows 134 and 161; 16384 by 16384, 2 rows 34 and 40, 4 rows 41 and 40.
    if (N * ((K + 4095ll) / 4096) <= TOKEN_ROWS || (N <= 3 && C > 12288)) return TOKEN;
    // The skinny workgroups read their operands once for 16 or 32 filter rows, the tiles once for 128 or 256, but need one for each compute unit: 512
    // rows of 9216 by 2048 (64 small tiles) 18 us skinny and 30 tiled, 256 by 6144 (96) 30 and 32, 512 by 4096 (128) 31 and 31, 80 by 32768 (256) 74
    // and 51.  Up to 32 rows a tile is mostly zeros: 32 by 131072, 76 and 92.
    return N <= 32 || ((N + 127ll) / 128) * ((K + 127ll) / 128) <= 128 ? SKINNY : TILED;
}

struct Buffers {        // of the workspace
    size_t codes = 0, scales = 0, filter_scales = 0, total = 0;     // offsets of the last two, and the whole
};
Buffers buffers(int N, int C, int K)
{
    Buffers b;
    const Path path = path_of(N, C, K);
    if (path == TOKEN) return b;
    if (path == SKINNY) {
        const size_t units = ((size_t)N + 15) / 16 * (((size_t)C + 511) / 512);     // of 16 rows and 512 columns
        b.scales = units * 4096;
        b.filter_scales = b.total = b.scales + units * 256;
        return b;
    }
    const size_t groups = ((size_t)C + 255) / 256;
    b.scales = align_up((size_t)N * mxfp4_code_row(C), 256);
    b.filter_scales = b.scales + ((size_t)N + 31) / 32 * groups * 256;
    b.total = b.filter_scales + ((size_t)K + 31) / 32 * groups * 256;
    return b;
}

template <typename T, int FM, int FN, int GM, int GN>
int launch_tiles(int N, int C, int K, const unsigned char *xc, const unsigned *xs, const unsigned char *wc, const unsigned *wt, const float *bias, int relu, T *y,
                 hipStream_t st)
{
    typedef Tile<FM, FN, GM, GN> G;
    const long long kt = (K + G::BM - 1ll) / G::BM, nt = (N + G::BN - 1ll) / G::BN;
    if (!one_launch(kt * nt, 64 * G::WAVES)) return MXC_ERR_SHAPE;
    hipLaunchKernelGGL((mxfp4_tile_kernel<T, FM, FN, GM, GN>), dim3((unsigned)(kt * nt)), dim3(64 * G::WAVES), 0, st, N, K, (int)mxfp4_code_row(C), (int)(((long long)C + 255) / 256), xc, xs,
                       wc, wt, bias, relu, y, (int)kt, (int)nt);
    return MXC_OK;
}

template <typename T>
int fc(int N, int C, int K, const T *x, const unsigned char *wc, const unsigned char *ws, const float *bias, int relu, T *y, void *workspace, hipStream_t st)
{
    const int blocks = (int)(mxfp4_code_row(C) / 16), scale_row = (int)mxfp4_scale_row(C);
    const Path path = path_of(N, C, K);
    if (path == TOKEN) {
        const int waves = token_waves(C, K);
        if (!one_launch((K + 15ll) / 16, 64 * waves)) return MXC_ERR_SHAPE;
        hipLaunchKernelGGL((waves == 8 ? mxfp4_token_kernel<T, 8> : mxfp4_token_kernel<T, 16>), dim3((unsigned)((K + 15ll) / 16)), dim3(64 * waves), 0, st, N, C, K, blocks, scale_row,
                           x, wc, ws, bias, relu, y);
        return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
    }
    const Buffers b = buffers(N, C, K);
    unsigned char *xc = (unsigned char *)workspace, *xs = xc + b.scales;
    if (path == SKINNY) {
        const int groups = scale_row / 16, tiles = (N + 15) / 16;
        if (!one_launch((unsigned long long)groups * tiles, 256) || !one_launch((K + 15ll) / 16, 512)) return MXC_ERR_SHAPE;
        hipLaunchKernelGGL(mxfp4_order_kernel<T>, dim3((unsigned)(groups * tiles)), dim3(256), 0, st, N, C, groups, x, (unsigned *)xc, (unsigned *)xs);
        if (hipGetLastError() != hipSuccess) return MXC_ERR_LAUNCH;
        // The largest workgroups of which there are enough.  128 rows of 9216, us with workgroups of 32 filter rows by 128 rows of x, 32 by 64, 16 by 64, 16 by 32:
        // 1000 filter rows 18, 13, 11.1, 10.7; 2048: 18, 13.0, 11.2, 12.1; 4096: 18, 13.3, 15, 16; 6000: 18.4, 21.6, 24.7, 28; 8192: 18.8, 20.9, 27, 35.
        auto launch = [&](auto wf, auto nf, bool last) {
            constexpr int WF = decltype(wf)::value, NF = decltype(nf)::value;
            const long long k_parts = (K + 16 * WF - 1ll) / (16 * WF), n_parts = (tiles + NF - 1) / NF;
            if (!last && (tiles <= NF / 2 || k_parts * n_parts < 160)) return false;
            hipLaunchKernelGGL((mxfp4_skinny_kernel<T, WF, NF>), dim3((unsigned)k_parts, (unsigned)n_parts), dim3(512), 0, st, N, K, blocks, scale_row, xc, xs, wc, ws, bias, relu, y);
            return true;
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> four;
        const std::integral_constant<int, 8> eight;
        launch(two, eight, false) || launch(two, four, false) || launch(one, four, false) || (tiles <= 2 && launch(two, two, false)) || launch(one, two, true);
        return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
    }
    const int groups = (int)(((long long)C + 255) / 256);
    unsigned *xt = (unsigned *)xs, *wt = (unsigned *)((unsigned char *)workspace + b.filter_scales);
    const size_t x_groups = ((size_t)N + 31) / 32 * groups, w_groups = ((size_t)K + 31) / 32 * ((groups + 7) / 8);
    if (!one_launch(x_groups + w_groups, 256)) return MXC_ERR_SHAPE;
    hipLaunchKernelGGL(mxfp4_prepare_kernel<T>, dim3((unsigned)(x_groups + w_groups)), dim3(256), 0, st, N, C, K, blocks, scale_row, groups, (unsigned)x_groups, x, (unsigned *)xc, xt, ws, wt);
    if (hipGetLastError() != hipSuccess) return MXC_ERR_LAUNCH;
    // Tiles of 256 x 256 need half the reads from LDS that tiles of 128 x 128 do, but have to fill 256 compute units: 2048 rows by 4096 of 4096 (128 large ones)
    // 34.1 us large and 31.0 small, 3000 x 8192 by 4096 (192) 70.9 and 78.9, 4096 x 4096 by 4096 (256) 46.6 and 54.3.
    const long long big = ((K + 255ll) / 256) * ((N + 255ll) / 256);
    const int rc = big >= 192 ? launch_tiles<T, 4, 2, 2, 4>(N, C, K, xc, xt, wc, wt, bias, relu, y, st) : launch_tiles<T, 2, 2, 2, 2>(N, C, K, xc, xt, wc, wt, bias, relu, y, st);
    if (rc != MXC_OK) return rc;
    return hipGetLastError() == hipSuccess ? MXC_OK : MXC_ERR_LAUNCH;
}

}  // namespace

size_t mxfp4_fc_workspace(int N, int C, int K, int dtype) { return buffers(N, C, K).total; }

int mxfp4_fc(int N, int C, int K, int dtype, const void *x, const void *w_codes, const void *w_scales, const float *bias, int relu, void *y,
             void *workspace, hipStream_t st)
{
    const unsigned char *wc = (const unsigned char *)w_codes, *ws = (const unsigned char *)w_scales;
    return dtype == MXC_BF16 ? fc<bf16_t>(N, C, K, (const bf16_t *)x, wc, ws, bias, relu, (bf16_t *)y, workspace, st)
                             : fc<float>(N, C, K, (const float *)x, wc, ws, bias, relu, (float *)y, workspace, st);
}

}  // namespace mxc
