// Rows in pieces of 16 bytes that begin wherever the row does: the memory pipeline takes 16-byte accesses at any element's address, so
// that rows of odd lengths move as fast as others (16383 x 4097 bf16 in place of x 4096: see layernorm.hip).  A row's last piece may be short.
#pragma once
#include "mxc_internal.h"

namespace mxc {

typedef unsigned Bytes16 __attribute__((ext_vector_type(4), aligned(2)));       // 16 bytes at any element

// Keeps a value where it is in registers: what is made of it before is not kept for after, in more of them.
__device__ __forceinline__ void held(uint4 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }

// x rounded to 32 bits: the compiler does not join what made it with what it goes into.
__device__ __forceinline__ float in_32_bits(float x)
{
    asm("" : "+v"(x));
    return x;
}

template <class T> struct Piece;
template <> struct Piece<float> {
    static constexpr int VE = 4;
    uint4 raw;
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w); }
    __device__ __forceinline__ void set(const float *v) { raw = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])); }
    static __device__ __forceinline__ float rounded(float v) { return v; }
};
template <> struct Piece<bf16_t> {
    static constexpr int VE = 8;
    uint4 raw;
    __device__ __forceinline__ float get(int i) const
    {
        const unsigned w = i < 2 ? raw.x : i < 4 ? raw.y : i < 6 ? raw.z : raw.w;
        return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
    }
    __device__ __forceinline__ void set(const float *v)
    {
        raw = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
    static __device__ __forceinline__ bf16_t rounded(float v) { return (bf16_t)pack_bf16x2(v, 0.f); }
};

// four bf16: where a lane's results are 32 bits, so that 16 bytes of them follow each other
struct Quad {
    static constexpr int VE = 4;
    uint2 raw;
    __device__ __forceinline__ float get(int i) const
    {
        const unsigned w = i < 2 ? raw.x : raw.y;
        return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
    }
};
// Elements [at, at + VE) of a row of `len`, zeros past its end, in two steps, so that loads stay under way: the load, which for a piece that the row ends in brings the
// row's last VE elements (of rows of fewer, one by one), and settle_piece, which moves these down.  (Loads in the branch of a short piece would wait there
// for all before them: a gradient of 40000 x 1000 bf16, 125 pieces by 128 lanes, took 100 us where 65536 x 512 took 51.)
template <bool PAST = false, class T>
__device__ __forceinline__ Piece<T> begin_piece(const T *row, int at, int len)
{
    constexpr int VE = Piece<T>::VE;
    Piece<T> p;
    if (len >= VE) {
        const Bytes16 *from = reinterpret_cast<const Bytes16 *>(row + (at + VE <= len ? at : len - VE));
        const Bytes16 b = PAST ? __builtin_nontemporal_load(from) : *from;
        p.raw = make_uint4(b.x, b.y, b.z, b.w);
    } else {
        float v[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = at + i < len ? load_f32(row + at + i) : 0.f;
        p.set(v);
    }
    return p;
}
template <class T>
__device__ __forceinline__ void settle_piece(Piece<T> &p, int at, int len)
{
    constexpr int VE = Piece<T>::VE;
    if (at + VE > len && len >= VE) {
        const int bits = (at + VE - len) * (int)sizeof(T) * 8;
        unsigned long long lo = p.raw.x | (unsigned long long)p.raw.y << 32, hi = p.raw.z | (unsigned long long)p.raw.w << 32;
        if (bits >= 64) {
            lo = bits >= 128 ? 0 : hi >> (bits - 64);
            hi = 0;
        } else {
            lo = lo >> bits | hi << (64 - bits);
            hi >>= bits;
        }
        p.raw = make_uint4((unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32));
    }
}
template <class T>
__device__ __forceinline__ Piece<T> load_piece(const T *row, int at, int len)
{
    Piece<T> p = begin_piece(row, at, len);
    settle_piece(p, at, len);
    return p;
}
// the same for four values: a Quad of bf16, a Piece of fp32
__device__ __forceinline__ Quad begin_quad(const bf16_t *row, int at, int len)
{
    typedef unsigned Bytes8 __attribute__((ext_vector_type(2), aligned(2)));
    Quad q;
    if (len >= 4) {
        const Bytes8 b = *reinterpret_cast<const Bytes8 *>(row + (at + 4 <= len ? at : len - 4));
        q.raw = make_uint2(b.x, b.y);
    } else {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = at + i < len ? row[at + i] : 0;
        q.raw = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
    return q;
}
__device__ __forceinline__ void settle_quad(Quad &q, int at, int len)
{
    if (at + 4 > len && len >= 4) {
        const int bits = (at + 4 - len) * 16;
        const unsigned long long v = q.raw.x | (unsigned long long)q.raw.y << 32, down = bits >= 64 ? 0 : v >> bits;
        q.raw = make_uint2((unsigned)down, (unsigned)(down >> 32));
    }
}
__device__ __forceinline__ Piece<float> begin_quad(const float *row, int at, int len) { return begin_piece(row, at, len); }
__device__ __forceinline__ void settle_quad(Piece<float> &p, int at, int len) { settle_piece(p, at, len); }
template <bool PAST = false, class T>
__device__ __forceinline__ void store_piece(T *row, int at, int len, const Piece<T> &p)
{
    if (at + Piece<T>::VE <= len) {
        const Bytes16 b = {p.raw.x, p.raw.y, p.raw.z, p.raw.w};
        if (PAST) __builtin_nontemporal_store(b, reinterpret_cast<Bytes16 *>(row + at));
        else *reinterpret_cast<Bytes16 *>(row + at) = b;
    } else {
#pragma unroll
        for (int i = 0; i < Piece<T>::VE; ++i)
            if (at + i < len) row[at + i] = Piece<T>::rounded(p.get(i));
    }
}

// four values rounded to bf16
__device__ __forceinline__ void store_quad(bf16_t *row, int at, int len, const float (&v)[4])
{
    typedef unsigned Bytes8 __attribute__((ext_vector_type(2), aligned(2)));
    if (at + 4 <= len) {
        *reinterpret_cast<Bytes8 *>(row + at) = Bytes8{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (at + i < len) row[at + i] = Piece<bf16_t>::rounded(v[i]);
    }
}

// Sum over aligned groups of G lanes (a power of two), the same in each of them.  Exchanges within 16 lanes are part of an instruction; the four sixteens of a wave
// meet as scalars.
template <int CONTROL>
__device__ __forceinline__ float lane_exchanged(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CONTROL, 0xF, 0xF, true)); }
template <int G>
__device__ __forceinline__ float lane_sum(float x)
{
    if constexpr (G >= 2) x += lane_exchanged<0xB1>(x);        // lanes 1 0 3 2
    if constexpr (G >= 4) x += lane_exchanged<0x4E>(x);        // lanes 2 3 0 1
    if constexpr (G >= 8) x += lane_exchanged<0x141>(x);       // the other half of eight
    if constexpr (G >= 16) x += lane_exchanged<0x140>(x);      // the other half of sixteen
    if constexpr (G == 32) x += __shfl_xor(x, 16);
    if constexpr (G == 64) {
        auto of = [&](int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane)); };
        x = (of(0) + of(16)) + (of(32) + of(48));
    }
    return x;
}

}  // namespace mxc
