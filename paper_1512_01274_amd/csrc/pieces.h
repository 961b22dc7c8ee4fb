// Rows in pieces of 16 bytes that begin wherever the row does: the memory pipeline takes 16-byte accesses at any element's address, so
// that rows of odd lengths move as fast as others (16383 x 4097 bf16 in place of x 4096: see layernorm.hip).  A row's last piece may be short.
#pragma once
#include "mxc_internal.h"

namespace mxc {

struct __attribute__((packed, aligned(2))) Bytes16 { unsigned x, y, z, w; };

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

// elements [at, at + VE) of a row of `len`: zeros past its end
template <class T>
__device__ __forceinline__ Piece<T> load_piece(const T *row, int at, int len)
{
    Piece<T> p;
    if (at + Piece<T>::VE <= len) {
        const Bytes16 b = *reinterpret_cast<const Bytes16 *>(row + at);
        p.raw = make_uint4(b.x, b.y, b.z, b.w);
    } else {
        float v[Piece<T>::VE];
#pragma unroll
        for (int i = 0; i < Piece<T>::VE; ++i) v[i] = at + i < len ? load_f32(row + at + i) : 0.f;
        p.set(v);
    }
    return p;
}
template <class T>
__device__ __forceinline__ void store_piece(T *row, int at, int len, const Piece<T> &p)
{
    if (at + Piece<T>::VE <= len) {
        *reinterpret_cast<Bytes16 *>(row + at) = Bytes16{p.raw.x, p.raw.y, p.raw.z, p.raw.w};
    } else {
#pragma unroll
        for (int i = 0; i < Piece<T>::VE; ++i)
            if (at + i < len) row[at + i] = Piece<T>::rounded(p.get(i));
    }
}

}  // namespace mxc
