// Eight neighbouring elements of a tensor ("octet"): the piece a thread of the recurrence and of dropout works on (internal).
// An octet starts at a multiple of eight elements of the whole tensor, so that it can be loaded whole whatever the row length;
// rows that start or end inside one mask the elements that are not theirs.
#pragma once
#include "common.cuh"

namespace hn {

__device__ __forceinline__ void unpack2(unsigned w, float &a, float &b) { a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ unsigned pack2(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned *>(&h);
}

template <typename T> struct Octet;
template <> struct Octet<bf16> {
    uint4 w;
    // elements [i, i + 8) of the n at p; those from n on are zero
    __device__ __forceinline__ void ld(const bf16 *p, long long i, long long n)
    {
        if (i + 8 <= n) {
            HN_G(p + i, 16);
            w = __ldg(reinterpret_cast<const uint4 *>(p + i));
        } else {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = i + e < n ? IO<bf16>::ld(p, i + e) : 0.f;
            w = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
        }
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        unpack2(w.x, f[0], f[1]); unpack2(w.y, f[2], f[3]); unpack2(w.z, f[4], f[5]); unpack2(w.w, f[6], f[7]);
    }
};
template <> struct Octet<float> {
    float4 a, b;
    __device__ __forceinline__ void ld(const float *p, long long i, long long n)
    {
        if (i + 8 <= n) {
            HN_G(p + i, 32);
            a = __ldg(reinterpret_cast<const float4 *>(p + i));
            b = __ldg(reinterpret_cast<const float4 *>(p + i + 4));
        } else {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = i + e < n ? IO<float>::ld(p, i + e) : 0.f;
            a = make_float4(f[0], f[1], f[2], f[3]);
            b = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
};

// elements [lo, hi) of the octet at element i
template <typename T> __device__ __forceinline__ void st_octet(T *p, long long i, int lo, int hi, const float (&f)[8])
{
    if (lo <= 0 && hi >= 8) {
        HN_G(p + i, 8 * sizeof(T));
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(p + i) = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
        } else {
            *reinterpret_cast<float4 *>(p + i) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4 *>(p + i + 4) = make_float4(f[4], f[5], f[6], f[7]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= lo && e < hi) IO<T>::st(p, i + e, f[e]);
    }
}

}  // namespace hn
