// Device helpers of the kernels that go over rows of features or logits: vectors of elements whose rows start where they
// start, sums over lanes.
#pragma once

#include "common.hpp"
#include "mfma_util.hpp"

namespace swimba {

// 16 and 8 bytes at an address that is a multiple of the element size only (rows of an odd width): global memory is read and
// written in one piece all the same.
typedef uint32_t __attribute__((ext_vector_type(4), aligned(2))) any_u32x4_t;
typedef uint32_t __attribute__((ext_vector_type(2), aligned(2))) any_u32x2_t;

// eight consecutive elements from and to memory, as floats
__device__ __forceinline__ void load8(float (&f)[8], const bf16 *p)
{
    const any_u32x4_t v = *reinterpret_cast<const any_u32x4_t *>(p);
    unpack8(f, make_uint4(v.x, v.y, v.z, v.w));
}
__device__ __forceinline__ void load8(float (&f)[8], const float *p)
{
    const any_u32x4_t a = *reinterpret_cast<const any_u32x4_t *>(p), b = *reinterpret_cast<const any_u32x4_t *>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = __uint_as_float(a[i]); f[4 + i] = __uint_as_float(b[i]); }
}
__device__ __forceinline__ void store8(bf16 *p, const float (&f)[8])
{
    const uint4 v = pack8(f);
    *reinterpret_cast<any_u32x4_t *>(p) = any_u32x4_t{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8])
{
    any_u32x4_t a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = __float_as_uint(f[i]); b[i] = __float_as_uint(f[4 + i]); }
    *reinterpret_cast<any_u32x4_t *>(p) = a;
    *reinterpret_cast<any_u32x4_t *>(p + 4) = b;
}
// the first n of them (n <= 0: none), the others as `rest` / left alone
template <typename T> __device__ __forceinline__ void load8(float (&f)[8], const T *p, int n, float rest)
{
    if (n >= 8) return load8(f, p);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? to_float(p[i]) : rest;
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&f)[8], int n)
{
    if (n >= 8) return store8(p, f);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = from_float<T>(f[i]);
}

// sum over the 64 lanes, in every lane
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

}  // namespace swimba
