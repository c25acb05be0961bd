// What the kernels that quantize rows of activations share: loads of eight elements and their exact widening, the maximum over a
// workgroup, rounding to int8 codes.  Every floating-point step is one binary32 operation of the definition: the files that
// include this are compiled without contraction.
#pragma once
#include "w4a8_common.hpp"

namespace w4a8 {

constexpr float AQ_FLT_MAX = 3.402823466e+38f;   // a token whose 127 / max|t| is not finite counts as all-zero

constexpr int AQ_VEC = 8;

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]);

template <>
__device__ __forceinline__ void load8<float>(const float *p, float (&v)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p);
    const float4 b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<__half>(const __half *p, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __half2float(__ushort_as_half((uint16_t)(w[i] & 0xffffu)));
        v[2 * i + 1] = __half2float(__ushort_as_half((uint16_t)(w[i] >> 16)));
    }
}
template <>
__device__ __forceinline__ void load8<bf16_t>(const bf16_t *p, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// maximum over a workgroup of WAVES waves; red: WAVES floats
template <int WAVES>
__device__ __forceinline__ float block_max(float v, float *red)
{
    v = wave_max(v);
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // `red` may still be read by the previous row
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = fmaxf(v, red[w]);
    return v;
}

// Eight consecutive elements of a row as they come from memory (16 bytes of a 16-bit type, 32 of
// binary32), and their exact widening.
template <typename T> struct Raw8 { uint4 v; };
template <> struct Raw8<float> { float4 a, b; };

template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T *p)
{
    Raw8<T> r;
    // (streaming loads: the unquantized activations are read exactly once)
    const v4u t = __builtin_nontemporal_load(reinterpret_cast<const v4u *>(p));
    r.v = make_uint4(t.x, t.y, t.z, t.w);
    return r;
}
template <>
__device__ __forceinline__ Raw8<float> load_raw8<float>(const float *p)
{
    Raw8<float> r;
    const v4f a = __builtin_nontemporal_load(reinterpret_cast<const v4f *>(p));
    const v4f b = __builtin_nontemporal_load(reinterpret_cast<const v4f *>(p + 4));
    r.a = make_float4(a.x, a.y, a.z, a.w);
    r.b = make_float4(b.x, b.y, b.z, b.w);
    return r;
}
__device__ __forceinline__ void widen8(const Raw8<float> &r, float (&v)[8])
{
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
    v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
__device__ __forceinline__ void widen8(const Raw8<__half> &r, float (&v)[8])
{
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __half2float(__ushort_as_half((uint16_t)(w[i] & 0xffffu)));
        v[2 * i + 1] = __half2float(__ushort_as_half((uint16_t)(w[i] >> 16)));
    }
}
__device__ __forceinline__ void widen8(const Raw8<bf16_t> &r, float (&v)[8])
{
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// Four rounded codes (the low bytes of q0..q3) packed into one word.
__device__ __forceinline__ uint32_t pack4_low_bytes(uint32_t q0, uint32_t q1, uint32_t q2, uint32_t q3)
{
    const uint32_t lo = __builtin_amdgcn_perm(q1, q0, 0x0c0c0400u);   // [q0.b0, q1.b0, 0, 0]
    const uint32_t hi = __builtin_amdgcn_perm(q3, q2, 0x04000c0cu);   // [0, 0, q2.b0, q3.b0]
    return lo | hi;
}

// Symmetric form, rne and the conversion to an integer in one binary32 addition: y + 1.5 * 2^23 is
// 1.5 * 2^23 + rne(y) exactly for |y| <= 2^22 (the sum is rounded to nearest even at unit
// granularity), so the low byte of its bit pattern is rne(y) in two's complement.  The clamp to
// +-127 of the definition never changes a value: |t| <= a and inv = fl(127 / a) give
// |fl(t * inv)| <= 127 (1 + 2^-23), which rounds to 127.  (No contraction in this file: the product
// is rounded before the addition, as in the definition.)
__device__ __forceinline__ uint32_t quant1_bits(float t, float inv)
{
    return __float_as_uint(t * inv + 12582912.0f);
}

}  // namespace w4a8
