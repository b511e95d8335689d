// Element types of the operators around the expert layer (FP32, BF16, FP16):
// eight elements at a time to and from FP32 registers.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "pmpe_internal.cuh"

namespace pmpe {

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<bf16>(bf16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void unpack8(const uint4 &u, float (&v)[8], bf16)
{
    const __nv_bfloat162 *b = reinterpret_cast<const __nv_bfloat162 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __bfloat1622float2(b[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void unpack8(const uint4 &u, float (&v)[8], __half)
{
    const __half2 *b = reinterpret_cast<const __half2 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(b[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8], bf16)
{
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8], __half)
{
    uint4 u;
    __half2 *b = reinterpret_cast<__half2 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
    return u;
}

// Eight elements of a row in a thread.  kVec: consecutive ones at p, which is
// aligned to their 16 or 32 bytes; n > 0: they exist (rows hold whole chunks).
// Otherwise p, p + 32, ..., so that a warp's accesses are contiguous one
// element at a time; n: elements from p to the row's end.  What does not exist
// reads as zero.
template <typename T> struct Raw8 { uint4 u; };
template <> struct Raw8<float> { uint4 u, hi; };

template <bool kVec> __device__ __forceinline__ void load8(Raw8<float> &r, const float *p, int n)
{
    if (kVec) {
        r.u = r.hi = make_uint4(0u, 0u, 0u, 0u);
        // one access of 32 bytes: two of 16, each touching every other half
        // sector, took the norm's backward from 17.5 us to 26.9 with FP32 rows
        // in the place of BF16 ones
        if (n > 0)
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(r.u.x), "=r"(r.u.y), "=r"(r.u.z), "=r"(r.u.w), "=r"(r.hi.x), "=r"(r.hi.y), "=r"(r.hi.z), "=r"(r.hi.w)
                         : "l"(p) : "memory");
    } else {
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = 32 * i < n ? __float_as_uint(p[32 * i]) : 0u;
        r.u = make_uint4(q[0], q[1], q[2], q[3]);
        r.hi = make_uint4(q[4], q[5], q[6], q[7]);
    }
}
template <bool kVec, typename T> __device__ __forceinline__ void load8(Raw8<T> &r, const T *p, int n)
{
    if (kVec) {
        r.u = make_uint4(0u, 0u, 0u, 0u);
        if (n > 0) r.u = *reinterpret_cast<const uint4 *>(p);
    } else {
        uint32_t q[8];
        const uint16_t *s = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = 32 * i < n ? s[32 * i] : 0u;
        r.u = make_uint4(q[0] | q[1] << 16, q[2] | q[3] << 16, q[4] | q[5] << 16, q[6] | q[7] << 16);
    }
}
__device__ __forceinline__ void unpack(const Raw8<float> &r, float (&v)[8])
{
    v[0] = __uint_as_float(r.u.x); v[1] = __uint_as_float(r.u.y); v[2] = __uint_as_float(r.u.z); v[3] = __uint_as_float(r.u.w);
    v[4] = __uint_as_float(r.hi.x); v[5] = __uint_as_float(r.hi.y); v[6] = __uint_as_float(r.hi.z); v[7] = __uint_as_float(r.hi.w);
}
template <typename T> __device__ __forceinline__ void unpack(const Raw8<T> &r, float (&v)[8]) { unpack8(r.u, v, T()); }

// Rounded to nearest, ties to even.
template <bool kVec> __device__ __forceinline__ void store8(float *p, const float (&v)[8], int n)
{
    if (kVec) {
        if (n > 0)
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                         "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                         : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (32 * i < n) p[32 * i] = v[i];
    }
}
template <bool kVec, typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8], int n)
{
    if (kVec) {
        if (n > 0) *reinterpret_cast<uint4 *>(p) = pack8(v, T());
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (32 * i < n) p[32 * i] = from_f32<T>(v[i]);
    }
}

// Sums rounded once to the type: two 16-bit elements an instruction.
__device__ __forceinline__ void add8(Raw8<float> &r, const Raw8<float> &q)
{
    float a[8], b[8];
    unpack(r, a);
    unpack(q, b);
    r.u = make_uint4(__float_as_uint(a[0] + b[0]), __float_as_uint(a[1] + b[1]), __float_as_uint(a[2] + b[2]), __float_as_uint(a[3] + b[3]));
    r.hi = make_uint4(__float_as_uint(a[4] + b[4]), __float_as_uint(a[5] + b[5]), __float_as_uint(a[6] + b[6]), __float_as_uint(a[7] + b[7]));
}
__device__ __forceinline__ void add8(Raw8<bf16> &r, const Raw8<bf16> &q)
{
    __nv_bfloat162 *a = reinterpret_cast<__nv_bfloat162 *>(&r.u);
    const __nv_bfloat162 *b = reinterpret_cast<const __nv_bfloat162 *>(&q.u);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __hadd2_rn(a[i], b[i]);
}
__device__ __forceinline__ void add8(Raw8<__half> &r, const Raw8<__half> &q)
{
    __half2 *a = reinterpret_cast<__half2 *>(&r.u);
    const __half2 *b = reinterpret_cast<const __half2 *>(&q.u);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = __hadd2_rn(a[i], b[i]);
}

// The words as they are.
template <bool kVec> __device__ __forceinline__ void store_raw(float *p, const Raw8<float> &r, int n)
{
    float v[8];
    unpack(r, v);
    store8<kVec>(p, v, n);
}
template <bool kVec, typename T> __device__ __forceinline__ void store_raw(T *p, const Raw8<T> &r, int n)
{
    if (kVec) {
        if (n > 0) *reinterpret_cast<uint4 *>(p) = r.u;
    } else {
        const uint32_t q[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
        uint16_t *s = reinterpret_cast<uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (32 * i < n) s[32 * i] = (uint16_t)(q[i >> 1] >> 16 * (i & 1));
    }
}

// Aligned for eight elements at a time.
inline bool aligned8(const void *q, bool f32) { return ((uintptr_t)q & (f32 ? 31u : 15u)) == 0; }

template <typename V> __device__ __forceinline__ V warp_sum(V v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(~0u, v, off);
    return v;
}

// The larger of two values; NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// The same of two magnitudes; the sign is that of the product.
__device__ __forceinline__ float max_magnitude(float a, float b)
{
    float r;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Eight bits: e4m3 with a scale.
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126: the smallest scale, so that its reciprocal is finite

// A factor in two words: v times 448 / amax with one rounding in all, so that
// a value goes to the e4m3 neighbour of the exact quotient but within 2^-24 of
// the middle between two.
struct Divide {
    float hi, lo;
};
// For values u of a block whose largest is amax in magnitude and which stand
// for u m: the scale s = max(amax m / 448, 2^-126) and the factor u -> u m / s.
__device__ __forceinline__ Divide divide_by(float amax, float m, float &s)
{
    amax = fabsf(amax);
    s = max_nan(amax * m * (1.f / 448.f), kMinScale);
    if (!(s > kMinScale)) return {m * 0x1p126f, 0.f};  // zeros (or NaN)
    // the product's remainder is exact in one fused operation
    const float inv = __frcp_rn(amax), hi = 448.f * inv;
    return {hi, hi > 0.f ? fmaf(-hi, amax, 448.f) * inv : 0.f};
}
__device__ __forceinline__ uint32_t e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
// Four e4m3 as two pairs of FP16.
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t four, uint32_t &low, uint32_t &high)
{
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(low), "=r"(high) : "r"(four));
}

}  // namespace pmpe
