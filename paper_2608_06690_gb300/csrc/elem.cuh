// Element types of the operators around the expert layer (FP32, BF16, FP16):
// eight elements at a time to and from FP32 registers.
#pragma once

#include <cuda_fp16.h>

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

// Eight consecutive elements at p, as loaded: the loads of several operands
// are issued before the first is unpacked.
template <typename T> struct Raw8 { uint4 u; };
template <> struct Raw8<float> { float4 lo, hi; };

// kVec: p is aligned for 16-byte accesses; otherwise element by element.
// n: how many of the eight exist (the others read as zeros).
template <bool kVec> __device__ __forceinline__ void load8(Raw8<float> &r, const float *p, int n)
{
    if (kVec) {
        r.lo = r.hi = make_float4(0.f, 0.f, 0.f, 0.f);
        if (n > 0) {
            r.lo = reinterpret_cast<const float4 *>(p)[0];
            r.hi = reinterpret_cast<const float4 *>(p)[1];
        }
    } else {
        r.lo = make_float4(n > 0 ? p[0] : 0.f, n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, n > 3 ? p[3] : 0.f);
        r.hi = make_float4(n > 4 ? p[4] : 0.f, n > 5 ? p[5] : 0.f, n > 6 ? p[6] : 0.f, n > 7 ? p[7] : 0.f);
    }
}
template <bool kVec, typename T> __device__ __forceinline__ void load8(Raw8<T> &r, const T *p, int n)
{
    if (kVec) {
        r.u = make_uint4(0u, 0u, 0u, 0u);
        if (n > 0) r.u = *reinterpret_cast<const uint4 *>(p);
    } else {
        uint32_t q[4];
        const uint16_t *s = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            q[i] = (n > 2 * i ? s[2 * i] : 0u) | (uint32_t)(n > 2 * i + 1 ? s[2 * i + 1] : 0u) << 16;
        r.u = make_uint4(q[0], q[1], q[2], q[3]);
    }
}
__device__ __forceinline__ void unpack(const Raw8<float> &r, float (&v)[8])
{
    v[0] = r.lo.x; v[1] = r.lo.y; v[2] = r.lo.z; v[3] = r.lo.w;
    v[4] = r.hi.x; v[5] = r.hi.y; v[6] = r.hi.z; v[7] = r.hi.w;
}
template <typename T> __device__ __forceinline__ void unpack(const Raw8<T> &r, float (&v)[8]) { unpack8(r.u, v, T()); }

// Rounded to nearest, ties to even.
template <bool kVec> __device__ __forceinline__ void store8(float *p, const float (&v)[8], int n)
{
    if (kVec) {
        if (n > 0) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}
template <bool kVec, typename T> __device__ __forceinline__ void store8(T *p, const float (&v)[8], int n)
{
    if (kVec) {
        if (n > 0) *reinterpret_cast<uint4 *>(p) = pack8(v, T());
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = from_f32<T>(v[i]);
    }
}

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

}  // namespace pmpe
