// What the norm and its backward share: a thread's place in a row, and
// typed loads of eight elements.
#pragma once

#include "elem.cuh"

namespace pmpe {

// A thread's place in its row: columns col(i) .. of chunk i (elem.cuh says
// which eight), G threads a row.
template <bool kWarpRow, bool kVec> struct Place {
    int G, t;
    __device__ __forceinline__ Place()
        : G(kWarpRow ? 32 : (int)blockDim.x), t(kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x) {}
    __device__ __forceinline__ int col(int i) const { return kVec ? 8 * (i * G + t) : 256 * (i * (G >> 5) + (t >> 5)) + (t & 31); }
};

// Eight elements of T or FP32, as loaded.
template <bool kVec, typename T> __device__ __forceinline__ void load_any(Raw8<float> &r, const void *p, int f32, long long at, int n)
{
    if (f32 || sizeof(T) == 4) {
        load8<kVec>(r, (const float *)p + at, n);
    } else if constexpr (sizeof(T) == 2) {
        Raw8<T> q;
        load8<kVec>(q, (const T *)p + at, n);
        r.u = q.u;
    }
}
template <typename T> __device__ __forceinline__ void unpack_any(const Raw8<float> &r, int f32, float (&v)[8])
{
    if (f32 || sizeof(T) == 4) {
        unpack(r, v);
    } else if constexpr (sizeof(T) == 2) {
        unpack8(r.u, v, T());
    }
}

}  // namespace pmpe
