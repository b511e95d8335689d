// The paged key-value cache: rows into their pages, in 16 bits or in e4m3 with
// a scale per position and head, and back.
//
//   8 bits:  s = max(amax |x| / 448, 2^-126),  q = e4m3(x / s),  x ~ q s
//
// A group of lanes holds one head of one row's key or value, eight elements a
// lane (into 8 bits 16 where the rows' alignment allows), so that the largest magnitude is a few shuffles and both sides are
// accessed 16 bytes a lane.  A CTA takes a run of rows.  Where they go (the
// sequence by a search over the offsets, the page by the table: a chain of
// loads) is found for all of them at once, a thread a row, while the first rows
// are on the way; then the groups go through the rows' heads, the next ones'
// loads ahead.  Bytes bound the way back (65533 positions of 4 heads of 128 out
// of e4m3, 203 MB: 37.5 us, 5.4 TB/s); into e4m3 instructions count as much (16377
// rows, 51 MB: 13.5 us, 3.8 TB/s), so that a lane takes 16 elements there.  The same
// rows take 13.7 us into BF16 (their bytes 9.9), in FP32 19.4 into BF16 (14.8) and
// 16.5 into e4m3 (12.4); FP32 rows into 16 bits spill 48 bytes of the 32 registers
// that eight CTAs an SM leave a thread.
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "kv_cache.cuh"

namespace pmpe {
namespace {

// CTAs of an SM.  8 bits back: eight with a head on the way for each group 37.5
// us, four with two 51.  Into 8 bits with 16 elements a lane: four 13.4 us, eight
// (32 registers) 16.9; with eight elements a lane 16.0.
constexpr int kThreads = 256;
constexpr int ctas_of_sm(int wide) { return wide == 2 ? 4 : 8; }
constexpr int kMaxRowsOfCta = 512;

struct CacheParams {
    KvView kv;
    const void *k, *v;        // append: source
    void *k_out, *v_out;      // read: destination
    long long k_ld, k_head_ld, v_ld, v_head_ld;
    int T;
    int sms;                  // of the device
    int rows, heads;          // of a CTA: rows, and of each as many of its keys' and values' heads
    FastDiv by_heads;
};

// The entry (page * kv_heads * page_size + place: of head 0) of row r, -1 for none.
__device__ __forceinline__ long long entry_of(const KvView &kv, int r)
{
    int b = r, last = r + 1;
    if (kv.B == 0) return -1;
    if (kv.cu) {
        int lo = 0, hi = kv.B;  // the last b < B with cu[b] <= r; offsets that decrease lead to some b, checked below
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (__ldg(kv.cu + mid) <= r) lo = mid;
            else hi = mid;
        }
        b = lo;
        last = __ldg(kv.cu + b + 1);
        if (r < __ldg(kv.cu + b) || r >= last) return -1;
    }
    const long long pos = (long long)__ldg(kv.lengths + b) - last + r;
    if (pos < 0 || pos >= kv.capacity) return -1;
    const int j = kv.by_page.quotient((int)pos), page = __ldg(kv.table + b * kv.table_ld + j);
    if ((unsigned)page >= (unsigned)kv.pages) return -1;
    return (long long)page * kv.kv_heads * kv.page_size + ((int)pos - j * kv.page_size);
}

// One head of one row.
struct Item {
    int row, head;  // row: of the CTA's
    bool is_v, live;
};

// kBack: out of the cache.  kLanes: of a head, 8 kWide elements each.  T: the
// rows' type, C: the cache's (uint8_t: e4m3).  kVec: whole vectors.
template <typename T, typename C, int kLanes, bool kVec, bool kBack, int kWide>
__global__ void __launch_bounds__(kThreads, ctas_of_sm(kWide)) cache_kernel(const __grid_constant__ CacheParams p)
{
    constexpr int kGroups = kThreads / kLanes;
    constexpr bool k8 = sizeof(C) == 1;
    __shared__ long long s_entry[kMaxRowsOfCta];
    pdl_trigger();
    pdl_wait();
    const int D = p.kv.head_dim, r0 = blockIdx.x * p.rows, rows = min(p.rows, p.T - r0), h0 = blockIdx.y * p.heads, items = rows * p.heads;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes, c = 8 * kWide * lane;
    auto item = [&](int n) {
        Item it;
        it.row = p.by_heads.quotient(n);
        const int h = h0 + n - it.row * p.heads;
        it.is_v = h >= p.kv.kv_heads;
        it.head = it.is_v ? h - p.kv.kv_heads : h;
        it.live = n < items && it.head < p.kv.kv_heads && c < D;
        return it;
    };
    // an item's eight elements, and what scales them, as they lie in memory
    struct Loaded {
        typename std::conditional<kBack && k8, uint2, Raw8<typename std::conditional<kBack, typename std::conditional<k8, float, C>::type, T>::type>>::type raw[kWide];
        float scale;
    };
    auto fetch = [&](int n, Loaded &l) {
        const Item it = item(n);
        memset(&l, 0, sizeof(l));
        if (!it.live) return;
        if constexpr (!kBack) {
            const T *src = it.is_v ? (const T *)p.v + (r0 + it.row) * p.v_ld + it.head * p.v_head_ld
                                   : (const T *)p.k + (r0 + it.row) * p.k_ld + it.head * p.k_head_ld;
            if (kVec && kWide == 2 && sizeof(T) == 2) {  // 32 bytes at once
                Raw8<float> both;
                load8<true>(both, (const float *)(src + c), 8);
                memcpy(&l.raw, &both, sizeof(l.raw));
            } else if (kVec) {
#pragma unroll
                for (int w = 0; w < kWide; ++w) load8<true>(l.raw[w], src + c + 8 * w, 8);
            } else {
                T v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = src[c + j];
                memcpy(&l.raw, v, sizeof(v));
            }
        } else {
            const long long e0 = s_entry[it.row], e = e0 + (long long)it.head * p.kv.page_size;
            if (e0 < 0) return;
            const C *at = (const C *)(it.is_v ? p.kv.v : p.kv.k) + e * D + c;
            if constexpr (k8) {
                l.raw[0] = *reinterpret_cast<const uint2 *>(at);
                l.scale = (it.is_v ? p.kv.v_scale : p.kv.k_scale)[e];
            } else {
                load8<true>(l.raw[0], at, 8);
            }
        }
    };
    Loaded now, next;
    if (!kBack) fetch(group, now);
    for (int i = threadIdx.x; i < rows; i += kThreads) s_entry[i] = entry_of(p.kv, r0 + i);
    __syncthreads();
    if (kBack) fetch(group, now);
    for (int n = group; n - group < items; n += kGroups) {
        fetch(n + kGroups, next);
        const Item it = item(n);
        if constexpr (!kBack) {
            float x[kWide][8];
#pragma unroll
            for (int w = 0; w < kWide; ++w) unpack(now.raw[w], x[w]);
            const long long e0 = it.live ? s_entry[it.row] : -1, e = e0 + (long long)it.head * p.kv.page_size;
            C *at = (C *)(it.is_v ? p.kv.v : p.kv.k) + e * D + c;
            if constexpr (k8) {
                float amax = 0.f;
#pragma unroll
                for (int w = 0; w < kWide; ++w)
#pragma unroll
                    for (int j = 0; j < 8; ++j) amax = max_magnitude(amax, x[w][j]);
#pragma unroll
                for (int off = kLanes / 2; off > 0; off >>= 1) amax = max_magnitude(amax, __shfl_xor_sync(~0u, amax, off));
                float s;
                const Divide by = divide_by(amax, 1.f, s);
                if (e0 >= 0) {
                    if (lane == 0) (it.is_v ? p.kv.v_scale : p.kv.k_scale)[e] = s;
                    uint32_t q[2 * kWide];
#pragma unroll
                    for (int w = 0; w < kWide; ++w)
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            float y[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) y[k] = fmaf(x[w][j + k], by.hi, x[w][j + k] * by.lo);
                            q[2 * w + j / 4] = e4m3x2(y[0], y[1]) | e4m3x2(y[2], y[3]) << 16;
                        }
                    if constexpr (kWide == 2)
                        *reinterpret_cast<uint4 *>(at) = make_uint4(q[0], q[1], q[2], q[3]);
                    else
                        *reinterpret_cast<uint2 *>(at) = make_uint2(q[0], q[1]);
                }
            } else {
                if (e0 >= 0) store8<true>(at, x[0], 8);
            }
        } else {
            float x[8];
            if constexpr (k8) {
                uint32_t h[4];
                e4m3x4_to_f16(now.raw[0].x, h[0], h[1]);
                e4m3x4_to_f16(now.raw[0].y, h[2], h[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[j]));
                    x[2 * j] = f.x * now.scale;
                    x[2 * j + 1] = f.y * now.scale;
                }
            } else {
                unpack(now.raw[0], x);
            }
            if (it.live) {
                T *to = (T *)(it.is_v ? p.v_out : p.k_out) + ((long long)(r0 + it.row) * p.kv.kv_heads + it.head) * D + c;
                if (kVec) {
                    store8<true>(to, x, 8);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) to[j] = from_f32<T>(x[j]);
                }
            }
        }
        now = next;
    }
}

template <typename T, typename C, int kLanes, bool kVec, bool kBack, int kWide = 1> cudaError_t launch_l(CacheParams &p, cudaStream_t st)
{
    // rows of a CTA: as many as fill its groups once, or more, so that the CTAs
    // of all SMs take all rows at once
    constexpr int kGroups = kThreads / kLanes;
    const int all = 2 * p.kv.kv_heads;
    p.heads = std::min(all, kGroups);
    const int parts = (all + p.heads - 1) / p.heads;
    const long long ctas = p.sms * ctas_of_sm(kWide), share = ((long long)p.T * parts + ctas - 1) / ctas;
    p.rows = (int)std::min<long long>(std::max<long long>(kGroups / p.heads, share), kMaxRowsOfCta);
    p.by_heads = FastDiv(p.heads);
    return launch_pdl(cache_kernel<T, C, kLanes, kVec, kBack, kWide>, dim3((p.T + p.rows - 1) / p.rows, parts), dim3(kThreads), 0, st, p);
}
// vec: 0 single elements, 1 vectors of eight, 2 pairs of those.
template <typename T, typename C, bool kBack> cudaError_t launch_tc(CacheParams &p, int vec, cudaStream_t st)
{
    const int lanes = (p.kv.head_dim + 7) / 8;
    if (vec == 0) return launch_l<T, C, 32, false, kBack>(p, st);
    if constexpr (!kBack && sizeof(C) == 1) {
        // into 8 bits, where instructions bound it, 16 elements a lane
        if (vec == 2) return lanes <= 16 ? launch_l<T, C, 8, true, kBack, 2>(p, st) : launch_l<T, C, 16, true, kBack, 2>(p, st);
    }
    if (lanes <= 8) return launch_l<T, C, 8, true, kBack>(p, st);
    if (lanes <= 16) return launch_l<T, C, 16, true, kBack>(p, st);
    return launch_l<T, C, 32, true, kBack>(p, st);
}
template <bool kBack> cudaError_t launch_types(CacheParams p, int type, int cache_type, int vec, cudaStream_t st)
{
    auto by_cache = [&](auto t) {
        using T = decltype(t);
        if (cache_type == PMPE_BF16) return launch_tc<T, bf16, kBack>(p, vec, st);
        if (cache_type == PMPE_F16) return launch_tc<T, __half, kBack>(p, vec, st);
        return launch_tc<T, uint8_t, kBack>(p, vec, st);
    };
    if (type == PMPE_F32) return by_cache(0.f);
    if (type == PMPE_BF16) return by_cache(bf16());
    return by_cache(__half());
}

}  // namespace

cudaError_t launch_kv_append(const pmpe_kv_cache &c, const pmpe_kv_sequences &s, const pmpe_kv_append_desc &d, int num_sms, cudaStream_t st)
{
    const CacheParams p = {KvView(c, s), d.k, d.v, nullptr, nullptr, d.k_ld, d.k_head_ld, d.v_ld, d.v_head_ld, d.T, num_sms, 0, 0, FastDiv(1)};
    const bool f32 = d.type == PMPE_F32;
    const int64_t ld = d.k_ld | d.v_ld | d.k_head_ld | d.v_head_ld;
    int vec = aligned8(d.k, f32) && aligned8(d.v, f32) && ld % 8 == 0;
    if (vec && (f32 || (((uintptr_t)d.k | (uintptr_t)d.v) % 32 == 0 && ld % 16 == 0))) vec = 2;
    return launch_types<false>(p, d.type, c.type, vec, st);
}

cudaError_t launch_kv_read(const pmpe_kv_cache &c, const pmpe_kv_sequences &s, int T, int type, void *k, void *v, int num_sms, cudaStream_t st)
{
    const CacheParams p = {KvView(c, s), nullptr, nullptr, k, v, 0, 0, 0, 0, T, num_sms, 0, 0, FastDiv(1)};
    const bool f32 = type == PMPE_F32;
    return launch_types<true>(p, type, c.type, aligned8(k, f32) && aligned8(v, f32), st);
}

}  // namespace pmpe
