// The paged key-value cache: rows into their pages, in 16 bits or in e4m3 with
// a scale per position and head, and back.
//
//   8 bits:  s = max(amax |x| / 448, 2^-126),  q = e4m3(x / s),  x ~ q s
//
// A group of lanes holds one head of one row's key or value, eight elements a
// lane, so that the largest magnitude is a few shuffles and both sides are
// accessed 16 bytes a lane.  Where a row goes (its sequence by a search over
// the offsets, its page by the table) is found once a CTA, by one thread a row,
// while the rows' loads are on the way: four dependent loads that every group
// would wait for otherwise.  Bytes bound both directions.
#include <algorithm>

#include "kv_cache.cuh"

namespace pmpe {
namespace {

constexpr int kThreads = 256;

struct CacheParams {
    KvView kv;
    const void *k, *v;        // append: source
    void *k_out, *v_out;      // read: destination
    long long k_ld, k_head_ld, v_ld, v_head_ld;
    int T;
    long long items;          // T * 2 * kv_heads
};

// The entry (page * kv_heads * page_size + place: of head 0) of row r, -1 for none.
__device__ __forceinline__ long long entry_of(const KvView &kv, int r)
{
    int b = r, pos;
    if (kv.B == 0) return -1;
    if (kv.cu) {
        int lo = 0, hi = kv.B;  // the last b < B with cu[b] <= r; offsets that decrease lead to some b, checked below
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (__ldg(kv.cu + mid) <= r) lo = mid;
            else hi = mid;
        }
        b = lo;
        const int first = __ldg(kv.cu + b), last = __ldg(kv.cu + b + 1);
        if (r < first || r >= last) return -1;
        const long long at = (long long)__ldg(kv.lengths + b) - last + r;
        if (at < 0 || at >= kv.capacity) return -1;
        pos = (int)at;
    } else {
        pos = __ldg(kv.lengths + b) - 1;
        if (pos < 0 || pos >= kv.capacity) return -1;
    }
    const int j = kv.by_page.quotient(pos), page = __ldg(kv.table + b * kv.table_ld + j);
    if ((unsigned)page >= (unsigned)kv.pages) return -1;
    return (long long)page * kv.kv_heads * kv.page_size + (pos - j * kv.page_size);
}

// kBack: out of the cache.  kLanes: of a head, 8 elements each.  T: the rows'
// type, C: the cache's (uint8_t: e4m3).  kVec: whole vectors.  kPer: heads of a group.
template <typename T, typename C, int kLanes, bool kVec, bool kBack, int kPer>
__global__ void __launch_bounds__(kThreads) cache_kernel(const __grid_constant__ CacheParams p)
{
    constexpr int kGroups = kThreads / kLanes, kItems = kGroups * kPer;
    constexpr bool k8 = sizeof(C) == 1;
    __shared__ long long s_entry[kItems / 2 + 2];
    pdl_trigger();
    pdl_wait();
    const int per_row = 2 * p.kv.kv_heads, D = p.kv.head_dim;
    const long long first = (long long)blockIdx.x * kItems;
    const int r0 = (int)(first / per_row), rows = (int)((min(first + kItems, p.items) - 1) / per_row) - r0 + 1;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes, c = 8 * lane;
    float x[kPer][8];
    int row[kPer], head[kPer];
    bool is_v[kPer], live[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const long long item = first + i * kGroups + group;
        live[i] = item < p.items && c < D;
        const int at = (int)(item - (long long)r0 * per_row);  // below kItems + per_row
        row[i] = at / per_row;
        const int h = at - row[i] * per_row;
        is_v[i] = h >= p.kv.kv_heads;
        head[i] = is_v[i] ? h - p.kv.kv_heads : h;
        if (!kBack && live[i]) {
            const T *src = is_v[i] ? (const T *)p.v + (r0 + row[i]) * p.v_ld + head[i] * p.v_head_ld
                                   : (const T *)p.k + (r0 + row[i]) * p.k_ld + head[i] * p.k_head_ld;
            if (kVec) {
                Raw8<T> raw;
                load8<true>(raw, src + c, 8);
                unpack(raw, x[i]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[i][j] = to_f32<T>(src[c + j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
        }
    }
    for (int i = threadIdx.x; i < rows; i += kThreads) s_entry[i] = entry_of(p.kv, r0 + i);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const long long e0 = live[i] ? s_entry[row[i]] : -1;
        const long long e = e0 + (long long)head[i] * p.kv.page_size;
        C *at = (C *)(is_v[i] ? p.kv.v : p.kv.k) + e * D + c;
        float *scale = (is_v[i] ? p.kv.v_scale : p.kv.k_scale) + e;
        if (!kBack) {
            if constexpr (k8) {
                float amax = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) amax = max_magnitude(amax, x[i][j]);
#pragma unroll
                for (int off = kLanes / 2; off > 0; off >>= 1) amax = max_magnitude(amax, __shfl_xor_sync(~0u, amax, off));
                float s;
                const Divide by = divide_by(amax, 1.f, s);
                if (e0 < 0) continue;
                if (lane == 0) *scale = s;
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = fmaf(x[i][j], by.hi, x[i][j] * by.lo);
                *reinterpret_cast<uint2 *>(at) =
                    make_uint2(e4m3x2(q[0], q[1]) | e4m3x2(q[2], q[3]) << 16, e4m3x2(q[4], q[5]) | e4m3x2(q[6], q[7]) << 16);
            } else {
                if (e0 < 0) continue;
                store8<true>(at, x[i], 8);
            }
        } else {
            if (!live[i]) continue;
            if (e0 >= 0) {
                if constexpr (k8) {
                    const uint2 u = *reinterpret_cast<const uint2 *>(at);
                    const float s = *scale;
                    const uint32_t w[2] = {u.x, u.y};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 f = e4m3x2_to_f32(w[j >> 1] >> 16 * (j & 1));
                        x[i][2 * j] = f.x * s;
                        x[i][2 * j + 1] = f.y * s;
                    }
                } else {
                    Raw8<C> raw;
                    load8<true>(raw, at, 8);
                    unpack(raw, x[i]);
                }
            }
            T *to = (T *)(is_v[i] ? p.v_out : p.k_out) + ((long long)(r0 + row[i]) * p.kv.kv_heads + head[i]) * D + c;
            if (kVec) {
                store8<true>(to, x[i], 8);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) to[j] = from_f32<T>(x[i][j]);
            }
        }
    }
}

template <typename T, typename C, int kLanes, bool kVec, bool kBack> cudaError_t launch_l(const CacheParams &p, cudaStream_t st)
{
    // one head a group until the grid fills the GPU (152 SMs of eight CTAs), then four
    constexpr int kGroups = kThreads / kLanes;
    const long long one = (p.items + kGroups - 1) / kGroups;
    if (one <= 152 * 8) return launch_pdl(cache_kernel<T, C, kLanes, kVec, kBack, 1>, dim3((unsigned)one), dim3(kThreads), 0, st, p);
    const long long four = (p.items + 4 * kGroups - 1) / (4 * kGroups);
    if (four > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_pdl(cache_kernel<T, C, kLanes, kVec, kBack, 4>, dim3((unsigned)four), dim3(kThreads), 0, st, p);
}
template <typename T, typename C, bool kBack> cudaError_t launch_tc(const CacheParams &p, bool vec, cudaStream_t st)
{
    const int lanes = (p.kv.head_dim + 7) / 8;
    if (!vec) return launch_l<T, C, 32, false, kBack>(p, st);
    if (lanes <= 8) return launch_l<T, C, 8, true, kBack>(p, st);
    if (lanes <= 16) return launch_l<T, C, 16, true, kBack>(p, st);
    return launch_l<T, C, 32, true, kBack>(p, st);
}
template <bool kBack> cudaError_t launch_types(const CacheParams &p, int type, int cache_type, bool vec, cudaStream_t st)
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

cudaError_t launch_kv_append(const pmpe_kv_cache &c, const pmpe_kv_sequences &s, const pmpe_kv_append_desc &d, cudaStream_t st)
{
    CacheParams p = {KvView(c, s), d.k, d.v, nullptr, nullptr, d.k_ld, d.k_head_ld, d.v_ld, d.v_head_ld, d.T, (long long)d.T * 2 * c.kv_heads};
    const bool f32 = d.type == PMPE_F32;
    const bool vec = aligned8(d.k, f32) && aligned8(d.v, f32) && d.k_ld % 8 == 0 && d.v_ld % 8 == 0 && d.k_head_ld % 8 == 0 && d.v_head_ld % 8 == 0;
    return launch_types<false>(p, d.type, c.type, vec, st);
}

cudaError_t launch_kv_read(const pmpe_kv_cache &c, const pmpe_kv_sequences &s, int T, int type, void *k, void *v, cudaStream_t st)
{
    CacheParams p = {KvView(c, s), nullptr, nullptr, k, v, 0, 0, 0, 0, T, (long long)T * 2 * c.kv_heads};
    const bool f32 = type == PMPE_F32;
    return launch_types<true>(p, type, c.type, aligned8(k, f32) && aligned8(v, f32), st);
}

}  // namespace pmpe
