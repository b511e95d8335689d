// Clipping of many gradients by their global norm:
//
//   n = sqrt(sum over all tensors of g^2),  f = min(1, max_norm / (n + 1e-6)),  g <- f g
//
// The first launch sums the squares, the second forms n and f from the CTAs'
// partial sums (every CTA the same way) and scales.  Two launches rather than
// a grid barrier: no CTA waits for another.  The tensors' pointers travel as
// kernel arguments, so nothing is copied to the device before the call and a
// captured graph keeps them.
//
// A chunk is 16 KB of one tensor.  Bytes bound both launches: every gradient
// is read by each, and written once.  The second takes the chunks from last
// to first, so that it finds in L2 what the first read last.
//
// A vector's squares are summed in FP32, the vectors' sums in pairs of FP32
// words (a value and what its rounding lost, 48 bits: FP64 adds, two a clock
// and SM, took longer than the small cases' loads).  A vector whose sum of
// squares leaves 2^-120 .. 2^90 (values that overflow or vanish when squared)
// goes to a 64-bit sum instead, which exists in the CTAs that met one.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <new>

#include "elem.cuh"

namespace pmpe {
namespace {

constexpr int kClipThreads = 256;
constexpr int kClipVecs = 4;                                   // 16-byte vectors of a thread and chunk
constexpr int kChunkBytes = kClipThreads * kClipVecs * 16;
constexpr int kClipCtasPerSm = 8;
constexpr int kScaleCtasPerSm = 5;  // its registers allow no more
constexpr int kClipMaxCtas = 152 * kClipCtasPerSm;
constexpr int kScaleMaxCtas = 152 * kScaleCtasPerSm;

// The tensors of a launch.  first[i]: chunks before tensor i.
template <int kCap> struct ClipTable {
    const void *g[kCap];
    void *o[kCap];
    long long n[kCap];
    uint32_t first[kCap + 1];
    uint8_t type[kCap];
    int count;
};
constexpr int kSmallTable = 64, kLargeTable = 1024;
static_assert(sizeof(ClipTable<kLargeTable>) + 64 <= 32764, "kernel arguments");

__host__ __device__ __forceinline__ int elem_bytes(int type) { return type == PMPE_F32 ? 4 : 2; }
// Elements before the first 16-byte boundary of a tensor.
__host__ __device__ __forceinline__ long long head_of(const void *p, long long n, int bytes)
{
    const long long h = (long long)((16u - ((uintptr_t)p & 15u)) & 15u) / bytes;
    return h < n ? h : n;
}
// Chunks of a tensor: its whole vectors, and one at least for what is before and after them.
__host__ __device__ __forceinline__ long long chunks_of(const void *p, long long n, int type)
{
    const int b = elem_bytes(type);
    const long long bytes = (n - head_of(p, n, b)) * b;
    const long long c = (bytes + kChunkBytes - 1) / kChunkBytes;
    return n > 0 && c < 1 ? 1 : c;
}

__device__ __forceinline__ void unpack_vec(const uint4 &u, int type, float (&v)[8])
{
    if (type == PMPE_F32) {
        v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
        v[4] = v[5] = v[6] = v[7] = 0.f;
    } else if (type == PMPE_BF16) {
        unpack8(u, v, bf16());
    } else {
        unpack8(u, v, __half());
    }
}
__device__ __forceinline__ float load_one(const void *p, long long i, int type)
{
    return type == PMPE_F32 ? ((const float *)p)[i]
                            : type == PMPE_BF16 ? to_f32(((const bf16 *)p)[i]) : to_f32(((const __half *)p)[i]);
}
__device__ __forceinline__ void store_one(void *p, long long i, int type, float v)
{
    if (type == PMPE_F32) ((float *)p)[i] = v;
    else if (type == PMPE_BF16) ((bf16 *)p)[i] = from_f32<bf16>(v);
    else ((__half *)p)[i] = from_f32<__half>(v);
}

// A sum of FP32 values and what its roundings lost.
struct Sum2 {
    float hi, lo;
};
__device__ __forceinline__ void add2(Sum2 &s, float v)
{
    const float t = s.hi + v, bb = t - s.hi;
    s.lo += (s.hi - (t - bb)) + (v - bb);
    s.hi = t;
}

// What a CTA (or all of them) found: the pair, and the 64-bit sum of the rest.
struct Squares {
    Sum2 s;
    double rare;
};

// The squares of a vector, added to the sums.
__device__ __forceinline__ void add_squares(const float (&v)[8], float &fast, double &rare)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[i] * v[i];
    if (s >= 0x1p-120f && s < 0x1p90f) {
        fast += s;
    } else {
        uint32_t any = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) any |= __float_as_uint(v[i]);
        if (any << 1) {  // zeros stay here
#pragma unroll
            for (int i = 0; i < 8; ++i) rare += (double)v[i] * v[i];
        }
    }
}

// The sums over the CTA's threads, in a fixed order, in all of them.
__device__ __forceinline__ Squares cta_sum(Sum2 s, double rare)
{
    __shared__ Sum2 s_sum[kClipThreads / 32];
    __shared__ double s_rare[kClipThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const float hi = __shfl_xor_sync(~0u, s.hi, off), lo = __shfl_xor_sync(~0u, s.lo, off);
        add2(s, hi);
        s.lo += lo;
    }
    if (lane == 0) s_sum[warp] = s;
    const int any = __syncthreads_or(!(rare == 0.));  // NaN too
    Squares r;
    r.s = s_sum[0];
    r.rare = 0.;
#pragma unroll
    for (int w = 1; w < kClipThreads / 32; ++w) {
        add2(r.s, s_sum[w].hi);
        r.s.lo += s_sum[w].lo;
    }
    if (any) {
        rare = warp_sum(rare);
        if (lane == 0) s_rare[warp] = rare;
        __syncthreads();
        for (int w = 0; w < kClipThreads / 32; ++w) r.rare += s_rare[w];
    }
    return r;
}

// The tensor of chunk c.
template <int kCap> __device__ __forceinline__ int tensor_of(const ClipTable<kCap> &tab, uint32_t c)
{
    int lo = 0, hi = tab.count - 1;  // the last tensor with first <= c and chunks of its own
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.first[mid] <= c) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <int kCap>
__global__ void __launch_bounds__(kClipThreads, kClipCtasPerSm) clip_squares_kernel(const __grid_constant__ ClipTable<kCap> tab, Squares *partial)
{
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x;
    Sum2 sum = {0.f, 0.f};
    double rare = 0.;
    const uint32_t chunks = tab.first[tab.count];
    int i = 0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        if (c < tab.first[i] || c >= tab.first[i + 1]) i = tensor_of(tab, c);
        const int type = tab.type[i], b = elem_bytes(type);
        const void *g = tab.g[i];
        const long long n = tab.n[i], head = head_of(g, n, b), vecs = (n - head) * b / 16;
        const uint4 *body = reinterpret_cast<const uint4 *>((const uint8_t *)g + head * b);
        const long long v0 = (long long)(c - tab.first[i]) * (kChunkBytes / 16);
        uint4 u[kClipVecs];
#pragma unroll
        for (int q = 0; q < kClipVecs; ++q) {
            const long long at = v0 + q * kClipThreads + tid;
            u[q] = at < vecs ? __ldg(body + at) : make_uint4(0u, 0u, 0u, 0u);
        }
        float fast = 0.f, v[8];
#pragma unroll
        for (int q = 0; q < kClipVecs; ++q) {
            unpack_vec(u[q], type, v);
            add_squares(v, fast, rare);
        }
        if (v0 == 0) {  // what the vectors leave: fewer than 16 bytes before and after them
            const long long tail = head + vecs * (16 / b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
            if (tid < head) v[0] = load_one(g, tid, type);
            if (tid < n - tail) v[1] = load_one(g, tail + tid, type);
            if (tid < 8) add_squares(v, fast, rare);
        }
        add2(sum, fast);
    }
    const Squares r = cta_sum(sum, rare);
    if (tid == 0) partial[blockIdx.x] = r;
}

template <int kCap>
__global__ void __launch_bounds__(kClipThreads, kScaleCtasPerSm) clip_scale_kernel(const __grid_constant__ ClipTable<kCap> tab,
                                                                  const Squares *partial, int n_partial, float max_norm,
                                                                  float *norm_out)
{
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x;
    Sum2 sum = {0.f, 0.f};
    double rare = 0.;
    for (int i = tid; i < n_partial; i += kClipThreads) {
        const Squares q = partial[i];
        add2(sum, q.s.hi);
        sum.lo += q.s.lo;
        rare += q.rare;
    }
    const Squares all = cta_sum(sum, rare);
    // a norm that is not finite clips nothing: the caller sees it and drops the step
    float norm, f = 1.f;
    if (all.rare == 0.) {
        norm = sqrtf(all.s.hi + all.s.lo);
        f = fminf(1.f, max_norm / (norm + 1e-6f));
    } else {
        const double n64 = sqrt((double)all.s.hi + all.s.lo + all.rare);
        norm = (float)n64;
        if (isfinite(n64)) f = (float)fmin(1., max_norm / (n64 + 1e-6));
    }
    if (blockIdx.x == 0 && tid == 0 && norm_out) *norm_out = norm;
    int i = tab.count - 1;
    const uint32_t chunks = tab.first[tab.count];
    for (uint32_t k = blockIdx.x; k < chunks; k += gridDim.x) {
        const uint32_t c = chunks - 1 - k;
        if (c < tab.first[i] || c >= tab.first[i + 1]) i = tensor_of(tab, c);
        const int type = tab.type[i], b = elem_bytes(type);
        const void *g = tab.g[i];
        void *o = tab.o[i];
        if (f == 1.f && g == o) continue;
        const long long n = tab.n[i], head = head_of(g, n, b), vecs = (n - head) * b / 16, per = 16 / b;
        const uint4 *body = reinterpret_cast<const uint4 *>((const uint8_t *)g + head * b);
        uint8_t *out = (uint8_t *)o + head * b;
        const bool vec_out = ((uintptr_t)out & 15u) == 0;
        const long long v0 = (long long)(c - tab.first[i]) * (kChunkBytes / 16);
        uint4 u[kClipVecs];
#pragma unroll
        for (int q = 0; q < kClipVecs; ++q) {
            const long long at = v0 + q * kClipThreads + tid;
            u[q] = at < vecs ? __ldcs(body + at) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int q = 0; q < kClipVecs; ++q) {
            const long long at = v0 + q * kClipThreads + tid;
            if (at >= vecs) continue;
            float v[8];
            unpack_vec(u[q], type, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= f;
            if (vec_out) {
                const uint4 r = type == PMPE_F32 ? make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]),
                                                              __float_as_uint(v[2]), __float_as_uint(v[3]))
                                                 : type == PMPE_BF16 ? pack8(v, bf16()) : pack8(v, __half());
                __stcs(reinterpret_cast<uint4 *>(out) + at, r);
            } else {  // an output that is not aligned as its gradient is
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < per) store_one(out, at * per + j, type, v[j]);
            }
        }
        if (v0 == 0) {
            const long long tail = head + vecs * per;
            if (tid < head) store_one(o, tid, type, f * load_one(g, tid, type));
            if (tid < n - tail) store_one(o, tail + tid, type, f * load_one(g, tail + tid, type));
        }
    }
}

template <int kCap>
cudaError_t clip_tables(const pmpe_grad *g, int n, float max_norm, float *norm_out, Squares *partial, cudaStream_t st, int phase,
                        int n_partial_all)
{
    int parts = 0;
    for (int at = 0; at == 0 || at < n; at += kCap) {
        ClipTable<kCap> tab;
        tab.count = std::min(kCap, n - at);
        uint32_t chunks = 0;
        for (int i = 0; i < tab.count; ++i) {
            const pmpe_grad &t = g[at + i];
            tab.g[i] = t.grad;
            tab.o[i] = t.out ? t.out : t.grad;
            tab.n[i] = t.n;
            tab.type[i] = (uint8_t)t.type;
            tab.first[i] = chunks;
            chunks += (uint32_t)chunks_of(t.grad, t.n, t.type);
        }
        tab.first[tab.count] = chunks;
        const int grid = (int)std::max<uint32_t>(1u, std::min<uint32_t>(chunks, (uint32_t)kClipMaxCtas));
        const cudaError_t err =
            phase == 0 ? launch_pdl(clip_squares_kernel<kCap>, dim3(grid), dim3(kClipThreads), 0, st, tab, partial + parts)
                       : launch_pdl(clip_scale_kernel<kCap>, dim3(std::min(grid, kScaleMaxCtas)), dim3(kClipThreads), 0, st, tab,
                                    (const Squares *)partial, n_partial_all, max_norm, at == 0 ? norm_out : (float *)nullptr);
        if (err != cudaSuccess) return err;
        parts += grid;
    }
    return cudaSuccess;
}

template <int kCap> int count_partials(const pmpe_grad *g, int n)
{
    int parts = 0;
    for (int at = 0; at == 0 || at < n; at += kCap) {
        long long chunks = 0;
        for (int i = at; i < std::min(n, at + kCap); ++i) chunks += chunks_of(g[i].grad, g[i].n, g[i].type);
        parts += (int)std::max<long long>(1, std::min<long long>(chunks, kClipMaxCtas));
    }
    return parts;
}

}  // namespace

size_t clip_workspace_bytes(int n)
{
    return (size_t)std::max(1, (n + kLargeTable - 1) / kLargeTable) * kClipMaxCtas * sizeof(Squares);
}

// Whether no two of the tensors (gradients and outputs, a gradient and its
// own output apart where they are the same) share memory, and every launch's
// chunks can be counted.  -1: no memory for the check.
int clip_tensors_ok(const pmpe_grad *g, int n)
{
    struct Span { uintptr_t lo, hi; };
    Span *s = new (std::nothrow) Span[2 * (size_t)n + 1];
    if (!s) return -1;
    size_t m = 0;
    long long chunks = 0;
    for (int i = 0; i < n; ++i) {
        if (g[i].n == 0) continue;
        const uintptr_t bytes = (uintptr_t)g[i].n * elem_bytes(g[i].type);
        s[m++] = {(uintptr_t)g[i].grad, (uintptr_t)g[i].grad + bytes};
        if (g[i].out && g[i].out != g[i].grad) s[m++] = {(uintptr_t)g[i].out, (uintptr_t)g[i].out + bytes};
        chunks += chunks_of(g[i].grad, g[i].n, g[i].type);
    }
    std::sort(s, s + m, [](const Span &a, const Span &b) { return a.lo < b.lo; });
    bool ok = chunks < (1LL << 31);
    for (size_t i = 1; i < m; ++i) ok = ok && s[i - 1].hi <= s[i].lo;
    delete[] s;
    return ok ? 1 : 0;
}

cudaError_t launch_clip(const pmpe_grad *g, int n, float max_norm, float *norm_out, void *workspace, cudaStream_t st)
{
    Squares *partial = static_cast<Squares *>(workspace);
    // the table is copied into every launch's arguments: 1.9 KB or 30 KB
    const bool small = n <= kSmallTable;
    const int parts = small ? count_partials<kSmallTable>(g, n) : count_partials<kLargeTable>(g, n);
    for (int phase = 0; phase < 2; ++phase) {
        const cudaError_t err = small ? clip_tables<kSmallTable>(g, n, max_norm, norm_out, partial, st, phase, parts)
                                      : clip_tables<kLargeTable>(g, n, max_norm, norm_out, partial, st, phase, parts);
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

}  // namespace pmpe
