// Clipping of many gradients by their global norm:
//
//   n = sqrt(sum over all tensors of g^2),  f = min(1, max_norm / (n + 1e-6)),  g <- f g
//
// The first launch sums the squares, the second forms n and f from the CTAs'
// partial sums (every CTA the same way) and scales.  Two launches rather than
// a grid barrier: no CTA waits for another.  The tensors' pointers travel as
// kernel arguments, so nothing is copied to the device before the call and a
// captured graph keeps them.  (One cluster of 16 CTAs for the small cases, its
// sums exchanged through shared memory, took 13 us where two launches take 5.)
//
// A chunk is 16 KB of one tensor.  Bytes bound both launches: every gradient
// is read by each, and written once.  The second takes the chunks from last
// to first, so that it finds in L2 what the first read last.
//
// A thread's squares of a chunk are summed in FP32 (four vectors by themselves,
// then those), the chunks' sums in pairs of FP32 words (a value and what its
// rounding lost, 48 bits: FP64 adds, two a clock and SM, took longer than the
// small cases' loads).  Where a thread's sum leaves 2^-120 .. 2^90 (values that
// overflow or vanish when squared) its vectors go to a 64-bit sum instead,
// which exists in the CTAs that met one: five times the time where all of a
// gradient is such (94 MB of BF16 at 1e-20: 208 us); zeros of either sign are not.
#include <algorithm>
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
// Chunks at the end of the first launch that are left in L2 for the second
// (72 MB; what comes before them passes through): 604 MB of FP32 283 us (277 now), with
// all of them or none 293; 2500 to 7000 chunks are within a microsecond.
constexpr uint32_t kKept = 4500;

// The tensors of a launch: their whole 16-byte vectors, and the elements
// before and after those (fewer than 16 bytes each).  first[i]: chunks before
// tensor i.
template <int kCap> struct ClipTable {
    const uint4 *body[kCap];
    uint8_t *out[kCap];  // where the clipped vectors go
    long long vecs[kCap];
    uint32_t first[kCap + 1];
    uint8_t type[kCap], head[kCap], tail[kCap];
    int count;
};
constexpr int kSmallTable = 64, kLargeTable = 1024;
static_assert(sizeof(ClipTable<kLargeTable>) + 64 <= 32764, "kernel arguments");

__host__ __device__ __forceinline__ int elem_shift(int type) { return type == PMPE_F32 ? 2 : 1; }
// Elements before the first 16-byte boundary of a tensor.
inline long long head_of(const void *p, long long n, int type)
{
    const long long h = (long long)((16u - ((uintptr_t)p & 15u)) & 15u) >> elem_shift(type);
    return std::min(h, n);
}
// Chunks of a tensor: its whole vectors, and one at least for what is before and after them.
inline long long chunks_of(const pmpe_grad &g)
{
    const long long bytes = (g.n - head_of(g.grad, g.n, g.type)) << elem_shift(g.type);
    const long long c = (bytes + kChunkBytes - 1) / kChunkBytes;
    return g.n > 0 && c < 1 ? 1 : c;
}

// A vector's elements.
template <typename T> struct Elems {
    static constexpr int n = 16 / (int)sizeof(T);
    float v[n];
};
__device__ __forceinline__ Elems<float> elems(const uint4 &u, float)
{
    return {{__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)}};
}
template <typename T> __device__ __forceinline__ Elems<T> elems(const uint4 &u, T)
{
    Elems<T> e;
    unpack8(u, e.v, T());
    return e;
}
__device__ __forceinline__ uint4 vector_of(const Elems<float> &e)
{
    return make_uint4(__float_as_uint(e.v[0]), __float_as_uint(e.v[1]), __float_as_uint(e.v[2]), __float_as_uint(e.v[3]));
}
template <typename T> __device__ __forceinline__ uint4 vector_of(const Elems<T> &e) { return pack8(e.v, T()); }
// Calls go with an element of the type.
template <typename Go> __device__ __forceinline__ void by_type(int type, Go go)
{
    if (type == PMPE_F32) go(0.f);
    else if (type == PMPE_BF16) go(bf16());
    else go(__half());
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

// A chunk: its tensor's vectors, and with the tensor's first chunk the
// elements before and after them.
struct Chunk {
    const uint4 *body;
    uint8_t *out;
    long long vecs, v0;
    int type, head, tail;
};
template <int kCap> __device__ __forceinline__ Chunk chunk_at(const ClipTable<kCap> &tab, uint32_t c, int &i)
{
    if (c < tab.first[i] || c >= tab.first[i + 1]) i = tensor_of(tab, c);
    Chunk k;
    k.body = tab.body[i];
    k.out = tab.out[i];
    k.vecs = tab.vecs[i];
    k.v0 = (long long)(c - tab.first[i]) * (kChunkBytes / 16);
    k.type = tab.type[i];
    k.head = k.v0 == 0 ? tab.head[i] : 0;
    k.tail = k.v0 == 0 ? tab.tail[i] : 0;
    return k;
}

// The chunk's vectors of thread t; zeros past the last one.  kLast: not needed
// in L2 afterwards.
template <bool kLast> __device__ __forceinline__ void load_chunk(uint4 (&u)[kClipVecs], const Chunk &k, int t)
{
#pragma unroll
    for (int q = 0; q < kClipVecs; ++q) {
        const long long at = k.v0 + q * kClipThreads + t;
        u[q] = at >= k.vecs ? make_uint4(0u, 0u, 0u, 0u) : kLast ? __ldcs(k.body + at) : k.body[at];
    }
}

// The squares of a thread's part of a chunk in 64 bits, from memory again.
__device__ __forceinline__ double exact_squares(const Chunk &k, int t)
{
    double sum = 0.;
    const int per = 16 >> elem_shift(k.type);
#pragma unroll 1
    for (int q = 0; q < kClipVecs; ++q) {
        const long long at = k.v0 + q * kClipThreads + t;
#pragma unroll 1
        for (int j = 0; j < per && at < k.vecs; ++j) {
            const double x = load_one(k.body, at * per + j, k.type);
            sum += x * x;
        }
    }
    if (t < k.head) {
        const double x = load_one(k.body, t - k.head, k.type);
        sum += x * x;
    }
    if (t < k.tail) {
        const double x = load_one(k.body + k.vecs, t, k.type);
        sum += x * x;
    }
    return sum;
}

__device__ __forceinline__ void square_chunk(const uint4 (&u)[kClipVecs], const Chunk &k, int t, Sum2 &sum, double &rare)
{
    float all = 0.f;
    uint32_t any = 0, any_end = 0;  // bits of the elements: without the signs, zero for zeros alone
    if (t < max(k.head, k.tail)) {  // at most seven of each
        const float a = t < k.head ? load_one(k.body, t - k.head, k.type) : 0.f;
        const float b = t < k.tail ? load_one(k.body + k.vecs, t, k.type) : 0.f;
        all = a * a + b * b;
        any_end = (__float_as_uint(a) | __float_as_uint(b)) & 0x7fffffffu;
    }
#pragma unroll
    for (int q = 0; q < kClipVecs; ++q) any |= u[q].x | u[q].y | u[q].z | u[q].w;
    by_type(k.type, [&](auto zero) {
#pragma unroll
        for (int q = 0; q < kClipVecs; ++q) {
            const auto e = elems(u[q], zero);
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < e.n; ++j) s += e.v[j] * e.v[j];
            all += s;
        }
    });
    if (all >= 0x1p-120f && all < 0x1p90f) add2(sum, all);
    else if ((any & (k.type == PMPE_F32 ? 0x7fffffffu : 0x7fff7fffu)) | any_end) rare += exact_squares(k, t);
}

// f times a power of two: 1, or 2^-126 where f alone would be subnormal and
// lose its bits (gradients near FP32's limit, a small max_norm).
struct Factor {
    float f, post;
};

// A chunk scaled by such a factor, an element at a time: the second product is
// exact but where its result is subnormal.  (Both products for every chunk:
// 94 MB of BF16 43.9 -> 45.1 us.)
__device__ __forceinline__ void scale_chunk_twice(const Chunk &k, int t, const Factor &f)
{
    const int per = 16 >> elem_shift(k.type);
    auto scale = [&](long long i) { store_one(k.out, i, k.type, load_one(k.body, i, k.type) * f.f * f.post); };
#pragma unroll 1
    for (int q = 0; q < kClipVecs; ++q) {
        const long long at = k.v0 + q * kClipThreads + t;
#pragma unroll 1
        for (int j = 0; j < per && at < k.vecs; ++j) scale(at * per + j);
    }
    if (t < k.head) scale(t - k.head);
    if (t < k.tail) scale(k.vecs * per + t);
}

__device__ __forceinline__ void scale_chunk(const uint4 (&u)[kClipVecs], const Chunk &k, int t, float f)
{
    const int per = 16 >> elem_shift(k.type);
    const bool vec_out = ((uintptr_t)k.out & 15u) == 0;
    by_type(k.type, [&](auto zero) {
#pragma unroll
        for (int q = 0; q < kClipVecs; ++q) {
            const long long at = k.v0 + q * kClipThreads + t;
            if (at >= k.vecs) continue;
            auto e = elems(u[q], zero);
#pragma unroll
            for (int j = 0; j < e.n; ++j) e.v[j] *= f;
            if (vec_out) {
                __stcs(reinterpret_cast<uint4 *>(k.out) + at, vector_of(e));
            } else {  // an output that is not aligned as its gradient is
#pragma unroll
                for (int j = 0; j < e.n; ++j) store_one(k.out, at * e.n + j, k.type, e.v[j]);
            }
        }
    });
    if (t < k.head) store_one(k.out, t - k.head, k.type, f * load_one(k.body, t - k.head, k.type));
    if (t < k.tail) store_one(k.out, k.vecs * per + t, k.type, f * load_one(k.body + k.vecs, t, k.type));
}

// n and f from the sums of all squares.  A norm that is not finite as FP32,
// as the caller sees it, clips nothing: the step is dropped.
__device__ __forceinline__ Factor factor_of(const Squares &all, float max_norm, float &norm)
{
    double n64;
    if (all.rare == 0.) {
        norm = sqrtf(all.s.hi + all.s.lo);
        const float f = fminf(1.f, max_norm / (norm + 1e-6f));
        if (f >= 0x1p-126f || max_norm == 0.f) return {f, 1.f};
        n64 = norm;
    } else {
        n64 = sqrt((double)all.s.hi + all.s.lo + all.rare);
        norm = (float)n64;
        if (!isfinite(norm)) return {1.f, 1.f};
    }
    const double f64 = fmin(1., max_norm / (n64 + 1e-6));
    return f64 >= 0x1p-126 || max_norm == 0.f ? Factor{(float)f64, 1.f} : Factor{(float)(f64 * 0x1p126), 0x1p-126f};
}

template <int kCap>
__global__ void __launch_bounds__(kClipThreads, kClipCtasPerSm) clip_squares_kernel(const __grid_constant__ ClipTable<kCap> tab, Squares *partial)
{
    pdl_trigger();
    pdl_wait();
    Sum2 sum = {0.f, 0.f};
    double rare = 0.;
    const uint32_t chunks = tab.first[tab.count];
    int i = 0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = chunk_at(tab, c, i);
        uint4 u[kClipVecs];
        if (c + kKept < chunks) load_chunk<true>(u, k, threadIdx.x);
        else load_chunk<false>(u, k, threadIdx.x);
        square_chunk(u, k, threadIdx.x, sum, rare);
    }
    const Squares r = cta_sum(sum, rare);
    if (threadIdx.x == 0) partial[blockIdx.x] = r;
}

template <int kCap>
__global__ void __launch_bounds__(kClipThreads, kScaleCtasPerSm) clip_scale_kernel(const __grid_constant__ ClipTable<kCap> tab,
                                                                  const Squares *partial, int n_partial, float max_norm,
                                                                  float *norm_out)
{
    pdl_trigger();
    pdl_wait();
    Sum2 sum = {0.f, 0.f};
    double rare = 0.;
    for (int i = threadIdx.x; i < n_partial; i += kClipThreads) {
        const Squares q = partial[i];
        add2(sum, q.s.hi);
        sum.lo += q.s.lo;
        rare += q.rare;
    }
    float norm;
    const Factor f = factor_of(cta_sum(sum, rare), max_norm, norm);
    if (blockIdx.x == 0 && threadIdx.x == 0 && norm_out) *norm_out = norm;
    int i = tab.count - 1;
    const uint32_t chunks = tab.first[tab.count];
    if (f.post != 1.f) {
#pragma unroll 1
        for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) scale_chunk_twice(chunk_at(tab, c, i), threadIdx.x, f);
        return;
    }
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = chunk_at(tab, chunks - 1 - c, i);
        if (f.f == 1.f && (const uint8_t *)k.body == k.out) continue;
        uint4 u[kClipVecs];
        load_chunk<true>(u, k, threadIdx.x);
        scale_chunk(u, k, threadIdx.x, f.f);
    }
}

template <int kCap> void fill(ClipTable<kCap> &tab, const pmpe_grad *g, int n)
{
    tab.count = n;
    uint32_t chunks = 0;
    for (int i = 0; i < n; ++i) {
        const int sh = elem_shift(g[i].type);
        const long long head = head_of(g[i].grad, g[i].n, g[i].type), vecs = ((g[i].n - head) << sh) / 16;
        tab.body[i] = (const uint4 *)((const uint8_t *)g[i].grad + (head << sh));
        tab.out[i] = (uint8_t *)(g[i].out ? g[i].out : g[i].grad) + (head << sh);
        tab.vecs[i] = vecs;
        tab.head[i] = (uint8_t)head;
        tab.tail[i] = (uint8_t)(g[i].n - head - (vecs * 16 >> sh));
        tab.type[i] = (uint8_t)g[i].type;
        tab.first[i] = chunks;
        chunks += (uint32_t)chunks_of(g[i]);
    }
    tab.first[n] = chunks;
}

long long count_chunks(const pmpe_grad *g, int n)
{
    long long chunks = 0;
    for (int i = 0; i < n; ++i) chunks += chunks_of(g[i]);
    return chunks;
}
int ctas_for(long long chunks) { return (int)std::max<long long>(1, std::min<long long>(chunks, kClipMaxCtas)); }

// Both launches for every kCap tensors; all of the first kind come before the second's.
template <int kCap>
cudaError_t clip_tables(const pmpe_grad *g, int n, float max_norm, float *norm_out, Squares *partial, cudaStream_t st)
{
    int all = 0;
    for (int phase = 0; phase < 2; ++phase) {
        int parts = 0;
        for (int at = 0; at == 0 || at < n; at += kCap) {
            ClipTable<kCap> tab;
            fill(tab, g + at, std::min(kCap, n - at));
            const int grid = ctas_for(tab.first[tab.count]);
            const cudaError_t err =
                phase == 0 ? launch_pdl(clip_squares_kernel<kCap>, dim3(grid), dim3(kClipThreads), 0, st, tab, partial + parts)
                           : launch_pdl(clip_scale_kernel<kCap>, dim3(std::min(grid, kScaleMaxCtas)), dim3(kClipThreads), 0, st, tab,
                                        (const Squares *)partial, all, max_norm, at == 0 ? norm_out : (float *)nullptr);
            if (err != cudaSuccess) return err;
            parts += grid;
        }
        all = parts;
    }
    return cudaSuccess;
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
    for (int i = 0; i < n; ++i) {
        if (g[i].n == 0) continue;
        const uintptr_t bytes = (uintptr_t)g[i].n << elem_shift(g[i].type);
        s[m++] = {(uintptr_t)g[i].grad, (uintptr_t)g[i].grad + bytes};
        if (g[i].out && g[i].out != g[i].grad) s[m++] = {(uintptr_t)g[i].out, (uintptr_t)g[i].out + bytes};
    }
    std::sort(s, s + m, [](const Span &a, const Span &b) { return a.lo < b.lo; });
    bool ok = count_chunks(g, n) < (1LL << 31);
    for (size_t i = 1; i < m; ++i) ok = ok && s[i - 1].hi <= s[i].lo;
    delete[] s;
    return ok ? 1 : 0;
}

cudaError_t launch_clip(const pmpe_grad *g, int n, float max_norm, float *norm_out, void *workspace, cudaStream_t st)
{
    Squares *partial = static_cast<Squares *>(workspace);
    // the table travels with every launch: 1.9 KB or 30 KB
    return n <= kSmallTable ? clip_tables<kSmallTable>(g, n, max_norm, norm_out, partial, st)
                            : clip_tables<kLargeTable>(g, n, max_norm, norm_out, partial, st);
}

}  // namespace pmpe
