// The next token of each row of logits, from given random numbers:
//
//   r_i = e^((z_i - z_max) / temperature), down to 2^-40
//   kept: in the order (z descending, id ascending) the first top_k; of those
//         the ones with less than top_p of their sum before them; of those
//         r >= min_p -- always a prefix of that order
//   drawn: the lowest kept id whose running sum of r, by id, is above u times the sum
//
// A token is an integer, so that sums that differ in their last bits would give
// another one now and then.  Therefore r is evaluated to 2^-31 (not FP32's
// 2^-22; FP64 has a sixty-fourth of its rate here) and held as an integer of
// 2^-46 of the best (finer in short rows): sums of integers do not depend on
// their order.
//
//   x = (z_max - z) log2(e) / temperature  in two words, x = k / 256 + f
//   r = 2^-x = 2^(-k / 256) (1 + q(f)),    the power from a table (Tang 1989),
//   q = 2^-f - 1 a cubic, |f| <= 2^-9:     its FP32 rounding is 2^-33 of r
//
// A cluster of CTAs takes a row, each a run of ids.  One pass finds the largest
// logit.
//   top_k up to 1024: the largest logits of every thread's four runs of loads, in
//     a histogram over x, tell how far down the best top_k tokens reach at most,
//     since each run that shows one there holds one: k runs' tokens at most,
//     nearly k where ids are random.  A second pass lists those, and one CTA
//     finishes with the list.  (With one a thread, top_k 1000 in rows of one CTA
//     had no border and listed all: 400 rows of 32003 119 us, with four 61.)
//   top_p alone, or a larger top_k: a second pass makes histograms of counts and
//     sums over x; the bin where the border lies is listed in a third, which also
//     sums what is above it by runs of ids; the border is found in the list.
//   neither: the second pass sums by runs of ids.
// A list that does not fit (many tokens of about the same logit) is replaced by
// further passes, over the bits of the logits in the border's bin, down to one
// value.  Of equal logits at the border the lowest ids stay.
//
// Latency bounds a single row (131072 tokens, top_k 50, top_p 0.95: 13.3 us, the
// largest logit and the list 5 and 3 of them).  Many rows: r takes 39 instructions a
// token, two tokens at a time, whose issue is half of the 41.5 us of 400 rows of
// 32003; the other half is the grid, 400 CTAs on 304 places (two CTAs a row: 58).
// (64 rows of 131072 22 us with top_k, 29 with neither, 67 with top_p over as many as
// a fifth of the tokens.  16-bit logits spill 36 bytes a thread.)  A row's passes run a few times each, so that fetching their code
// counts: they are not unrolled, and what is seldom needed is out of line.
#include <string.h>

#include <algorithm>

#include <cooperative_groups.h>

#include "elem.cuh"
#include "tc_ptx.cuh"

namespace pmpe {
namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kSegs = 8 * kWarps;    // runs of ids whose sums a CTA keeps
constexpr int kBins = 2048;          // of a histogram
constexpr float kLeast = 40.f;       // log2 of the smallest r, negated
constexpr int kFine = 46;            // bits of r behind the point, for 2^17 tokens
constexpr int kList = 2048;          // tokens of a list
constexpr int kShort = 384;          // of one that each token is compared with all of
constexpr int kWanted = 1024;        // top_k up to which runs' largest logits show the border
constexpr float kLog2eHi = 1.44269502f, kLog2eLo = 1.92596303e-8f;  // log2(e) in two words
constexpr float kFltMax = 3.402823466e38f;

// 2^(-j / 256) as an integer of 2^-31, and 2^31 times it in FP32.
struct Power {
    uint32_t fixed;
    float value;
};
struct Powers {
    Power at[256];
    constexpr Powers() : at()
    {
        for (int j = 0; j < 256; ++j) {
            const double y = -j * (0.69314718055994530942 / 256);
            double term = 1, sum = 1;
            for (int n = 1; n < 30; ++n) {
                term *= y / n;
                sum += term;
            }
            at[j].fixed = (uint32_t)(sum * 2147483648.0 + 0.5);
            at[j].value = (float)(sum * 2147483648.0);
        }
    }
};
__device__ const Powers g_powers;

struct SampleParams {
    const void *logits;
    long long ld;
    const float *u, *temperature, *top_p, *min_p;  // of each row, or NULL:
    const int32_t *top_k;
    float temperature1, top_p1, min_p1;            // of all
    int top_k1;
    int T, V, shift;                               // sums are of 2^(shift - 46)
    int32_t *token;
    float *prob;
};

// A finite logit's place among others: unsigned order is that of the values.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t b = __float_as_uint(z + 0.f);  // -0 becomes 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
// The value below a finite logit.
__device__ __forceinline__ float below(float z)
{
    const uint32_t key = key_of(z);
    return logit_of(key - (key == 0x80000000u ? 2 : 1));  // (the key before that of 0 is -0)
}

// +inf counts as the largest finite logit; NaN stays, and is above and below nothing.
__device__ __forceinline__ float clip(float z)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(kFltMax));
    return r;
}

// What turns logits into x = (pre top - pre z) post (hi + lo).
struct Slope {
    float top, hi, lo, pre, post;
    int shift;
    bool plain;    // pre = post = 1
    float bins;    // of a histogram, for a step of one in x
};
__device__ __forceinline__ Slope slope_of(float top, float temperature, int shift)
{
    Slope s = {top, 0.f, 0.f, 1.f, 1.f, shift, true, 0.f};
    // a power of two keeps the quotient among FP32's normal numbers
    if (temperature > 0x1p90f) {
        s.pre = 0x1p-100f;
        temperature *= 0x1p-100f;
    } else if (temperature < 0x1p-90f) {
        s.post = 0x1p100f;
        temperature *= 0x1p100f;
    }
    s.plain = s.pre == 1.f && s.post == 1.f;
    s.hi = kLog2eHi / temperature;
    if (s.hi > 0.f) s.lo = (fmaf(-s.hi, temperature, kLog2eHi) + kLog2eLo) / temperature;
    return s;
}
// x in one word: it does not decrease as z falls.
__device__ __forceinline__ float x_near(const Slope &s, float z) { return (s.top * s.pre - z * s.pre) * s.post * s.hi; }
struct Ratio {
    float hi, lo;
};
__device__ __forceinline__ Ratio x_of(const Slope &s, float z)
{
    const float a = s.top * s.pre, b = z * s.pre;
    float d = a - b;
    const float bb = a - d;  // the difference's rounding, exactly (Knuth)
    float e = ((a - (d + bb)) + (bb - b));
    d *= s.post;
    e *= s.post;
    const float hi = d * s.hi;
    return {hi, fmaf(d, s.hi, -hi) + fmaf(d, s.lo, e * s.hi)};
}
// r = w 2^-(31 + n), for 0 <= x <= 40.
__device__ __forceinline__ uint32_t power_of(const Ratio &x, const Power *powers, int &n)
{
    const float kf = fmaf(x.hi, 256.f, 12582912.f);  // (an integer in the low bits: 1.5 2^23 is added)
    const int k = __float_as_int(kf) - 0x4b400000;
    const float f = fmaf(kf - 12582912.f, -1.f / 256.f, x.hi) + x.lo;
    const float q = f * fmaf(f, fmaf(f, -0.055504109f, 0.240226507f), -0.693147181f);
    const Power p = powers[k & 255];
    n = k >> 8;
    return p.fixed + __float2int_rn(p.value * q);
}
// r as the sums take it, of a row of up to 2^17 tokens a multiple of 2^-46 or finer:
// rounded to nearest, so that what small ones lose has no direction.  (Cut off,
// 16000 tokens together lost what one of 2^-33 of the sum weighs, and with the
// logits in descending order u = 1 - 2^-24 drew a neighbour.)
__device__ __forceinline__ u64 weight_of(const Slope &s, float z, const Power *powers)
{
    int n;
    const uint32_t w = power_of(x_of(s, z), powers, n);
    n += s.shift - (kFine - 31);
    return n <= 0 ? (u64)w << -n : (u64)((w + ((1u << n) >> 1)) >> n);
}
// The smallest logit for which `in` holds, as it does for the largest and does
// not again further down, by 32 tries at a time; the same in every lane.
template <typename F> __device__ float lowest(float top, F in)
{
    uint32_t below = key_of(-kFltMax) - 1, at = key_of(top);  // not in at `below` (or that is no logit), in at `at`
    while (at - below > 1) {
        const uint32_t step = (at - below + 32) / 33, k = min(at, below + step * ((threadIdx.x & 31) + 1));
        const uint32_t is = __ballot_sync(~0u, in(logit_of(k)));
        const int first = is ? __ffs(is) - 1 : 32;
        const uint32_t from = below;
        if (first < 32) at = min(at, from + step * (first + 1));
        below = min(at - 1, from + step * first);
    }
    return logit_of(at);
}
// Whether x <= (hi, lo).  (Not of infinities.)
__device__ __forceinline__ bool within(const Ratio &x, float hi, float lo) { return (x.hi - hi) + (x.lo - lo) <= 0.f; }

// Two values to an instruction.
struct Two {
    uint64_t v;
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ explicit Two(uint64_t w) : v(w) {}
    __device__ __forceinline__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
};
__device__ __forceinline__ Two fma2(Two a, Two b, Two c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a.v), "l"(b.v), "l"(c.v));
    return Two(r);
}
__device__ __forceinline__ Two add2(Two a, Two b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a.v), "l"(b.v));
    return Two(r);
}
__device__ __forceinline__ Two mul2(Two a, Two b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a.v), "l"(b.v));
    return Two(r);
}
// (For temperatures far from 1: out of line, where rows seldom go.  A row runs
// each of its passes once: their code is fetched as they run, and time is lost
// with what is skipped as well.)
__device__ __noinline__ u64 weight_apart(Slope s, float z, const Power *powers) { return weight_of(s, z, powers); }
// weight_of() of two logits, the same arithmetic; 0 where `in` is false.
__device__ __forceinline__ void weights_of(const Slope &s, float z0, float z1, bool in0, bool in1, const Power *powers, u64 &w0, u64 &w1)
{
    if (!s.plain) {
        w0 = in0 ? weight_apart(s, z0, powers) : 0;
        w1 = in1 ? weight_apart(s, z1, powers) : 0;
        return;
    }
    const Two minus(-1.f, -1.f), a(s.top, s.top), z(z0, z1), c(s.hi, s.hi);
    const Two d = fma2(z, minus, a), bb = fma2(d, minus, a);
    const Two e = add2(fma2(add2(d, bb), minus, a), fma2(z, minus, bb));
    const Two hi = mul2(d, c), lo = fma2(d, c, mul2(hi, minus)), lo2 = add2(lo, fma2(d, Two(s.lo, s.lo), mul2(e, c)));
    const Two kf = fma2(hi, Two(256.f, 256.f), Two(12582912.f, 12582912.f));
    const Two f = add2(fma2(add2(kf, Two(-12582912.f, -12582912.f)), Two(-1.f / 256.f, -1.f / 256.f), hi), lo2);
    const Two q = mul2(f, fma2(f, fma2(f, Two(-0.055504109f, -0.055504109f), Two(0.240226507f, 0.240226507f)), Two(-0.693147181f, -0.693147181f)));
    float k[2], qs[2];
    kf.get(k[0], k[1]);
    q.get(qs[0], qs[1]);
    u64 w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int bits = __float_as_int(k[i]);
        const Power p = powers[bits & 255];
        const uint32_t v = p.fixed + __float2int_rn(p.value * qs[i]);
        const bool in = i ? in1 : in0;
        const int down = in ? (bits >> 8) - (0x4b400000 >> 8) + s.shift - (kFine - 31) : 0;  // v 2^-down
        const int by = max(down, 0);
        w[i] = (u64)((v + ((1u << by) >> 1)) >> by) * (in ? 1u << max(-down, 0) : 0u);
    }
    w0 = w[0];
    w1 = w[1];
}

struct Shared {
    Power powers[256];
    uint32_t mass_lo[kBins], mass_hi[kBins], count[kBins];
    u64 mass_x[kBins];       // of the histogram over x, all CTAs': each CTA has a share of the bins
    uint32_t count_x[kBins];
    u64 mass_of[kMaxCluster], count_of[kMaxCluster];  // of the CTAs' shares
    u64 border_mass;         // before the bin of the border
    uint32_t border_bin, border_count;
    float list_z[kList];
    int list_id[kList];
    u64 list_w[kList];
    u64 seg[kSegs], warp_mass[kWarps], total[3][kMaxCluster], found_mass;
    uint32_t warp_count[kWarps], found_count, found_bin, range_lo, range_hi, listed;
    int id;
    // what the first CTA found in a list: the border, and the sum up to it
    float logit;
    int last;
    u64 upto;
    float floors[2];
};

template <typename T> constexpr int kChunk = 16 / sizeof(T);  // logits of a load

template <typename T> struct Sampler {
    const SampleParams &p;
    Shared &s;
    cg::cluster_group cluster;
    const T *z;               // the row from the 16-byte boundary before it on: token i is at position i + head
    int head;
    Slope slope;
    float floor;              // the lowest logit that sums and counts take
    int rank, ranks, lo, hi;  // this CTA's positions, from whole loads on; what is called id below is a position too
    int listed;               // tokens in the list

    // kChunk logits from id i on, as they lie in memory; NaN from `end` on.
    __device__ __forceinline__ uint4 fetch(int i, int end) const
    {
        return i >= head && i + kChunk<T> <= end ? __ldg(reinterpret_cast<const uint4 *>(z + i)) : fetch_apart(z, i, end, head);
    }
    static __device__ __noinline__ uint4 fetch_apart(const T *z, int i, int end, int head)
    {
        uint4 u;
        T v[kChunk<T>];
#pragma unroll
        for (int j = 0; j < kChunk<T>; ++j) v[j] = i + j >= head && i + j < end ? z[i + j] : from_f32<T>(NAN);
        memcpy(&u, v, sizeof(u));
        return u;
    }
    // As FP32, clipped.
    static __device__ __forceinline__ void spread(const uint4 &u, float (&v)[kChunk<T>])
    {
        if constexpr (sizeof(T) == 4) {
            v[0] = __uint_as_float(u.x), v[1] = __uint_as_float(u.y), v[2] = __uint_as_float(u.z), v[3] = __uint_as_float(u.w);
        } else {
            unpack8(u, v, T());
        }
#pragma unroll
        for (int j = 0; j < kChunk<T>; ++j) v[j] = clip(v[j]);
    }
    __device__ __forceinline__ void load(int i, int end, float (&v)[kChunk<T>]) const { spread(fetch(i, end), v); }
    // f(values, id of the first) of kChunk logits a load, `step` loads apart, the
    // next load ahead.
    template <typename F> __device__ __forceinline__ void loads(int begin, int end, int step, F f) const
    {
        if (begin >= end) return;
        uint4 next = fetch(begin, end);
#pragma unroll 1
        for (int i = begin; i < end; i += step * kChunk<T>) {
            const uint4 now = next;
            if (i + step * kChunk<T> < end) next = fetch(i + step * kChunk<T>, end);
            float v[kChunk<T>];
            spread(now, v);
            f(v, i);
        }
    }
    template <typename F> __device__ __forceinline__ void each(F f) const  // f(z, id) of this CTA's
    {
        loads(lo + threadIdx.x * kChunk<T>, hi, kThreads, [&](const float (&v)[kChunk<T>], int i) {
#pragma unroll
            for (int j = 0; j < kChunk<T>; ++j) f(v[j], i + j);
        });
    }
    // f(z, id, w) of what the sums take: of the list, or of this CTA's part of the row.
    template <bool kOfList, typename F> __device__ __forceinline__ void each_weight(F f) const
    {
        if constexpr (kOfList) {
            for (int i = threadIdx.x; i < listed; i += kThreads) f(s.list_z[i], s.list_id[i], s.list_w[i]);
        } else {
            loads(lo + threadIdx.x * kChunk<T>, hi, kThreads, [&](const float (&v)[kChunk<T>], int i) {
#pragma unroll
                for (int j = 0; j < kChunk<T>; j += 2) {
                    const bool in0 = v[j] >= floor, in1 = v[j + 1] >= floor;
                    u64 w0, w1;
                    weights_of(slope, v[j], v[j + 1], in0, in1, s.powers, w0, w1);
                    if (in0) f(v[j], i + j, w0);
                    if (in1) f(v[j + 1], i + j + 1, w1);
                }
            });
        }
    }
    // All CTAs of the row.
    __device__ __forceinline__ void all_meet() const
    {
        if (ranks > 1) cluster.sync();
        else __syncthreads();
    }
    template <bool kOfList> __device__ __forceinline__ void meet() const
    {
        if constexpr (kOfList) __syncthreads();
        else all_meet();
    }
    __device__ __forceinline__ void clear() const
    {
        for (int b = threadIdx.x; b < kBins; b += kThreads) s.mass_lo[b] = 0, s.mass_hi[b] = 0, s.count[b] = 0;
        __syncthreads();
    }
    __device__ __forceinline__ void add_mass(int bin, u64 w) const
    {
        const uint32_t low = (uint32_t)w, old = atomicAdd(&s.mass_lo[bin], low), high = (uint32_t)(w >> 32) + (old > ~low);
        if (high) atomicAdd(&s.mass_hi[bin], high);
    }
    __device__ __forceinline__ void add(int bin, u64 w) const
    {
        atomicAdd(&s.count[bin], 1u);
        add_mass(bin, w);
    }
    __device__ __forceinline__ u64 mass_at(int b) const { return ((u64)s.mass_hi[b] << 32) + s.mass_lo[b]; }
    // The histogram of all CTAs in place of each one's.
    template <bool kOfList> __device__ void merge() const
    {
        meet<kOfList>();
        if (kOfList || ranks == 1) return;
        constexpr int kPer = kBins / kThreads;
        u64 m[kPer];
        uint32_t c[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) m[j] = 0, c[j] = 0;
        for (int r = 0; r < ranks; ++r) {
            const uint32_t *hi32 = cluster.map_shared_rank(s.mass_hi, r), *lo32 = cluster.map_shared_rank(s.mass_lo, r), *n = cluster.map_shared_rank(s.count, r);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const int b = threadIdx.x + j * kThreads;
                m[j] += ((u64)hi32[b] << 32) + lo32[b];
                c[j] += n[b];
            }
        }
        cluster.sync();
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int b = threadIdx.x + j * kThreads;
            s.mass_lo[b] = (uint32_t)m[j], s.mass_hi[b] = (uint32_t)(m[j] >> 32), s.count[b] = c[j];
        }
        __syncthreads();
    }

    // In kBins bins with mass(b) and count(b), the first whose running count (or
    // mass) reaches `want`: its number, and what comes before it.  false: none.
    template <typename M, typename C>
    __device__ bool crossing(M mass_of, C count_of, bool by_mass, u64 want, uint32_t &bin, u64 &before_mass, uint32_t &before_count) const
    {
        constexpr int kPer = kBins / kThreads;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        u64 m[kPer], mass = 0;
        uint32_t c[kPer], count = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            m[j] = mass_of(threadIdx.x * kPer + j);
            c[j] = count_of(threadIdx.x * kPer + j);
            mass += m[j], count += c[j];
        }
        u64 im = mass;
        uint32_t ic = count;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const u64 om = __shfl_up_sync(~0u, im, off);
            const uint32_t oc = __shfl_up_sync(~0u, ic, off);
            if (lane >= off) im += om, ic += oc;
        }
        if (lane == 31) s.warp_mass[warp] = im, s.warp_count[warp] = ic;
        if (threadIdx.x == 0) s.found_bin = ~0u;
        __syncthreads();
        u64 bm = im - mass;
        uint32_t bc = ic - count;
        for (int w = 0; w < warp; ++w) bm += s.warp_mass[w], bc += s.warp_count[w];
        if ((by_mass ? bm : bc) < want && (by_mass ? bm + mass : bc + count) >= want) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const u64 b0 = by_mass ? bm : bc, b1 = by_mass ? bm + m[j] : bc + c[j];
                if (b0 < want && b1 >= want) {
                    s.found_bin = threadIdx.x * kPer + j;
                    s.found_mass = bm;
                    s.found_count = bc;
                }
                bm += m[j];
                bc += c[j];
            }
        }
        __syncthreads();
        bin = s.found_bin;
        before_mass = s.found_mass;
        before_count = s.found_count;
        __syncthreads();
        return bin != ~0u;
    }
    // The bin of a histogram over x; the same number as it is compared with.
    __device__ __forceinline__ float place_of(float v) const { return __fmul_rn(x_near(slope, v), slope.bins); }

    // The histogram over x, into mass_x and count_x (counts only where they are wanted); the sum of all.
    __device__ u64 over_x(bool counts) const
    {
        clear();
        loads(lo + threadIdx.x * kChunk<T>, hi, kThreads, [&](const float (&v)[kChunk<T>], int) {
            constexpr int kN = kChunk<T>;
            u64 w[kN];
            uint32_t old[kN];
            int b[kN];
#pragma unroll
            for (int j = 0; j < kN; j += 2) {
                weights_of(slope, v[j], v[j + 1], v[j] >= floor, v[j + 1] >= floor, s.powers, w[j], w[j + 1]);
                b[j] = w[j] ? (int)place_of(v[j]) : 0;
                b[j + 1] = w[j + 1] ? (int)place_of(v[j + 1]) : 0;
            }
            // (one after another, each waiting for its carry, they took twice as long)
#pragma unroll
            for (int j = 0; j < kN; ++j) old[j] = w[j] ? atomicAdd(&s.mass_lo[b[j]], (uint32_t)w[j]) : 0;
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                const uint32_t high = (uint32_t)(w[j] >> 32) + (old[j] > ~(uint32_t)w[j]);
                if (high) atomicAdd(&s.mass_hi[b[j]], high);
                if (counts && w[j]) atomicAdd(&s.count[b[j]], 1u);
            }
        });
        all_meet();
        // each CTA adds up its share of the bins (every CTA all of them: 6 us)
        const int share_bins = kBins / ranks, first = rank * share_bins;
        u64 sum = 0, n = 0;
        for (int b = first + threadIdx.x; b < first + share_bins; b += kThreads) {
            u64 m = 0;
            uint32_t c = 0;
            for (int r = 0; r < ranks; ++r) {
                const Shared *o = cluster.map_shared_rank(&s, r);
                m += ((u64)o->mass_hi[b] << 32) + o->mass_lo[b];
                if (counts) c += o->count[b];
            }
            s.mass_x[b] = m;
            s.count_x[b] = c;
            sum += m;
            n += c;
        }
        sum = cta_sum(sum);
        n = cta_sum(n);
        if ((int)threadIdx.x < ranks) {
            Shared *o = cluster.map_shared_rank(&s, threadIdx.x);
            o->mass_of[rank] = sum;
            o->count_of[rank] = n;
        }
        all_meet();
        sum = 0;
        for (int r = 0; r < ranks; ++r) sum += s.mass_of[r];
        return sum;
    }
    // The bin over x where the running count (or sum) reaches `want`, and what
    // comes before it; found by the CTA that has it.  false: none does.
    __device__ bool crossing_x(bool by_mass, u64 want, uint32_t &bin, u64 &mass, uint32_t &count) const
    {
        u64 m = 0, c = 0;
        int r = 0;
        for (; r < ranks && (by_mass ? m + s.mass_of[r] : c + s.count_of[r]) < want; ++r) m += s.mass_of[r], c += s.count_of[r];
        if (r == ranks) return false;
        if (r == rank) {
            const int share_bins = kBins / ranks, first = rank * share_bins;
            auto mine = [&](int b) { return b >= first && b < first + share_bins; };
            crossing([&](int b) { return mine(b) ? s.mass_x[b] : 0ull; }, [&](int b) { return mine(b) ? s.count_x[b] : 0u; }, by_mass, want - (by_mass ? m : c), bin, mass, count);
            if ((int)threadIdx.x < ranks) {
                Shared *o = cluster.map_shared_rank(&s, threadIdx.x);
                o->border_bin = bin;
                o->border_mass = mass + m;
                o->border_count = count + (uint32_t)c;
            }
        }
        all_meet();
        bin = s.border_bin;
        mass = s.border_mass;
        count = s.border_count;
        return true;
    }

    // The logit at which the running count (or sum) reaches `want`, after what
    // comes before (mass, count), among those of bin `bin` over x (of a list:
    // among all): how many of that logit are wanted, and the sum up to them.
    template <bool kOfList> __device__ void border(bool by_mass, u64 want, uint32_t bin, u64 mass, uint32_t count, float &logit, u64 &ties, u64 &upto) const
    {
        // the logits' range
        if (threadIdx.x == 0) s.range_lo = ~0u, s.range_hi = 0;
        __syncthreads();
        uint32_t klo = ~0u, khi = 0;
        auto take = [&](float v) { klo = min(klo, key_of(v)), khi = max(khi, key_of(v)); };
        if constexpr (kOfList) {
            each_weight<true>([&](float v, int, u64) { take(v); });
        } else {
            each([&](float v, int) {
                if (v >= floor && (uint32_t)place_of(v) == bin) take(v);
            });
        }
        klo = __reduce_min_sync(~0u, klo);
        khi = __reduce_max_sync(~0u, khi);
        if ((threadIdx.x & 31) == 0) atomicMin(&s.range_lo, klo), atomicMax(&s.range_hi, khi);
        meet<kOfList>();
        klo = s.range_lo, khi = s.range_hi;
        if (!kOfList)
            for (int r = 0; r < ranks; ++r) {
                klo = min(klo, *cluster.map_shared_rank(&s.range_lo, r));
                khi = max(khi, *cluster.map_shared_rank(&s.range_hi, r));
            }
        uint32_t width = khi - klo;  // keys khi - width .. khi
        while (width > 0) {
            const int sh = max(0, 21 - __clz(width));  // width >> sh < kBins
            clear();
            auto bin_it = [&](float v, u64 w) {
                const uint32_t k = key_of(v);
                if (k <= khi && khi - k <= width) add((khi - k) >> sh, w);
            };
            if constexpr (kOfList) {
                each_weight<true>([&](float v, int, u64 w) { bin_it(v, w); });
            } else {
                const float least = logit_of(khi - width), most = logit_of(khi);
                each([&](float v, int) {
                    if (v >= least && v <= most && v >= floor) bin_it(v, weight_of(slope, v, s.powers));
                });
            }
            merge<kOfList>();
            u64 bm;
            uint32_t bc, b;
            crossing([&](int i) { return mass_at(i); }, [&](int i) { return s.count[i]; }, by_mass, want - (by_mass ? mass : count), b, bm, bc);
            mass += bm;
            count += bc;
            khi -= b << sh;
            width = min(width - (b << sh), (1u << sh) - 1);
        }
        meet<kOfList>();  // before another search sets the range
        logit = logit_of(khi);
        const u64 w = weight_of(slope, logit, s.powers);
        ties = by_mass ? (want - mass + w - 1) / w : want - count;
        upto = mass + ties * w;
    }

    // The id in the list at which the running sum of f(z, id, w), by id, passes `want`.
    template <typename F> __device__ int locate_in_list(F f, u64 want) const
    {
        u64 bm;
        uint32_t high, low, bc;
        auto mass = [&](int i) { return mass_at(i); };
        auto count = [&](int) { return 0u; };
        clear();
        each_weight<true>([&](float v, int i, u64 w) {
            w = f(v, i, w);
            if (w) add_mass((i - head) >> 10, w);
        });
        __syncthreads();
        ++want;
        if (!crossing(mass, count, true, want, high, bm, bc)) return -1;
        want -= bm;
        clear();
        each_weight<true>([&](float v, int i, u64 w) {
            w = (uint32_t)((i - head) >> 10) == high ? f(v, i, w) : 0;
            if (w) add_mass((i - head) & 1023, w);
        });
        __syncthreads();
        crossing(mass, count, true, want, low, bm, bc);
        return (int)(high << 10 | low) + head;
    }

    // Runs of ids: a warp's, kSegs of a CTA, of whole loads.
    __device__ __forceinline__ int run_length() const
    {
        constexpr int kStep = 32 * kChunk<T>;
        return ((hi - lo + kSegs - 1) / kSegs + kStep - 1) / kStep * kStep;
    }
    // Their sums of f(values, id of the first), into s.seg; a warp's runs lie one
    // after another, the next load ahead across them.
    template <typename F> __device__ __forceinline__ void sum_runs(F f) const
    {
        constexpr int kStep = 32 * kChunk<T>, kRuns = kSegs / kWarps;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, seg = run_length();
        const int begin = lo + warp * kRuns * seg, finish = min(hi, begin + kRuns * seg);
        int g = warp * kRuns, left = seg;
        u64 sum = 0;
        uint4 next = make_uint4(0, 0, 0, 0);
        if (begin < finish) next = fetch(begin + lane * kChunk<T>, hi);
#pragma unroll 1
        for (int i = begin; i < finish; i += kStep) {
            const uint4 now = next;
            if (i + kStep < finish) next = fetch(i + kStep + lane * kChunk<T>, hi);
            float v[kChunk<T>];
            spread(now, v);
            sum += f(v, i + lane * kChunk<T>);
            left -= kStep;
            if (left == 0 || i + kStep >= finish) {
                sum = warp_sum(sum);
                if (lane == 0) s.seg[g] = sum;
                ++g;
                sum = 0;
                left = seg;
            }
        }
        for (g += lane; g < (warp + 1) * kRuns; g += 32) s.seg[g] = 0;
        __syncthreads();
    }
    // The runs' sums of r of the tokens from `above` on, the ones below `least` left
    // out; those from `from` on and below `above` go into the list.  Where a fifth
    // of the tokens is from `from` on, nearly every warp's load has one: they are
    // packed together in a queue of the warp's before r is evaluated, 64 at a time.
    __device__ __forceinline__ void sum_runs_above(float from, float above, float least) const
    {
        constexpr int kStep = 32 * kChunk<T>, kRuns = kSegs / kWarps;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, seg = run_length();
        const int begin = lo + warp * kRuns * seg, finish = min(hi, begin + kRuns * seg);
        float *q_z = (float *)(s.mass_lo + warp * (kBins / kWarps));  // (the histogram's place: 128 of each)
        int *q_id = (int *)(s.mass_hi + warp * (kBins / kWarps)), queued = 0;
        int g = warp * kRuns, left = seg;
        u64 sum = 0;
        auto evaluate = [&](int n) {  // of the queue's first n <= 64
            __syncwarp();
            u64 w[2];
            const float z0 = q_z[lane], z1 = q_z[lane + 32];
            weights_of(slope, z0, z1, lane < n, lane + 32 < n, s.powers, w[0], w[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float z = k ? z1 : z0;
                if (lane + 32 * k >= n) continue;
                if (z < above) list(z, q_id[lane + 32 * k], w[k]);
                else if (z >= least) sum += w[k];
            }
            __syncwarp();
        };
        uint4 next = make_uint4(0, 0, 0, 0);
        if (begin < finish) next = fetch(begin + lane * kChunk<T>, hi);
#pragma unroll 1
        for (int i = begin; i < finish; i += kStep) {
            const uint4 now = next;
            if (i + kStep < finish) next = fetch(i + kStep + lane * kChunk<T>, hi);
            float v[kChunk<T>];
            spread(now, v);
#pragma unroll
            for (int j = 0; j < kChunk<T>; ++j) {
                const uint32_t in = __ballot_sync(~0u, v[j] >= from);
                if (v[j] >= from) {
                    const int at = queued + __popc(in & ((1u << lane) - 1));
                    q_z[at] = v[j];
                    q_id[at] = i + lane * kChunk<T> + j;
                }
                queued += __popc(in);
                if (queued >= 64) {
                    evaluate(64);
                    queued -= 64;
                    const float z = q_z[64 + lane];
                    const int id = q_id[64 + lane];
                    if (lane < queued) q_z[lane] = z, q_id[lane] = id;
                    __syncwarp();
                }
            }
            left -= kStep;
            if (left == 0 || i + kStep >= finish) {
                evaluate(queued);
                queued = 0;
                sum = warp_sum(sum);
                if (lane == 0) s.seg[g] = sum;
                ++g;
                sum = 0;
                left = seg;
            }
        }
        for (g += lane; g < (warp + 1) * kRuns; g += 32) s.seg[g] = 0;
        __syncthreads();
    }
    // The first id whose running sum is above target(sum of all), with the runs'
    // sums in s.seg and one(z, id) of single tokens; -1 for none.  The same in
    // every CTA.
    template <typename F, typename G> __device__ int locate(F one, G target, u64 &all) const
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, seg = run_length();
        if (threadIdx.x == 0) s.id = -1;
        if (warp == 0) {
            u64 sum = 0;
            for (int g = lane; g < kSegs; g += 32) sum += s.seg[g];
            sum = warp_sum(sum);
            if (lane < ranks) cluster.map_shared_rank(s.total[0], lane)[rank] = sum;
        }
        all_meet();
        u64 before = 0;
        all = 0;
        for (int r = 0; r < ranks; ++r) {
            if (r < rank) before += s.total[0][r];
            all += s.total[0][r];
        }
        const u64 want = target(all);
        if (warp == 0 && all > 0 && before <= want && want < before + s.total[0][rank]) {
            // 32 runs at a time, then 32 tokens
            int g = 0;
            for (; g < kSegs; g += 32) {
                u64 sum = g + lane < kSegs ? s.seg[g + lane] : 0;
                for (int off = 1; off < 32; off <<= 1) {
                    const u64 o = __shfl_up_sync(~0u, sum, off);
                    if (lane >= off) sum += o;
                }
                const uint32_t past = __ballot_sync(~0u, before + sum > want);
                if (past) {
                    const int first = __ffs(past) - 1;
                    if (first > 0) before += __shfl_sync(~0u, sum, first - 1);
                    g += first;
                    break;
                }
                before += __shfl_sync(~0u, sum, 31);
            }
            // (a load of each lane, then that lane's values one after another)
            for (int i0 = lo + g * seg; i0 < hi; i0 += 32 * kChunk<T>) {
                const int i = i0 + lane * kChunk<T>;
                float v[kChunk<T>];
                u64 w[kChunk<T>], sum = 0;
                load(i, hi, v);
#pragma unroll
                for (int j = 0; j < kChunk<T>; ++j) sum += w[j] = one(v[j], i + j);
                u64 upto = sum;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const u64 o = __shfl_up_sync(~0u, upto, off);
                    if (lane >= off) upto += o;
                }
                const uint32_t past = __ballot_sync(~0u, before + upto > want);
                if (past) {
                    u64 run = before + upto - sum;
                    int id = -1;
#pragma unroll
                    for (int j = 0; j < kChunk<T>; ++j) {
                        run += w[j];
                        if (id < 0 && run > want) id = i + j;
                    }
                    id = __shfl_sync(~0u, id, __ffs(past) - 1);
                    if (lane < ranks) *cluster.map_shared_rank(&s.id, lane) = id;
                    break;
                }
                before += __shfl_sync(~0u, upto, 31);
            }
        }
        all_meet();
        const int id = s.id;
        __syncthreads();  // before the next search resets it
        return id;
    }
    // A value of each CTA to all of them, in total[slot].
    __device__ __forceinline__ void share(int slot, u64 v) const
    {
        if ((int)threadIdx.x < ranks) cluster.map_shared_rank(s.total[slot], threadIdx.x)[rank] = v;
    }
    // The sum over the CTA's threads, in every one.
    __device__ __forceinline__ u64 cta_sum(u64 v) const
    {
        v = warp_sum(v);
        if ((threadIdx.x & 31) == 0) s.warp_mass[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0;
        for (int w = 0; w < kWarps; ++w) v += s.warp_mass[w];
        __syncthreads();
        return v;
    }
    // The lists of all CTAs (their lengths in total[2]) in the first one's, if
    // they fit; in all CTAs whether they do.  The others' parts stay theirs.
    __device__ bool gather()
    {
        int n = 0;
        for (int r = 0; r < ranks; ++r) n += (int)min(s.total[2][r], (u64)kList + 1);
        if (n > kList) return false;
        if (rank == 0) {
            const int own = (int)s.total[2][0];
            for (int i = threadIdx.x + own; i < n; i += kThreads) {
                int r = 0, at = i;
                while (at >= (int)s.total[2][r]) at -= (int)s.total[2][r++];
                s.list_z[i] = cluster.map_shared_rank(s.list_z, r)[at];
                s.list_id[i] = cluster.map_shared_rank(s.list_id, r)[at];
                s.list_w[i] = cluster.map_shared_rank(s.list_w, r)[at];
            }
            listed = n;
        } else {
            listed = (int)s.total[2][rank];
        }
        __syncthreads();
        return true;
    }
    __device__ __forceinline__ void list(float v, int i, u64 w) const
    {
        const uint32_t at = atomicAdd(&s.listed, 1u);
        if (at < kList) s.list_z[at] = v, s.list_id[at] = i, s.list_w[at] = w;
    }

    __device__ void answer(int t, int id, u64 all) const
    {
        if (id < head) {  // (none: what stands for a row without a token)
            p.token[t] = -1, p.prob[t] = 0.f;
            return;
        }
        p.token[t] = id - head;
        int n;  // (r itself: of small ones the sums take few bits)
        const uint32_t w = power_of(x_of(slope, clip(to_f32<T>(z[id]))), s.powers, n);
        p.prob[t] = (float)w * __int_as_float((127 - n + kFine - 31 - slope.shift) << 23) / (float)all;
    }
    // floor(sum f) for 0 <= f < 1 (above: as the largest such), or its ceiling.
    static __device__ __forceinline__ u64 share_of(u64 sum, float f, bool up)
    {
        f = fminf(fmaxf(f, 0.f), 0x1.fffffep-1f);  // (NaN becomes 0)
        if (f == 0.f) return 0;
        int e = (int)(__float_as_uint(f) >> 23);
        u64 m = __float_as_uint(f) & 0x7fffffu;
        if (e == 0) e = 1;
        else m |= 0x800000u;
        const int down = 150 - e;  // f = m 2^-down, 24 <= down <= 149
        const unsigned __int128 v = (unsigned __int128)sum * m;
        if (down >= 128) return up && v ? 1 : 0;
        const unsigned __int128 q = v >> down;
        return (u64)q + (up && (q << down) != v);
    }

    // What stands before a token in the order of the logits: the sum, and how many.
    // (Without branches: with one for each other token 104 took 12 us.)
    __device__ __forceinline__ u64 before_in_list(float v, int id, uint32_t &place) const
    {
        u64 sum = 0;
        place = 0;
#pragma unroll 8
        for (int j = 0; j < listed; ++j) {
            const float o = s.list_z[j];
            const int i = s.list_id[j];
            const u64 w = s.list_w[j];
            const bool before = o > v || (o == v && i < id);
            sum += before ? w : 0;
            place += before;
        }
        return sum;
    }
    // The border in a short list: the last token that is kept, and the sum up to
    // it, into s; a thread a token, by comparison with each other one.
    __device__ void short_border(bool by_mass, u64 want, u64 mass, uint32_t count) const
    {
        if ((int)threadIdx.x >= listed) return;
        const float v = s.list_z[threadIdx.x];
        const int id = s.list_id[threadIdx.x];
        const u64 w = s.list_w[threadIdx.x];
        uint32_t place;
        mass += before_in_list(v, id, place);
        count += place;
        if (by_mass ? mass < want && mass + w >= want : count + 1 == want) s.logit = v, s.last = id, s.upto = mass + w;
    }
    // A row whose best top_k are in a short list, a thread a token: what is before
    // it in the order of the logits, and in that of the ids, in the same way.
    __device__ void from_short_list(int t, int top_k, float top_p, float least, float u)
    {
        const bool is = (int)threadIdx.x < listed;
        const float v = is ? s.list_z[threadIdx.x] : 0.f;
        const int id = is ? s.list_id[threadIdx.x] : 0;
        const u64 w = is ? s.list_w[threadIdx.x] : 0;
        u64 before = 0;
        uint32_t place = 0;
        if (is) before = before_in_list(v, id, place);
        __syncthreads();  // the list has been read
        bool in = is && place < (uint32_t)top_k;
        if (!(top_p >= 1.f)) {
            const u64 sum = cta_sum(in ? w : 0);
            in = in && before < max(share_of(sum, top_p, true), 1ull);
        }
        in = in && v >= least;
        if (is && !in) s.list_w[threadIdx.x] = 0;  // (read again behind the sum's barriers)
        const u64 all = cta_sum(in ? w : 0), want = share_of(all, u, false);
        u64 upto = 0;
        if (in) {
#pragma unroll 8
            for (int j = 0; j < listed; ++j) {
                const u64 o = s.list_w[j];
                upto += s.list_id[j] <= id ? o : 0;
            }
        }
        if (in && upto > want && upto - w <= want) answer(t, id, all);
    }
    // A row whose best top_k are in the list: the first CTA by itself.
    __device__ void from_list(int t, int top_k, float top_p, float least, float u)
    {
        if (listed <= kShort) {
            from_short_list(t, top_k, top_p, least, u);
            return;
        }
        u64 sum = 0, ties = ~0ull, upto;
        float logit = -INFINITY;
        int last = 0x7fffffff;
        each_weight<true>([&](float, int, u64 w) { sum += w; });
        sum = cta_sum(sum);
        if (listed > top_k) {
            border<true>(false, (u64)top_k, 0, 0, 0, logit, ties, upto);
            sum = upto;
        }
        if (!(top_p >= 1.f)) border<true>(true, max(share_of(sum, top_p, true), 1ull), 0, 0, 0, logit, ties, upto);
        if (ties != ~0ull) last = locate_in_list([&](float v, int, u64) { return (u64)(v == logit); }, ties - 1);
        auto kept = [&](float v, int i, u64 w) { return v >= least && (v > logit || (v == logit && i <= last)) ? w : 0ull; };
        sum = 0;
        each_weight<true>([&](float v, int i, u64 w) { sum += kept(v, i, w); });
        sum = cta_sum(sum);
        const int id = locate_in_list(kept, share_of(sum, u, false));
        if (threadIdx.x == 0) answer(t, id, sum);
    }

    // Any other row, by all CTAs.
    __device__ void from_row(int t, int top_k, float top_p, float least, float u)
    {
        const bool by_sum = !(top_p >= 1.f);
        float logit = -INFINITY;  // kept: above it, and of those equal to it up to id `last`
        int last = 0x7fffffff;
        bool summed = false;      // s.seg holds the kept ones' sums
        if (top_k > 0 || by_sum) {
            u64 sum = over_x(top_k > 0);
            for (int turn = 0; turn < 2; ++turn) {  // top_k's border, then top_p's
                if (turn == 0 ? top_k <= 0 : !by_sum) continue;
                const u64 want = turn == 0 ? (u64)top_k : max(share_of(sum, top_p, true), 1ull);
                uint32_t bin, count;
                u64 mass, ties, upto;
                if (!crossing_x(turn == 1, want, bin, mass, count)) continue;
                // that bin's tokens into the list; the sums of what lies above it
                if (threadIdx.x == 0) s.listed = 0;
                const int warp = threadIdx.x >> 5;
                if (warp < 2) {  // the lowest logit of the bin, and the lowest above it
                    const float to = (float)(int)(bin + 1 - warp), z = to > 0.f ? lowest(slope.top, [&](float v) { return place_of(v) < to; }) : INFINITY;
                    if ((threadIdx.x & 31) == 0) s.floors[warp] = z;
                }
                __syncthreads();
                sum_runs_above(fmaxf(s.floors[0], floor), s.floors[1], least);
                share(2, s.listed);
                all_meet();
                summed = gather();
                if (summed) {
                    if (rank == 0) {
                        if (listed <= kShort) {
                            short_border(turn == 1, want, mass, count);
                        } else {
                            border<true>(turn == 1, want, 0, mass, count, logit, ties, upto);
                            last = locate_in_list([&](float v, int, u64) { return (u64)(v == logit); }, ties - 1);
                            if (threadIdx.x == 0) s.logit = logit, s.last = last, s.upto = upto;
                        }
                        __syncthreads();
                        if (threadIdx.x > 0 && (int)threadIdx.x < ranks) {
                            Shared *o = cluster.map_shared_rank(&s, threadIdx.x);
                            o->logit = s.logit, o->last = s.last, o->upto = s.upto;
                        }
                        listed = (int)s.total[2][0];
                    }
                    all_meet();
                    logit = s.logit, last = s.last, sum = s.upto;
                } else {
                    all_meet();  // the lengths have been read
                    border<false>(turn == 1, want, bin, mass, count, logit, ties, upto);
                    sum_runs([&](const float (&v)[kChunk<T>], int) {
                        u64 n = 0;
#pragma unroll
                        for (int j = 0; j < kChunk<T>; ++j) n += v[j] == logit;
                        return n;
                    });
                    u64 all;
                    last = locate([&](float v, int) { return (u64)(v == logit); }, [&](u64) { return ties - 1; }, all);
                    sum = upto;
                }
            }
        }
        // without a border above them, what the limits leave
        const float limit = fmaxf(floor, least);
        const bool bordered = logit >= limit;
        if (!bordered) logit = below(limit), last = -1;
        auto kept = [&](float v, int i) { return v > logit || (v == logit && i <= last); };
        if (summed) {  // the border's bin, from this CTA's list
            const int seg = run_length();
            for (int i = threadIdx.x; i < listed; i += kThreads)
                if (kept(s.list_z[i], s.list_id[i])) atomicAdd(&s.seg[(s.list_id[i] - lo) / seg], s.list_w[i]);
            __syncthreads();
        } else {
            auto sums = [&](auto in) {
                sum_runs([&](const float (&v)[kChunk<T>], int i) {
                    u64 run = 0;
#pragma unroll
                    for (int j = 0; j < kChunk<T>; j += 2) {
                        u64 w0, w1;
                        weights_of(slope, v[j], v[j + 1], in(v[j], i + j), in(v[j + 1], i + j + 1), s.powers, w0, w1);
                        run += w0 + w1;
                    }
                    return run;
                });
            };
            if (bordered) sums(kept);
            else sums([&](float v, int) { return v > logit; });
        }
        u64 all;
        const int id = locate([&](float v, int i) { return kept(v, i) ? weight_of(slope, v, s.powers) : 0ull; }, [&](u64 sum) { return share_of(sum, u, false); }, all);
        if (rank == 0 && threadIdx.x == 0) answer(t, id, all);
    }
};

template <typename T> __global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleParams p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    Shared &s = *reinterpret_cast<Shared *>(smem);
    pdl_trigger();
    cluster_arrive();
    if (threadIdx.x < 256) s.powers[threadIdx.x] = g_powers.at[threadIdx.x];
    pdl_wait();
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), t = blockIdx.x / ranks;
    const T *row = (const T *)p.logits + t * p.ld;
    const int head = (int)((uintptr_t)row & 15u) / (int)sizeof(T), end = head + p.V, slice = ((end + ranks - 1) / ranks + 31) / 32 * 32;
    Sampler<T> m = {p, s, cluster, row - head, head, Slope(), -INFINITY, rank, ranks, min(end, rank * slice), min(end, (rank + 1) * slice), 0};
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

    // ---- the largest logit, and the smallest
    float mine[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, least_of = INFINITY;  // of this thread's four runs of loads (NaN is passed over)
    for (int i = m.lo + threadIdx.x * kChunk<T>; i < m.hi; i += 4 * kThreads * kChunk<T>) {
        uint4 raw[4];  // four loads at a time, past the end the first again
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = i + k * kThreads * kChunk<T>;
            raw[k] = m.fetch(at < m.hi ? at : i, m.hi);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float v[kChunk<T>];
            m.spread(raw[k], v);
            float most = v[0];
#pragma unroll
            for (int j = 0; j < kChunk<T>; ++j) {
                most = fmaxf(most, v[j]);
                least_of = fminf(least_of, v[j]);
            }
            if (i + k * kThreads * kChunk<T> < m.hi) mine[k] = fmaxf(mine[k], most);
        }
    }
    float top = fmaxf(fmaxf(mine[0], mine[1]), fmaxf(mine[2], mine[3]));
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(~0u, top, off));
        least_of = fminf(least_of, __shfl_xor_sync(~0u, least_of, off));
    }
    if (lane == 0) s.warp_mass[warp] = (u64)__float_as_uint(top) << 32 | __float_as_uint(least_of);
    __syncthreads();
    auto join = [&](u64 v) {
        top = fmaxf(top, __uint_as_float((uint32_t)(v >> 32)));
        least_of = fminf(least_of, __uint_as_float((uint32_t)v));
    };
    for (int w = 0; w < kWarps; ++w) join(s.warp_mass[w]);
    cluster_wait();  // all CTAs have started: only now may their shared memory be written to
    m.share(2, (u64)__float_as_uint(top) << 32 | __float_as_uint(least_of));  // (a place that the next to share does not use)
    m.all_meet();
    for (int r = 0; r < ranks; ++r) join(s.total[2][r]);

    const float temperature = p.temperature ? p.temperature[t] : p.temperature1, top_p = p.top_p ? p.top_p[t] : p.top_p1;
    const float min_p = p.min_p ? p.min_p[t] : p.min_p1;  // (NaN limits nothing)
    int top_k = p.top_k ? p.top_k[t] : p.top_k1;
    if (top == -INFINITY || !(temperature > 0.f) || top_k == 1) {  // nothing to draw, or no choice
        int first = 0x7fffffff;
        if (top > -INFINITY)
            m.each([&](float v, int i) {
                if (v == top) first = min(first, i);
            });
        first = (int)__reduce_min_sync(~0u, (uint32_t)first);
        if (threadIdx.x == 0) s.id = 0x7fffffff;
        __syncthreads();
        if (lane == 0) atomicMin(&s.id, first);
        __syncthreads();
        m.share(1, (u64)s.id);
        m.all_meet();
        if (rank == 0 && threadIdx.x == 0) {
            for (int r = 0; r < ranks; ++r) first = min(first, (int)s.total[1][r]);
            p.token[t] = top > -INFINITY ? first - m.head : -1;
            p.prob[t] = top > -INFINITY ? 1.f : 0.f;
        }
        return;
    }
    const float u = p.u[t];
    m.slope = slope_of(top, temperature, p.shift);
    // what is too small for the sums, and for min_p; all that is a number where
    // the smallest is not
    const float far = x_near(m.slope, least_of);
    if (warp == 0) {
        const float f0 = far < kLeast - 1.f ? -kFltMax : lowest(top, [&](float z) { return within(x_of(m.slope, z), kLeast, 0.f); });
        if (lane == 0) s.floors[0] = f0;
    } else if (warp == 1) {
        float f1 = -kFltMax;
        if (min_p >= 1.f) {
            f1 = top;
        } else if (min_p > 0x1p-40f) {  // x's own limit, in two words: as near as x is, nearer than r
            const double x = -log2((double)min_p);
            const float hi = (float)x, lo = (float)(x - hi);
            f1 = lowest(top, [&](float z) { return within(x_of(m.slope, z), hi, lo); });
        }
        if (lane == 0) s.floors[1] = f1;
    }
    m.slope.bins = (float)(kBins - 2) / fminf(fmaxf(far, 0x1p-60f), kLeast + 1.f);  // (a NaN or infinity: 41)
    if (top_k >= p.V) top_k = 0;
    __syncthreads();
    m.floor = s.floors[0];
    const float least = s.floors[1];
    if (top_k > 0 && top_k <= kWanted) {
        // ---- how far down top_k tokens reach, by the runs' largest
        m.clear();
        if (threadIdx.x == 0) s.listed = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (mine[k] >= m.floor) atomicAdd(&s.count[(int)m.place_of(mine[k])], 1u);
        m.all_meet();
        uint32_t c[kBins / kThreads] = {}, bin, bc;
        for (int r = 0; r < ranks; ++r) {
            const uint4 v = *reinterpret_cast<const uint4 *>(cluster.map_shared_rank(s.count, r) + 4 * threadIdx.x);
            c[0] += v.x, c[1] += v.y, c[2] += v.z, c[3] += v.w;
        }
        u64 bm;
        const bool some = m.crossing([&](int) { return 0ull; }, [&](int b) { return b & 2 ? (b & 1 ? c[3] : c[2]) : (b & 1 ? c[1] : c[0]); }, false, (u64)top_k, bin, bm, bc);
        // Where fewer runs than top_k show a token the row has few, or top_k is
        // more than there are runs: most show one then, and a list would not fit.
        const bool few = some || p.V <= kList || 2 * m.cta_sum(c[0] + c[1] + c[2] + c[3]) < 4ull * ranks * kThreads;
        if (few) {
            const float lim = some ? (float)(bin + 1) : INFINITY;
            // ---- their list
            m.each([&](float v, int i) {
                if (v >= m.floor && m.place_of(v) < lim) m.list(v, i, weight_of(m.slope, v, s.powers));
            });
            __syncthreads();
            m.share(2, s.listed);
            m.all_meet();
            const bool fits = m.gather();
            m.all_meet();  // the lists and their lengths have been read
            if (fits) {
                if (rank == 0) m.from_list(t, top_k, top_p, least, u);
                return;
            }
        } else {
            m.all_meet();  // the histograms have been read
        }
    }
    m.from_row(t, top_k, top_p, least, u);
    m.all_meet();  // (no CTA ends while another reads from it)
}

template <typename T> cudaError_t launch_typed(const SampleParams &p, int num_sms, cudaStream_t st)
{
    // CTAs of a row: as many as there is room for, two an SM, down to 4096 tokens each
    int ranks = 1;
    while (ranks < kMaxCluster && 2 * ranks * (long long)p.T <= 2 * num_sms && p.V >= 8192 * ranks) ranks *= 2;
    static std::atomic<int> limit[64];
    cudaError_t err = ensure_dynamic_smem(sample_kernel<T>, sizeof(Shared), limit);
    if (err != cudaSuccess) return err;
    return launch_cluster_pdl(sample_kernel<T>, ranks, dim3((unsigned)(p.T * (long long)ranks)), dim3(kThreads), sizeof(Shared), st, p);
}

}  // namespace

cudaError_t launch_sample(const pmpe_sample_desc &d, int num_sms, cudaStream_t st)
{
    SampleParams p = {d.logits, d.ld, d.u, d.temperatures, d.top_ps, d.min_ps, d.top_ks, d.temperature, d.top_p, d.min_p, d.top_k, d.T, d.V, 0, d.token, d.prob};
    // as fine as sums of V tokens below 2^63 allow; a weight's shift to the left stays below 32
    p.shift = -14;
    while (p.shift < kFine && (int64_t)d.V > ((int64_t)1 << (63 - kFine + p.shift))) ++p.shift;
    if (d.logits_type == PMPE_F32) return launch_typed<float>(p, num_sms, st);
    if (d.logits_type == PMPE_BF16) return launch_typed<bf16>(p, num_sms, st);
    return launch_typed<__half>(p, num_sms, st);
}

}  // namespace pmpe
