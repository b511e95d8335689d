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
// 2^-46 of the best: sums of integers do not depend on their order.
//
//   x = (z_max - z) log2(e) / temperature  in two words, x = k / 256 + f
//   r = 2^-x = 2^(-k / 256) (1 + q(f)),    the power from a table (Tang 1989),
//   q = 2^-f - 1 a cubic, |f| <= 2^-9:     its FP32 rounding is 2^-33 of r
//
// A cluster of CTAs takes a row, each a run of ids.  One pass finds the largest
// logit; every thread's largest, in a histogram over x, tells how far down the
// best top_k (without it: 1024) tokens reach at most, since each thread that
// shows one there holds one: k threads' tokens at most, nearly k where ids are
// random.  The second pass lists those tokens (and sums r over all where top_p
// needs that), and one CTA finishes with the list in shared memory.  Rows whose
// list would be too long, or holds less than top_p, go through the whole row
// again instead.  Rows without top_k and top_p take one pass of sums.
//
// The filters' border is found in histograms of counts and sums, first over x,
// then over the bits of z where the border lies, down to one value of z; of
// equal ones the lowest ids stay.
#include <algorithm>

#include <cooperative_groups.h>

#include "elem.cuh"

namespace pmpe {
namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;
constexpr int kSegs = 8 * kWarps;    // runs of ids whose sums a CTA keeps
constexpr int kBins = 2048;          // of a histogram
constexpr int kBinsX = kThreads;     // of one over x
constexpr float kPerX = 12.f;        // its bins for a step of one in x
constexpr float kLeast = 40.f;       // log2 of the smallest r, negated
constexpr int kFine = 46;            // bits of r behind the point
constexpr int kList = 2048;          // tokens of a list
constexpr int kWanted = 1024;        // tokens that it should reach down to
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

// What turns logits into x = (pre top - pre z) post (hi + lo).
struct Slope {
    float top, hi, lo, pre, post;
    int shift;
};
__device__ __forceinline__ Slope slope_of(float top, float temperature, int shift)
{
    Slope s = {top, 0.f, 0.f, 1.f, 1.f, shift};
    // a power of two keeps the quotient among FP32's normal numbers
    if (temperature > 0x1p90f) {
        s.pre = 0x1p-100f;
        temperature *= 0x1p-100f;
    } else if (temperature < 0x1p-90f) {
        s.post = 0x1p100f;
        temperature *= 0x1p100f;
    }
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
// r as the sums take it.
__device__ __forceinline__ u64 weight_of(const Slope &s, float z, const Power *powers)
{
    int n;
    const uint32_t w = power_of(x_of(s, z), powers, n);
    n += s.shift - (kFine - 31);
    return n <= 0 ? (u64)w << -n : (u64)(w >> n);
}
// The smallest logit with x <= (hi, lo), by 32 tries at a time; the same in every lane.
__device__ float lowest(const Slope &s, float hi, float lo)
{
    uint32_t below = key_of(-kFltMax) - 1, at = key_of(s.top);  // x is above at `below` (or that is no logit), within at `at`
    while (at - below > 1) {
        const uint32_t step = (at - below + 32) / 33, k = min(at, below + step * ((threadIdx.x & 31) + 1));
        const Ratio x = x_of(s, logit_of(k));
        const uint32_t in = __ballot_sync(~0u, (x.hi - hi) + (x.lo - lo) <= 0.f);  // (not of infinities)
        const int first = in ? __ffs(in) - 1 : 32;
        const uint32_t from = below;
        if (first < 32) at = min(at, from + step * (first + 1));
        below = min(at - 1, from + step * first);
    }
    return logit_of(at);
}

struct Shared {
    Power powers[256];
    uint32_t mass_lo[kBins], mass_hi[kBins], count[kBins];
    u64 mass_x[kBinsX];      // merged: of the histogram over x
    uint32_t count_x[kBinsX];
    float list_z[kList];
    int list_id[kList];
    u64 list_w[kList];
    u64 seg[kSegs], warp_mass[kWarps], total[3][kMaxCluster], found_mass;
    uint32_t warp_count[kWarps], found_count, found_bin, range_lo, range_hi, listed;
    int id;
};

template <typename T> constexpr int kChunk = 16 / sizeof(T);  // logits of a load

template <typename T> struct Sampler {
    const SampleParams &p;
    Shared &s;
    cg::cluster_group cluster;
    const T *z;
    bool vec;                 // whole loads: rows are aligned for them
    Slope slope;
    float floor;              // the lowest logit that the sums take
    int rank, ranks, lo, hi;  // this CTA's ids (runs begin at whole loads)
    int listed;               // tokens in the list

    // f(z, id) of this CTA's logits from `begin` to `end`, `step` loads apart; NaN where there are none.
    template <typename F> __device__ __forceinline__ void each(int begin, int end, int step, F f) const
    {
        for (int i = begin; i < end; i += step * kChunk<T>) load(i, end, f);
    }
    template <typename F> __device__ __forceinline__ void load(int i, int end, F f) const
    {
        if (vec && i + kChunk<T> <= end) {
            const uint4 u = __ldg(reinterpret_cast<const uint4 *>(z + i));
            if constexpr (sizeof(T) == 4) {
                f(__uint_as_float(u.x), i);
                f(__uint_as_float(u.y), i + 1);
                f(__uint_as_float(u.z), i + 2);
                f(__uint_as_float(u.w), i + 3);
            } else {
                float v[8];
                unpack8(u, v, T());
#pragma unroll
                for (int j = 0; j < 8; ++j) f(v[j], i + j);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kChunk<T>; ++j)
                if (i + j < end) f(to_f32<T>(z[i + j]), i + j);
        }
    }
    // f(z, id, w) of what the sums take: of the list, or of the row.
    template <bool kOfList, typename F> __device__ __forceinline__ void each_weight(F f) const
    {
        if constexpr (kOfList) {
            for (int i = threadIdx.x; i < listed; i += kThreads) f(s.list_z[i], s.list_id[i], s.list_w[i]);
        } else {
            each(lo + threadIdx.x * kChunk<T>, hi, kThreads, [&](float v, int i) {
                if (v >= floor) {
                    v = fminf(v, kFltMax);
                    f(v, i, weight_of(slope, v, s.powers));
                }
            });
        }
    }
    template <bool kOfList> __device__ __forceinline__ void meet() const
    {
        if constexpr (kOfList) __syncthreads();
        else cluster.sync();
    }
    __device__ __forceinline__ void clear() const
    {
        for (int b = threadIdx.x; b < kBins; b += kThreads) s.mass_lo[b] = 0, s.mass_hi[b] = 0, s.count[b] = 0;
        __syncthreads();
    }
    __device__ __forceinline__ void add(int bin, u64 w) const
    {
        atomicAdd(&s.count[bin], 1u);
        const uint32_t low = (uint32_t)w, old = atomicAdd(&s.mass_lo[bin], low), high = (uint32_t)(w >> 32) + (old > ~low);
        if (high) atomicAdd(&s.mass_hi[bin], high);
    }
    // The histogram of all CTAs in place of each one's, kN bins.
    template <bool kOfList, int kN> __device__ void merge() const
    {
        meet<kOfList>();
        if (kOfList || ranks == 1) return;
        constexpr int kPer = kN / kThreads;
        u64 m[kPer];
        uint32_t c[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int b = threadIdx.x + j * kThreads;
            m[j] = 0, c[j] = 0;
            for (int r = 0; r < ranks; ++r) {
                m[j] += ((u64)cluster.map_shared_rank(s.mass_hi, r)[b] << 32) + cluster.map_shared_rank(s.mass_lo, r)[b];
                c[j] += cluster.map_shared_rank(s.count, r)[b];
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

    // In kN bins with mass(b) and count(b), the first whose running count (or
    // mass) reaches `want`: its number, and what comes before it.  false: none.
    template <int kN, typename M, typename C>
    __device__ bool crossing(M mass_at, C count_at, bool by_mass, u64 want, uint32_t &bin, u64 &before_mass, uint32_t &before_count) const
    {
        constexpr int kPer = kN / kThreads;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        u64 m[kPer], mass = 0;
        uint32_t c[kPer], count = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            m[j] = mass_at(threadIdx.x * kPer + j);
            c[j] = count_at(threadIdx.x * kPer + j);
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
    __device__ __forceinline__ int bin_of(float v) const { return (int)(x_near(slope, v) * kPerX); }

    // The histogram over x, into mass_x and count_x; the sum of all.
    template <bool kOfList> __device__ u64 over_x() const
    {
        clear();
        each_weight<kOfList>([&](float v, int, u64 w) { add(bin_of(v), w); });
        merge<kOfList, kBinsX>();
        u64 sum = ((u64)s.mass_hi[threadIdx.x] << 32) + s.mass_lo[threadIdx.x];
        s.mass_x[threadIdx.x] = sum;
        s.count_x[threadIdx.x] = s.count[threadIdx.x];
        sum = warp_sum(sum);
        if ((threadIdx.x & 31) == 0) s.warp_mass[threadIdx.x >> 5] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < kWarps; ++w) sum += s.warp_mass[w];
        __syncthreads();
        return sum;
    }

    // The logit at which the running count (or sum) reaches `want`, by the
    // histogram over x: how many of that logit are wanted, and the sum up to
    // them.  false: there is less than that.
    template <bool kOfList> __device__ bool border(bool by_mass, u64 want, float &logit, u64 &ties, u64 &upto) const
    {
        uint32_t bin, count;
        u64 mass;
        if (!crossing<kBinsX>([&](int b) { return s.mass_x[b]; }, [&](int b) { return s.count_x[b]; }, by_mass, want, bin, mass, count)) return false;
        // that bin's logits, from the largest on
        if (threadIdx.x == 0) s.range_lo = ~0u, s.range_hi = 0;
        __syncthreads();
        uint32_t klo = ~0u, khi = 0;
        each_weight<kOfList>([&](float v, int, u64) {
            if ((uint32_t)bin_of(v) == bin) klo = min(klo, key_of(v)), khi = max(khi, key_of(v));
        });
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
            each_weight<kOfList>([&](float v, int, u64 w) {
                const uint32_t k = key_of(v);
                if (k <= khi && khi - k <= width) add((khi - k) >> sh, w);
            });
            merge<kOfList, kBins>();
            u64 bm;
            uint32_t bc, b;
            crossing<kBins>([&](int i) { return ((u64)s.mass_hi[i] << 32) + s.mass_lo[i]; }, [&](int i) { return s.count[i]; }, by_mass,
                            want - (by_mass ? mass : count), b, bm, bc);
            mass += bm;
            count += bc;
            khi -= b << sh;
            width = min(width - (b << sh), (1u << sh) - 1);
        }
        if (!kOfList) cluster.sync();  // before another search sets the range
        logit = logit_of(khi);
        const u64 w = weight_of(slope, logit, s.powers);
        ties = by_mass ? (want - mass + w - 1) / w : want - count;
        upto = mass + ties * w;
        return true;
    }

    // The first id whose running sum of f(z, id, w) is above target(sum of
    // all); -1 for none.  The same in every CTA.
    template <bool kOfList, typename F, typename G> __device__ int locate(F f, G target, u64 &all) const
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        if constexpr (kOfList) {
            u64 sum = 0;
            each_weight<true>([&](float v, int i, u64 w) { sum += f(v, i, w); });
            sum = warp_sum(sum);
            if (lane == 0) s.warp_mass[warp] = sum;
            __syncthreads();
            all = 0;
            for (int w = 0; w < kWarps; ++w) all += s.warp_mass[w];
            u64 want = target(all) + 1, bm;
            uint32_t high, low, bc;
            clear();
            each_weight<true>([&](float v, int i, u64 w) {
                w = f(v, i, w);
                if (w) add(i >> 10, w);
            });
            __syncthreads();
            auto mass_at = [&](int i) { return ((u64)s.mass_hi[i] << 32) + s.mass_lo[i]; };
            auto count_at = [&](int i) { return s.count[i]; };
            if (!crossing<kBins>(mass_at, count_at, true, want, high, bm, bc)) return -1;
            want -= bm;
            clear();
            each_weight<true>([&](float v, int i, u64 w) {
                w = (uint32_t)(i >> 10) == high ? f(v, i, w) : 0;
                if (w) add(i & 1023, w);
            });
            __syncthreads();
            crossing<kBins>(mass_at, count_at, true, want, low, bm, bc);
            return (int)(high << 10 | low);
        } else {
            auto taken = [&](float v, int i) {
                if (!(v >= floor)) return 0ull;
                v = fminf(v, kFltMax);
                return f(v, i, weight_of(slope, v, s.powers));
            };
            constexpr int kStep = 32 * kChunk<T>;
            const int seg = ((hi - lo + kSegs - 1) / kSegs + kStep - 1) / kStep * kStep;
            for (int g = warp; g < kSegs; g += kWarps) {
                u64 sum = 0;
                each(lo + g * seg + lane * kChunk<T>, min(hi, lo + (g + 1) * seg), 32, [&](float v, int i) { sum += taken(v, i); });
                sum = warp_sum(sum);
                if (lane == 0) s.seg[g] = sum;
            }
            if (threadIdx.x == 0) s.id = -1;
            __syncthreads();
            if (warp == 0) {
                u64 sum = 0;
                for (int g = lane; g < kSegs; g += 32) sum += s.seg[g];
                sum = warp_sum(sum);
                if (lane < ranks) cluster.map_shared_rank(s.total[0], lane)[rank] = sum;
            }
            cluster.sync();
            u64 before = 0;
            all = 0;
            for (int r = 0; r < ranks; ++r) {
                if (r < rank) before += s.total[0][r];
                all += s.total[0][r];
            }
            const u64 want = target(all);
            if (warp == 0 && all > 0 && before <= want && want < before + s.total[0][rank]) {
                int g = 0;
                while (before + s.seg[g] <= want) before += s.seg[g++];
                for (int i = lo + g * seg + lane;; i += 32) {
                    u64 sum = i < hi ? taken(to_f32<T>(z[i]), i) : 0;
                    for (int off = 1; off < 32; off <<= 1) {
                        const u64 o = __shfl_up_sync(~0u, sum, off);
                        if (lane >= off) sum += o;
                    }
                    const uint32_t past = __ballot_sync(~0u, before + sum > want);
                    if (past) {
                        if (lane < ranks) *cluster.map_shared_rank(&s.id, lane) = i - lane + __ffs(past) - 1;
                        break;
                    }
                    before += __shfl_sync(~0u, sum, 31);
                }
            }
            cluster.sync();
            const int id = s.id;
            __syncthreads();  // before the next search resets it
            return id;
        }
    }
    // Values of the CTAs (one each, from thread 0's point of view) to all of them.
    __device__ __forceinline__ void share(int slot, u64 v) const
    {
        if ((int)threadIdx.x < ranks) cluster.map_shared_rank(s.total[slot], threadIdx.x)[rank] = v;
    }
    // A warp's values' sum over the CTA, in every thread.
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

    // The filters' border and the draw.
    template <bool kOfList> __device__ void finish(int t, int top_k, float top_p, float min_p, float u)
    {
        float logit = -INFINITY;  // kept: above it, and of those equal to it up to id `last`
        u64 ties = ~0ull, all;
        int last = 0x7fffffff;
        if (top_k > 0 || !(top_p >= 1.f)) {
            u64 sum = over_x<kOfList>(), upto;
            if (top_k > 0) {
                if (border<kOfList>(false, (u64)top_k, logit, ties, upto)) sum = upto;
            } else if (kOfList) {  // the list is not all
                sum = 0;
                for (int r = 0; r < ranks; ++r) sum += s.total[1][r];
            }
            if (!(top_p >= 1.f)) border<kOfList>(true, max(share_of(sum, top_p, true), 1ull), logit, ties, upto);
        }
        // of equal logits at the border the lowest ids stay
        if (ties != ~0ull)
            last = locate<kOfList>([&](float v, int, u64) { return (u64)(v == logit); }, [&](u64) { return ties - 1; }, all);
        if (min_p > 0.f) {
            const double lim = -log2((double)min_p);
            if (lim < kLeast) floor = lowest(slope, (float)lim, (float)(lim - (float)lim));
        }
        const float least = floor;
        const int id = locate<kOfList>([&](float v, int i, u64 w) { return v >= least && (v > logit || (v == logit && i <= last)) ? w : 0ull; },
                                       [&](u64 sum) { return share_of(sum, u, false); }, all);
        if (rank == 0 && threadIdx.x == 0) {
            p.token[t] = id;
            int n;  // (r itself: of small ones the sums take few bits)
            const uint32_t w = power_of(x_of(slope, fminf(to_f32<T>(z[id]), kFltMax)), s.powers, n);
            p.prob[t] = (float)w * __int_as_float((127 - n) << 23) * (float)(1 << (kFine - 31)) / ((float)all * (float)(1 << slope.shift));
        }
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
};

template <typename T> __global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleParams p)
{
    extern __shared__ __align__(16) uint8_t smem[];
    Shared &s = *reinterpret_cast<Shared *>(smem);
    pdl_trigger();
    if (threadIdx.x < 256) s.powers[threadIdx.x] = g_powers.at[threadIdx.x];
    pdl_wait();
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), t = blockIdx.x / ranks;
    const int slice = ((p.V + ranks - 1) / ranks + 31) / 32 * 32;
    const T *row = (const T *)p.logits + t * p.ld;
    Sampler<T> m = {p, s, cluster, row, ((uintptr_t)row & 15u) == 0, Slope(), -INFINITY, rank, ranks, min(p.V, rank * slice), min(p.V, (rank + 1) * slice), 0};
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

    // ---- the largest logit
    float mine = -INFINITY;  // of this thread (NaN is passed over)
    m.each(m.lo + threadIdx.x * kChunk<T>, m.hi, kThreads, [&](float v, int) { mine = fmaxf(mine, v); });
    mine = fminf(mine, kFltMax);
    float top = mine;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, off));
    if (lane == 0) s.warp_mass[warp] = (u64)__float_as_uint(top);
    __syncthreads();
    top = __uint_as_float((uint32_t)s.warp_mass[lane < kWarps ? lane : 0]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, off));
    m.share(2, (u64)__float_as_uint(top));  // (a place of its own: no barrier stands between this and the next)
    cluster.sync();
    for (int r = 0; r < ranks; ++r) top = fmaxf(top, __uint_as_float((uint32_t)s.total[2][r]));

    const float temperature = p.temperature ? p.temperature[t] : p.temperature1, top_p = p.top_p ? p.top_p[t] : p.top_p1;
    float min_p = p.min_p ? p.min_p[t] : p.min_p1;
    if (min_p > 1.f) min_p = 1.f;  // (NaN stays, and limits nothing)
    const int top_k = p.top_k ? p.top_k[t] : p.top_k1;
    if (top == -INFINITY || !(temperature > 0.f) || top_k == 1) {  // nothing to draw, or no choice
        int first = 0x7fffffff;
        if (top > -INFINITY)
            m.each(m.lo + threadIdx.x * kChunk<T>, m.hi, kThreads, [&](float v, int i) {
                if (fminf(v, kFltMax) == top) first = min(first, i);
            });
        first = (int)__reduce_min_sync(~0u, (uint32_t)first);
        if (threadIdx.x == 0) s.id = 0x7fffffff;
        __syncthreads();
        if (lane == 0) atomicMin(&s.id, first);
        __syncthreads();
        m.share(1, (u64)s.id);
        cluster.sync();
        if (rank == 0 && threadIdx.x == 0) {
            for (int r = 0; r < ranks; ++r) first = min(first, (int)s.total[1][r]);
            p.token[t] = top > -INFINITY ? first : -1;
            p.prob[t] = top > -INFINITY ? 1.f : 0.f;
        }
        return;
    }
    m.slope = slope_of(top, temperature, p.shift);
    m.floor = lowest(m.slope, kLeast, 0.f);
    const float u = p.u[t];
    const bool by_sum = !(top_p >= 1.f);
    if (top_k <= kWanted && (top_k > 0 || by_sum)) {
        // ---- how far down the wanted tokens reach, by the threads' largest
        m.clear();
        if (threadIdx.x == 0) s.listed = 0;
        if (mine >= m.floor) atomicAdd(&s.count[m.bin_of(mine)], 1u);
        cluster.sync();
        uint32_t c = 0, bin, bc;
        for (int r = 0; r < ranks; ++r) c += cluster.map_shared_rank(s.count, r)[threadIdx.x];
        u64 bm;
        const bool whole = !m.template crossing<kBinsX>([&](int) { return 0ull; }, [&](int) { return c; }, false, (u64)(top_k > 0 ? top_k : kWanted), bin, bm, bc);
        const float lim = whole ? INFINITY : (float)(bin + 1);
        // ---- their list; r of those, and of all
        u64 in_list = 0, in_all = 0;
        m.each(m.lo + threadIdx.x * kChunk<T>, m.hi, kThreads, [&](float v, int i) {
            if (!(v >= m.floor)) return;
            v = fminf(v, kFltMax);
            const bool in = x_near(m.slope, v) * kPerX < lim;
            u64 w = 0;
            if (in || top_k <= 0) w = weight_of(m.slope, v, s.powers);
            if (in) {
                const uint32_t at = atomicAdd(&s.listed, 1u);
                if (at < kList) s.list_z[at] = v, s.list_id[at] = i, s.list_w[at] = w;
                in_list += w;
            }
            in_all += w;
        });
        in_list = m.cta_sum(in_list);
        in_all = m.cta_sum(in_all);
        m.share(0, in_list);
        m.share(1, in_all);
        m.share(2, s.listed);
        cluster.sync();
        u64 n = 0, before = 0;
        in_list = in_all = 0;
        for (int r = 0; r < ranks; ++r) in_list += s.total[0][r], in_all += s.total[1][r], n += s.total[2][r];
        if (n <= kList && (top_k > 0 || in_list >= Sampler<T>::share_of(in_all, top_p, true))) {
            // ---- the first CTA goes on by itself
            if (rank == 0) {
                before = s.total[2][0];
                for (int r = 1; r < ranks; ++r) {
                    const int part = (int)s.total[2][r];
                    for (int i = threadIdx.x; i < part; i += kThreads) {
                        s.list_z[before + i] = cluster.map_shared_rank(s.list_z, r)[i];
                        s.list_id[before + i] = cluster.map_shared_rank(s.list_id, r)[i];
                        s.list_w[before + i] = cluster.map_shared_rank(s.list_w, r)[i];
                    }
                    before += part;
                }
            }
            cluster.sync();
            if (rank != 0) return;
            m.listed = (int)n;
            m.template finish<true>(t, top_k, top_p, min_p, u);
            return;
        }
        cluster.sync();  // the totals have been read
    }
    m.template finish<false>(t, top_k, top_p, min_p, u);
    cluster.sync();  // (no CTA ends while another reads from it)
}

template <typename T> cudaError_t launch_typed(const SampleParams &p, int num_sms, cudaStream_t st)
{
    // CTAs of a row: as many as there is room for, two an SM, down to 4096 tokens each
    int ranks = 1;
    while (ranks < kMaxCluster && 2 * ranks * (long long)p.T <= 2 * num_sms && p.V >= 8192 * ranks) ranks *= 2;
    static std::atomic<int> limit[64];
    cudaError_t err = ensure_dynamic_smem(sample_kernel<T>, sizeof(Shared), limit);
    if (err == cudaSuccess && ranks > 8) err = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (err != cudaSuccess) return err;
    return launch_cluster_pdl(sample_kernel<T>, ranks, dim3((unsigned)(p.T * (long long)ranks)), dim3(kThreads), sizeof(Shared), st, p);
}

}  // namespace

cudaError_t launch_sample(const pmpe_sample_desc &d, int num_sms, cudaStream_t st)
{
    SampleParams p = {d.logits, d.ld, d.u, d.temperatures, d.top_ps, d.min_ps, d.top_ks, d.temperature, d.top_p, d.min_p, d.top_k, d.T, d.V, 0, d.token, d.prob};
    while (p.shift < kFine && (int64_t)d.V > ((int64_t)1 << (63 - kFine + p.shift))) ++p.shift;
    if (d.logits_type == PMPE_F32) return launch_typed<float>(p, num_sms, st);
    if (d.logits_type == PMPE_BF16) return launch_typed<bf16>(p, num_sms, st);
    return launch_typed<__half>(p, num_sms, st);
}

}  // namespace pmpe
