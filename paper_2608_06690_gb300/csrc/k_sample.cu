// The next token of each row of logits, from given random numbers:
//
//   r_i = e^((z_i - z_max) / temperature), down to 2^-40
//   kept: in the order (z descending, id ascending) the first top_k; of those
//         the ones with less than top_p of their sum before them; of those
//         r >= min_p -- always a prefix of that order
//   drawn: the lowest kept id whose running sum of r, by id, is above u times the sum
//
// A token is an integer, so that sums that differ in their last bits would give
// another one now and then.  Therefore r is evaluated to some 2^-33 (not FP32's
// 2^-22; FP64 has a sixty-fourth of its rate here) and held as an integer of
// 2^-46 of the best: sums of integers do not depend on their order.
//
//   x = (z_max - z) log2(e) / temperature  in two words, x = j / 256 + f
//   r = 2^-x = 2^(-j / 256) (1 + q(f)),    the power from a table (Tang 1989),
//   q = 2^-f - 1 a cubic, |f| <= 2^-9:     its FP32 rounding is 2^-33 of r
//
// A cluster of CTAs takes a row, each a run of ids, and every CTA decides the
// same from the same sums, which they read from one another's shared memory.
// The filters' border is found by histograms, first over x in eighths, then over
// the bits of z in the eighth that holds the border, down to one value of z; of
// equal ones the lowest ids stay.
#include <algorithm>

#include <cooperative_groups.h>

#include "elem.cuh"

namespace pmpe {
namespace {

namespace cg = cooperative_groups;
typedef unsigned long long u64;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kSegs = 8 * kWarps;    // runs of ids whose sums a CTA keeps
constexpr int kBins = 2048, kBins0 = kThreads;  // of a histogram; of the one over x (321 of them)
constexpr float kLeast = 40.f;       // log2 of the smallest r, negated
constexpr int kFine = 46;            // bits of r behind the point
constexpr float kLog2eHi = 1.44269502f, kLog2eLo = 1.92596303e-8f;  // log2(e) in two words
constexpr float kFltMax = 3.402823466e38f;

// 2^(-j / 256) as an integer of 2^-46, and in FP32.
struct Powers {
    u64 fixed[256];
    float value[256];
    constexpr Powers() : fixed(), value()
    {
        for (int j = 0; j < 256; ++j) {
            const double y = -j * (0.69314718055994530942 / 256);
            double term = 1, sum = 1;
            for (int n = 1; n < 30; ++n) {
                term *= y / n;
                sum += term;
            }
            fixed[j] = (u64)(sum * 70368744177664.0 + 0.5);
            value[j] = (float)sum;
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

// A logit's place among others: unsigned order is that of the values, 0 for
// what cannot be drawn; +inf counts as the largest finite one.
__device__ __forceinline__ uint32_t key_of(float z)
{
    if (!(z > -INFINITY)) return 0u;
    const uint32_t b = __float_as_uint(fminf(z, kFltMax) + 0.f);  // -0 becomes 0
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// What turns logits into x.
struct Slope {
    float top, hi, lo, pre, post;  // x = (pre top - pre z) post (hi + lo)
};
__device__ __forceinline__ Slope slope_of(float top, float temperature)
{
    Slope s = {top, 0.f, 0.f, 1.f, 1.f};
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
__device__ __forceinline__ bool within(const Ratio &x, float lim_hi, float lim_lo)  // x <= the limit
{
    return (x.hi - lim_hi) + (x.lo - lim_lo) <= 0.f;  // (false for NaN, as of two infinite words)
}

struct Row {
    Slope slope;
    float lim_hi, lim_lo;  // x of what the sums take
    int shift;
};
// r = w 2^-(46 + n) for 0 <= x <= 40.
__device__ __forceinline__ u64 power_of(const Ratio &x, const u64 *s_fixed, const float *s_value, int &n)
{
    const int k = __float2int_rn(x.hi * 256.f), j = k & 255;
    const float f = fmaf((float)k, -1.f / 256.f, x.hi) + x.lo;
    const float q = f * fmaf(f, fmaf(f, -0.055504109f, 0.240226507f), -0.693147181f);
    n = k >> 8;
    return (u64)((long long)s_fixed[j] + ((long long)__float2int_rn(s_value[j] * q * 0x1p38f) << (kFine - 38)));
}
// r as the sums take it; 0 past the row's limit.
__device__ __forceinline__ u64 weight_of(const Row &row, const Ratio &x, const u64 *s_fixed, const float *s_value)
{
    if (!within(x, row.lim_hi, row.lim_lo)) return 0;
    int n;
    const u64 w = power_of(x, s_fixed, s_value, n);
    return w >> (n + row.shift);
}

struct Shared {
    u64 fixed[256];
    float value[256];
    u64 mass[kBins];
    uint32_t count[kBins];
    u64 mass0[kBins0];       // of the histogram over x
    uint32_t count0[kBins0];
    u64 seg[kSegs], warp_mass[kWarps], total[kMaxCluster], found_mass;
    uint32_t warp_count[kWarps], found_count, found_bin, range_lo, range_hi;
    uint32_t id;
};

template <typename T> struct Sampler {
    const SampleParams &p;
    Shared &s;
    cg::cluster_group cluster;
    const T *z;
    Row row;
    int rank, ranks, lo, hi;  // this CTA's ids

    __device__ __forceinline__ float at(int i) const { return to_f32<T>(z[i]); }
    __device__ __forceinline__ u64 weight(uint32_t key) const
    {
        return weight_of(row, x_of(row.slope, logit_of(key)), s.fixed, s.value);
    }

    // The cluster's histogram of bin_of(key, bin, weight) in count and mass, kN bins.
    template <int kN, typename F> __device__ void histogram(F bin_of)
    {
        constexpr int kPerThread = kN / kThreads;
        for (int b = threadIdx.x; b < kN; b += kThreads) s.mass[b] = 0, s.count[b] = 0;
        __syncthreads();
        for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
            const uint32_t key = key_of(at(i));
            if (key == 0) continue;
            int bin;
            u64 w;
            if (!bin_of(key, bin, w)) continue;
            atomicAdd(&s.count[bin], 1u);
            atomicAdd(&s.mass[bin], w);
        }
        cluster.sync();
        u64 m[kPerThread];
        uint32_t c[kPerThread];
        for (int j = 0; j < kPerThread; ++j) {
            m[j] = 0, c[j] = 0;
            for (int r = 0; r < ranks; ++r) {
                m[j] += cluster.map_shared_rank(s.mass, r)[threadIdx.x * kPerThread + j];
                c[j] += cluster.map_shared_rank(s.count, r)[threadIdx.x * kPerThread + j];
            }
        }
        cluster.sync();
        for (int j = 0; j < kPerThread; ++j) s.mass[threadIdx.x * kPerThread + j] = m[j], s.count[threadIdx.x * kPerThread + j] = c[j];
        __syncthreads();
    }

    // In bins of masses m and counts c, the first whose running count (or mass)
    // reaches `want`: its number, and what comes before it.  false: none does.
    template <int kN> __device__ bool crossing(const u64 *m, const uint32_t *c, bool by_mass, u64 want, uint32_t &bin, u64 &before_mass, uint32_t &before_count)
    {
        constexpr int kPerThread = kN / kThreads;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        u64 mass = 0;
        uint32_t count = 0;
        for (int j = 0; j < kPerThread; ++j) mass += m[threadIdx.x * kPerThread + j], count += c[threadIdx.x * kPerThread + j];
        u64 im = mass;
        uint32_t ic = count;
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
            for (int j = 0; j < kPerThread; ++j) {
                const int b = threadIdx.x * kPerThread + j;
                if ((by_mass ? bm + m[b] : bc + c[b]) >= want) {
                    s.found_bin = b;
                    s.found_mass = bm;
                    s.found_count = bc;
                    break;
                }
                bm += m[b];
                bc += c[b];
            }
        }
        __syncthreads();
        bin = s.found_bin;
        before_mass = s.found_mass;
        before_count = s.found_count;
        __syncthreads();
        return bin != ~0u;
    }

    // The key at which the running count (or mass) reaches `want`, from the
    // first histogram in mass0 and count0: the key, how many of that key are
    // wanted, and the mass up to them.  false: there is less than that.
    __device__ bool border(bool by_mass, u64 want, uint32_t &key, u64 &ties, u64 &upto)
    {
        uint32_t bin, count;
        u64 mass;
        if (!crossing<kBins0>(s.mass0, s.count0, by_mass, want, bin, mass, count)) return false;
        // the keys of that eighth, from the largest on
        if (threadIdx.x == 0) s.range_lo = ~0u, s.range_hi = 0;
        __syncthreads();
        uint32_t klo = ~0u, khi = 0;
        for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
            const uint32_t k = key_of(at(i));
            if (k == 0) continue;
            const Ratio x = x_of(row.slope, logit_of(k));
            if (within(x, row.lim_hi, row.lim_lo) && (uint32_t)eighth(x) == bin) klo = min(klo, k), khi = max(khi, k);
        }
        klo = __reduce_min_sync(~0u, klo);
        khi = __reduce_max_sync(~0u, khi);
        if ((threadIdx.x & 31) == 0) atomicMin(&s.range_lo, klo), atomicMax(&s.range_hi, khi);
        cluster.sync();
        for (int r = 0; r < ranks; ++r) {
            klo = min(klo, *cluster.map_shared_rank(&s.range_lo, r));
            khi = max(khi, *cluster.map_shared_rank(&s.range_hi, r));
        }
        uint32_t width = khi - klo;  // keys khi - width .. khi
        for (;;) {
            const int sh = max(0, 21 - __clz(width | 1u));  // width >> sh < kBins
            histogram<kBins>([&](uint32_t k, int &b, u64 &w) {
                if (k > khi || khi - k > width) return false;
                b = (int)((khi - k) >> sh);
                w = weight(k);
                return w > 0;
            });
            u64 bm;
            uint32_t bc, b;
            crossing<kBins>(s.mass, s.count, by_mass, want - (by_mass ? mass : count), b, bm, bc);
            mass += bm;
            count += bc;
            khi -= b << sh;
            if (sh == 0) break;
            width = min(width - (b << sh), (1u << sh) - 1);
        }
        key = khi;
        const u64 w = weight(key);
        ties = by_mass ? (want - mass + w - 1) / w : want - count;
        upto = mass + ties * w;
        return true;
    }
    static __device__ __forceinline__ int eighth(const Ratio &x) { return (int)(x.hi * 8.f); }

    // The first id whose running sum of f(key, id) is above target(sum of all);
    // ~0 for none.  The same in every CTA.
    template <typename F, typename G> __device__ uint32_t locate(F f, G target, u64 &all)
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        const int seg = ((hi - lo + kSegs - 1) / kSegs + 31) / 32 * 32;
        for (int g = warp; g < kSegs; g += kWarps) {
            u64 sum = 0;
            const int end = min(hi, lo + (g + 1) * seg);
            for (int i = lo + g * seg + lane; i < end; i += 32) {
                const uint32_t k = key_of(at(i));
                if (k) sum += f(k, i);
            }
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(~0u, sum, off);
            if (lane == 0) s.seg[g] = sum;
        }
        if (threadIdx.x == 0) s.id = ~0u;
        __syncthreads();
        if (warp == 0) {
            u64 sum = 0;
            for (int g = lane; g < kSegs; g += 32) sum += s.seg[g];
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(~0u, sum, off);
            if (lane < ranks) cluster.map_shared_rank(s.total, lane)[rank] = sum;
        }
        cluster.sync();
        u64 before = 0;
        all = 0;
        for (int r = 0; r < ranks; ++r) {
            if (r < rank) before += s.total[r];
            all += s.total[r];
        }
        const u64 want = target(all);
        if (warp == 0 && all > 0 && before <= want && want < before + s.total[rank]) {
            int g = 0;
            while (before + s.seg[g] <= want) before += s.seg[g++];
            for (int i = lo + g * seg + lane;; i += 32) {
                const uint32_t k = i < hi ? key_of(at(i)) : 0u;
                u64 sum = k ? f(k, i) : 0;
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
        const uint32_t id = s.id;
        __syncthreads();  // before the next search resets it
        return id;
    }
};

// floor(sum f), for 0 <= f < 1 (above: as the largest such), and its ceiling.
__device__ __forceinline__ u64 share(u64 sum, float f, bool up)
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

template <typename T> __global__ void __launch_bounds__(kThreads) sample_kernel(const __grid_constant__ SampleParams p)
{
    __shared__ Shared s;
    pdl_trigger();
    for (int j = threadIdx.x; j < 256; j += kThreads) s.fixed[j] = g_powers.fixed[j], s.value[j] = g_powers.value[j];
    pdl_wait();
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), t = blockIdx.x / ranks;
    const int slice = ((p.V + ranks - 1) / ranks + 31) / 32 * 32;
    Sampler<T> m = {p, s, cluster, (const T *)p.logits + t * p.ld, Row(), rank, ranks, min(p.V, rank * slice), min(p.V, (rank + 1) * slice)};
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

    // ---- the best token, the lowest id of equal ones
    u64 best = 0;
    for (int i = m.lo + threadIdx.x; i < m.hi; i += kThreads) {
        const uint32_t k = key_of(m.at(i));
        if (k) best = max(best, (u64)k << 32 | ~(uint32_t)i);
    }
    for (int off = 16; off > 0; off >>= 1) best = max(best, __shfl_xor_sync(~0u, best, off));
    if (lane == 0) s.warp_mass[warp] = best;
    __syncthreads();
    if (warp == 0) {
        best = lane < kWarps ? s.warp_mass[lane] : 0;
        for (int off = 16; off > 0; off >>= 1) best = max(best, __shfl_xor_sync(~0u, best, off));
        if (lane < ranks) cluster.map_shared_rank(s.total, lane)[rank] = best;
    }
    cluster.sync();
    best = 0;
    for (int r = 0; r < ranks; ++r) best = max(best, s.total[r]);
    cluster.sync();

    const float temperature = p.temperature ? p.temperature[t] : p.temperature1, top_p = p.top_p ? p.top_p[t] : p.top_p1;
    float min_p = p.min_p ? p.min_p[t] : p.min_p1;
    if (min_p > 1.f) min_p = 1.f;  // (NaN stays, and limits nothing)
    const int top_k = p.top_k ? p.top_k[t] : p.top_k1;
    if (best == 0 || !(temperature > 0.f) || top_k == 1) {  // nothing to draw, or no choice
        if (rank == 0 && threadIdx.x == 0) {
            p.token[t] = best ? (int32_t)~(uint32_t)best : -1;
            p.prob[t] = best ? 1.f : 0.f;
        }
        return;
    }
    m.row = {slope_of(logit_of((uint32_t)(best >> 32)), temperature), kLeast, 0.f, p.shift};

    // ---- the filters' border: keys above `key`, and of those equal to it the first `ties`
    uint32_t key = 0;
    u64 ties = ~0ull, upto;
    if (top_k > 0 || top_p < 1.f || top_p != top_p) {
        m.template histogram<kBins0>([&](uint32_t k, int &b, u64 &w) {
            const Ratio x = x_of(m.row.slope, logit_of(k));
            w = weight_of(m.row, x, s.fixed, s.value);
            b = Sampler<T>::eighth(x);
            return w > 0;
        });
        u64 sum = 0;
        s.mass0[threadIdx.x] = sum = s.mass[threadIdx.x];
        s.count0[threadIdx.x] = s.count[threadIdx.x];
        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(~0u, sum, off);
        if (lane == 0) s.warp_mass[warp] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < kWarps; ++w) sum += s.warp_mass[w];
        __syncthreads();
        if (top_k > 0 && m.border(false, (u64)top_k, key, ties, upto)) sum = upto;
        if (!(top_p >= 1.f)) m.border(true, max(share(sum, top_p, true), 1ull), key, ties, upto);
    }
    // of equal logits at the border the lowest ids stay
    uint32_t last = ~0u;
    u64 all;
    if (key && ties != ~0ull) {
        last = m.locate([&](uint32_t k, int) { return (u64)(k == key); }, [&](u64) { return ties - 1; }, all);
    }
    if (min_p > 0.f) {
        const double lim = -log2((double)min_p);
        if (lim < kLeast) {
            m.row.lim_hi = (float)lim;
            m.row.lim_lo = (float)(lim - m.row.lim_hi);
        }
    }

    // ---- the draw
    const float u = p.u[t];
    const uint32_t id = m.locate([&](uint32_t k, int i) { return k > key || (k == key && (uint32_t)i <= last) ? m.weight(k) : 0ull; },
                                 [&](u64 sum) { return share(sum, u, false); }, all);
    if (rank == 0 && threadIdx.x == 0) {
        p.token[t] = (int32_t)id;
        int n;  // (r itself: of small ones the sums take few bits)
        const u64 w = power_of(x_of(m.row.slope, logit_of(key_of(m.at((int)id)))), s.fixed, s.value, n);
        p.prob[t] = (float)w * __int_as_float((127 - n) << 23) / ((float)all * (float)(1 << m.row.shift));
    }
}

template <typename T> cudaError_t launch_typed(const SampleParams &p, int num_sms, cudaStream_t st)
{
    // CTAs of a row: as many as there are SMs for, down to 4096 tokens each
    int ranks = 1;
    while (ranks < kMaxCluster && 2 * ranks * (long long)p.T <= num_sms && p.V >= 8192 * ranks) ranks *= 2;
    return launch_cluster_pdl(sample_kernel<T>, ranks, dim3((unsigned)(p.T * (long long)ranks)), dim3(kThreads), 0, st, p);
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
