// Routing from given logits: scores (softmax or sigmoid), a balance bias,
// group limits, top-k, renormalised weights, each token inside the pool its
// policy byte selects (Sec. 3.1, Eq. 4: an expert outside that pool never
// enters the candidate set), and the gradient of the logits.
//
//   eligible(e) = e in the token's pool and z_e > -inf (NaN is not)
//   score_e     = exp(z_e) / sum_eligible exp(z)     or   1 / (1 + exp(-z_e))
//   choice_e    = score_e + bias_e, or z_e without a bias (score_e grows with it)
//   a group counts its best choice, or the sum of its two best score + bias;
//   only the best groups' experts stay candidates
//   the k largest choices, ties to the lower id; w_j = scale score_j, over the
//   sum of the k scores when renormalised; -1 with weight 0 where fewer than
//   k experts are eligible
//
// A warp takes a token: lane l holds kV consecutive experts of the pool, so a
// row is read once with one vector load a lane.  A lane orders its experts
// once; each of the k rounds is then one redux over packed words (24 bits of
// the choice, 8 of the expert) and a shift in the winner's lane.
//
// The selection is that of choices in 64 bits.  Where two neighbours in the
// order have equal packed words, the warp selects again by the whole choices
// (about one token in a hundred with FP32 logits).  Without a bias choices are
// logits, which compare exactly; with one they are FP32, a few 2^-24 off: where
// neighbours (or two groups at the limit) lie within the bound of that error,
// the token is put aside, and the CTA selects its experts at the end by 64-bit
// choices, an expert a thread, compared as integers: 3.8 us a token (softmax
// 8), where one warp alone took 11, as an FP64 instruction occupies a scheduler
// for some 60 clocks.  Equal 64-bit choices go by the lower id.
//
// The bound is one for all choices of a row, so how many tokens it leaves open
// goes by the data (256 experts, top 8, normal logits).  With biases of 0.05:
// 0.1 to 0.3 % at standard deviations of 1.5 to 8 (top 12: 0.2 to 9 %), and
// T = 8192 takes 14 to 20 us.  With biases of zero, where small scores lie
// close together: 0.1 % at 1.5 and 2 % at 3 (15 to 24 us), sigmoid 68 % at 5
// (136 us) and all at 8 or around a mean of -15 (180 us), softmax 4 % at 5 (38)
// and 23 % at 8 (92).  The groups' bound goes by the largest choice of the
// pool: a finite mask of one bias in sixteen, 8192 tokens, 4 of 8 groups: none
// 18 us, -100 0.4 % (25 us), -1e4 27 % (114), -1e9 all (252), -inf none (18).
#include <algorithm>
#include <type_traits>

#include "elem.cuh"

namespace pmpe {
namespace {

constexpr int kRouteWarps = 8;

struct ScoreParams {
    const void *logits;
    const uint8_t *policy;
    const float *bias;
    int32_t *idx;
    float *w;
    int32_t *load;
    long long ld;
    int T, E_pub, E_priv, k, renorm, sigmoid, top2;
    int groups[2], top_groups[2];  // public, private
    int tokens;                    // of a CTA at most
    float scale;
};

// Unsigned keys in the order of the floats; 0 is below every float, and -0 and
// +0 are one key.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

constexpr float kNone = -INFINITY;
constexpr float kLargest = 3.402823466e38f;  // stands for a logit of +inf

// The same for 64-bit values, compared as integers: FP64 compares are as slow
// as its arithmetic.
typedef unsigned long long u64;
__device__ __forceinline__ u64 key64(double x)
{
    const long long u = __double_as_longlong(x);
    return (u64)u ^ ((u64)(u >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double of(u64 key)
{
    return __longlong_as_double((long long)(key >> 63 ? key ^ 0x8000000000000000ull : ~key));
}
__device__ __forceinline__ u64 warp_max64(u64 v)
{
    const uint32_t hi = (uint32_t)(v >> 32), top = __reduce_max_sync(~0u, hi);
    return (u64)top << 32 | __reduce_max_sync(~0u, hi == top ? (uint32_t)v : 0u);
}

// A token's pool: what its selection goes by.
template <typename T> struct Pool {
    const T *row;       // the pool's logits
    const float *bias;  // and biases, or null
    int E, sigmoid, n, top, top2, k;
};

template <typename T> __device__ __forceinline__ float logit(const Pool<T> &p, int e) { return fminf(to_f32(p.row[e]), kLargest); }

// The two largest values seen, best first; kNone where there are fewer.
__device__ __forceinline__ void add_two(float &first, float &second, float v)
{
    second = fmaxf(second, fminf(first, v));
    first = fmaxf(first, v);
}

// A lane's largest packed choices in order: all of them up to four, the first
// four of eight.
template <int kV> __device__ __forceinline__ void sort_lane(uint32_t (&v)[kV])
{
    auto cex = [&](int i, int j) {
        const uint32_t hi = max(v[i], v[j]), lo = min(v[i], v[j]);
        v[i] = hi;
        v[j] = lo;
    };
    if constexpr (kV == 2) {
        cex(0, 1);
    } else if constexpr (kV == 4) {
        cex(0, 1); cex(2, 3); cex(0, 2); cex(1, 3); cex(1, 2);
    } else {
        cex(0, 1); cex(2, 3); cex(0, 2); cex(1, 3); cex(1, 2);
        cex(4, 5); cex(6, 7); cex(4, 6); cex(5, 7); cex(5, 6);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = max(v[i], v[7 - i]);  // the larger half, bitonic
        cex(0, 2); cex(1, 3); cex(0, 1); cex(2, 3);
    }
}

// The packed word of a choice: 24 bits of its key over 255 - expert, so that
// one redux gives the winner and who it is, and equal choices come by the
// lower id.  Those of -inf, no candidates, are below kLeast, all others above.
constexpr uint32_t kLeast = 0x00800000u;

// The `rounds` best of the packed choices in order: lane j gets the j-th, the
// last one is returned.  whole: a lane ran out of its sorted ones.
template <int kV> __device__ __forceinline__ uint32_t pick_packed(uint32_t (&v)[kV], int rounds, int lane, uint32_t &mine, bool &whole)
{
    constexpr int kDepth = kV < 4 ? kV : 4;
    sort_lane<kV>(v);
    mine = 0;
    uint32_t best = 0;
    for (int j = 0; j < rounds; ++j) {
        best = __reduce_max_sync(~0u, v[0]);
        mine = lane == j ? best : mine;
        const bool won = v[0] == best;  // one lane alone, while any is left
#pragma unroll
        for (int i = 0; i + 1 < kDepth; ++i) v[i] = won ? v[i + 1] : v[i];
        v[kDepth - 1] = won ? 0u : v[kDepth - 1];
    }
    whole = kV > kDepth && __any_sync(~0u, v[0] == 0u);
    return best;
}

// The same by whole 32-bit or 64-bit keys (0: no candidate), for the rows that
// packed ones do not settle: lane j <= k gets the j-th's expert (-1: none),
// e_next the (k + 1)-th's.
__device__ __forceinline__ uint32_t warp_max(uint32_t v) { return __reduce_max_sync(~0u, v); }
__device__ __forceinline__ u64 warp_max(u64 v) { return warp_max64(v); }
template <typename K, int kV> __device__ __forceinline__ void pick_whole(K (&key)[kV], int k, int lane, int &e_mine, int &e_next)
{
    e_mine = e_next = -1;
    for (int j = 0; j <= k; ++j) {
        K mine = 0;
        int e = -1;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const bool take = key[i] > mine;
            mine = take ? key[i] : mine;
            e = take ? lane * kV + i : e;
        }
        const K best = warp_max(mine);
        if (best == 0) return;  // uniform: no candidate is left
        // experts ascend with the lanes: the lowest lane holds the lowest one
        e = __shfl_sync(~0u, e, __ffs(__ballot_sync(~0u, mine == best)) - 1);
        if (lane == j) e_mine = e;
        if (j == k) e_next = e;
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (e == lane * kV + i) key[i] = 0;
    }
}

// A group's lanes where groups are whole lanes, a power of two of them; else 0.
template <int kV> __device__ __forceinline__ int lanes_of_group(int size)
{
    const int seg = size / kV;
    return seg * kV == size && (seg & (seg - 1)) == 0 ? seg : 0;
}

// Lane g's value of group g, of n <= 32 groups of any size, from the keys of
// what groups count by (0: no candidate).
template <typename K, int kV>
__device__ __forceinline__ auto group_value(const K (&key)[kV], int n, int size, int top2, int lane) -> decltype(of(K()))
{
    decltype(of(K())) mine = kNone;
    for (int g = 0; g < n; ++g) {
        K a = 0, b = 0;  // the lane's two best in the group
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const int e = lane * kV + i;
            const K v = e >= g * size && e < (g + 1) * size ? key[i] : 0;
            b = max(b, min(a, v));
            a = max(a, v);
        }
        const K first = warp_max(a);
        const int who = __ffs(__ballot_sync(~0u, a == first)) - 1;
        const K second = top2 ? warp_max(lane == who ? b : a) : 0;
        if (lane == g && first != 0) {
            mine = of(first);
            if (second != 0) mine += of(second);
            if constexpr (sizeof(K) == 4) mine = fmaxf(mine, -kLargest);  // two of the lowest value are still candidates
        }
    }
    return mine;
}

// Lane j's weight of its pick: z its logit, s its score where `scored`.  mine:
// there is a pick.  ordered: lane 0's logit is the largest.
__device__ __forceinline__ float weight_of(bool mine, float z, float s, int sigmoid, int renorm, bool ordered)
{
    float w = mine ? s : 0.f;
    if (renorm && sigmoid) {
        w = w / (warp_sum(w) + 1e-20f);
    } else if (renorm) {  // softmax over the k
        const float m = ordered ? __shfl_sync(~0u, z, 0) : of(__reduce_max_sync(~0u, key_of(mine ? z : kNone)));
        w = mine ? expf(z - m) : 0.f;
        const float total = warp_sum(w);
        if (mine) w = w / total;
    }
    return w;
}

template <typename T> __device__ __forceinline__ Pool<T> pool_of(const ScoreParams &p, long long t, int priv)
{
    const int base = priv ? p.E_pub : 0;
    return {(const T *)p.logits + t * p.ld + base, p.bias ? p.bias + base : nullptr, priv ? p.E_priv : p.E_pub, p.sigmoid,
            p.groups[priv], p.top_groups[priv], p.top2, p.k};
}

// A token that FP32 does not settle.  kept: its groups where those are settled
// (0: they are not), and then the FP32 choice below which no expert can be
// among the k.
struct Aside {
    int t;
    uint32_t kept;
    float least;
};

__device__ __forceinline__ float fast_sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

// Its selection by 64-bit choices, by the whole CTA: a thread evaluates an
// expert, warp 0 selects.  s_key: choices, then what groups count by (0: no
// candidate).
template <typename T, int kV>
__device__ __noinline__ void select_exactly(const ScoreParams &p, const Aside &a, u64 (&s_key)[2][kMaxPool], int *s_load)
{
    const int t = a.t;
    __shared__ double s_sum[kRouteWarps];
    __shared__ uint32_t s_max[kRouteWarps];
    const int e = threadIdx.x, lane = e & 31, warp = e >> 5;
    const int priv = p.policy != nullptr && p.policy[t] == 0x01 ? 1 : 0, base = priv ? p.E_pub : 0;
    const Pool<T> pool = pool_of<T>(p, t, priv);
    const float raw = e < pool.E ? to_f32(pool.row[e]) : kNone, z = raw > kNone ? fminf(raw, kLargest) + 0.f : kNone;
    bool on = z > kNone;
    if (a.kept) on = on && ((a.kept >> (e / (pool.E / pool.n))) & 1u);
    float mx = kNone;
    double sum = 1., v = 0.;
    if (p.sigmoid) {
        // a warp without a candidate has nothing to evaluate
        on = on && (!a.kept || !(fast_sigmoid(z) + pool.bias[e] < a.least));
        if (on) v = 1. / (1. + exp(-(double)z));
    } else {
        const uint32_t top = __reduce_max_sync(~0u, key_of(z));
        if (lane == 0) s_max[warp] = top;
        __syncthreads();
        uint32_t all = 0;
        for (int q = 0; q < kRouteWarps; ++q) all = max(all, s_max[q]);
        mx = of(all);
        if (z > kNone) v = exp((double)z - mx);
        const double part = warp_sum(v);
        if (lane == 0) s_sum[warp] = part;
        __syncthreads();
        sum = 0.;
        for (int q = 0; q < kRouteWarps; ++q) sum += s_sum[q];
        if (on) v /= sum;
    }
    if (pool.bias && on) v += pool.bias[e];
    on = on && v > (double)kNone;  // a bias of -inf (or NaN) takes its expert out
    s_key[0][e] = !on ? 0 : pool.bias ? key64(v) : key64((double)z);
    s_key[1][e] = !on ? 0 : p.top2 ? key64(v) : s_key[0][e];
    __syncthreads();
    if (warp == 0) {
        u64 key[kV], by[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            key[i] = s_key[0][lane * kV + i];
            by[i] = s_key[1][lane * kV + i];
        }
        if (!a.kept) {
            const int size = pool.E / pool.n;
            const u64 g = key64(group_value<u64, kV>(by, pool.n, size, p.top2, lane));
            int place = 0;
            for (int q = 0; q < pool.n; ++q) {
                const u64 o = __shfl_sync(~0u, g, q);
                place += o > g || (o == g && q < lane) ? 1 : 0;
            }
            const uint32_t kept = __ballot_sync(~0u, lane < pool.n && place < pool.top);
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const int q = lane * kV + i;
                if (q < pool.E && !((kept >> (q / size)) & 1u)) key[i] = 0;
            }
        }
        int pick, next;
        pick_whole<u64, kV>(key, p.k, lane, pick, next);
        const bool mine = lane < p.k && pick >= 0;
        const float zj = mine ? logit(pool, pick) : kNone, sum32 = (float)sum;
        const float sj = !mine ? 0.f : p.sigmoid ? 1.f / (1.f + expf(-zj)) : expf(zj - mx) / sum32;
        const float w = weight_of(mine, zj, sj, p.sigmoid, p.renorm, false);
        if (lane < p.k) {
            p.idx[(long long)t * p.k + lane] = mine ? base + pick : -1;
            p.w[(long long)t * p.k + lane] = w * p.scale;
            if (p.load && mine) atomicAdd(s_load + base + pick, 1);
        }
    }
    __syncthreads();  // the keys are read
}

// A lane's logits; -inf for what does not exist.
template <typename T, int kV> __device__ __forceinline__ void load_logits(float (&z)[kV], const T *p, int lane, int E, bool vec)
{
    struct alignas(sizeof(T) * kV) Pack { T v[kV]; };
    const int e0 = lane * kV;
    if (vec && e0 + kV <= E) {
        const Pack q = *reinterpret_cast<const Pack *>(p + e0);
#pragma unroll
        for (int i = 0; i < kV; ++i) z[i] = to_f32(q.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) z[i] = e0 + i < E ? to_f32(p[e0 + i]) : kNone;
    }
}

// kBias: choices are scores + biases.  kGroups: a pool's groups may be limited.
// smem: a CTA's tokens (those put aside) where either holds, the loads' counts.
template <typename T, int kV, bool kBias, bool kGroups>
__global__ void __launch_bounds__(32 * kRouteWarps) route_scores_kernel(const ScoreParams p)
{
    constexpr bool kAside = kBias || kGroups;
    extern __shared__ int s_dynamic[];
    __shared__ u64 s_key[kAside ? 2 : 1][kAside ? kMaxPool : 1];
    __shared__ int s_aside;
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E_all = p.E_pub + p.E_priv;
    Aside *s_tokens = reinterpret_cast<Aside *>(s_dynamic);
    int *s_load = s_dynamic + (kAside ? p.tokens * (int)(sizeof(Aside) / sizeof(int)) : 0);
    if (p.load)
        for (int e = threadIdx.x; e < E_all; e += blockDim.x) s_load[e] = 0;
    if (threadIdx.x == 0) s_aside = 0;
    if (kAside || p.load) __syncthreads();
    // a token's pool and logits are requested while the token before it is in work
    const int step = gridDim.x * kRouteWarps;
    auto pool_at = [&](int t) { return t < p.T && p.policy != nullptr && p.policy[t] == 0x01 ? 1 : 0; };
    float z_next[kV];
    auto fetch = [&](int t, int q) {
        if (t >= p.T) return;
        const T *row = (const T *)p.logits + t * p.ld + (q ? p.E_pub : 0);
        load_logits<T, kV>(z_next, row, lane, q ? p.E_priv : p.E_pub, ((uintptr_t)row & (sizeof(T) * kV - 1)) == 0);
    };
    int t = blockIdx.x * kRouteWarps + warp;
    int priv_next = pool_at(t), priv_after = pool_at(t + step), priv_bias = -1;
    float bias[kV];
    fetch(t, priv_next);
    for (; t < p.T; t += step) {
        const int priv = priv_next, base = priv ? p.E_pub : 0;
        const Pool<T> pool = pool_of<T>(p, t, priv);
        const int E = pool.E;
        const bool limited = kGroups && pool.top < pool.n, scored = kBias || (limited && p.top2);
        if (kBias && priv != priv_bias) {  // a lane's experts, and so its biases, change with the pool alone
#pragma unroll
            for (int i = 0; i < kV; ++i) bias[i] = lane * kV + i < E ? __ldg(pool.bias + lane * kV + i) : 0.f;
            priv_bias = priv;
        }
        float z[kV];  // -inf: not eligible
#pragma unroll
        for (int i = 0; i < kV; ++i) z[i] = fminf(fmaxf(z_next[i], kNone), kLargest);  // the larger of NaN and -inf is -inf
        fetch(t + step, priv_after);
        priv_next = priv_after;
        priv_after = pool_at(t + 2 * step);
        // The choices come from the fast exponential and quotient, whose error
        // is known: __expf(x) 2 + 1.2 |x| ulp, __fdividef 2 ulp, ulp <= 2^-23.
        // So a choice c is off by F + 2^-24 |c|, and those that expf and a whole
        // quotient give for the picks by A + 2^-24 |c|, with F + A <= err:
        // sigmoid, in 2^-23: the exponential's error enters with s (1 - s), and
        // the sum (0.5) and the quotient (2) with s: F = s (1 - s) (2 + 1.2 |z|)
        // + 2.5 s < 2.7, A = 2 s (1 - s) + s < 1.2, err 4;
        // softmax, in 2^-24 / sum, with d = z - max and |d| e^d < 0.4: F = e^d
        // (4 + 3.4 |d| + 2) < 7.4 (d's rounding with it), A < 5.5, and the sum's
        // own error, which scales every score alike and so a difference of two
        // scores by its 4 + 3.4 ln 256 + 12 < 35 (|d| weighted by p is at most
        // ln 256): err 50.
        float mx = kNone, sum = 1.f, err = 0x1p-21f;
        float val[kV];  // score + bias, where it is needed
        if (!p.sigmoid && (!p.renorm || scored)) {  // the pool's softmax
#pragma unroll
            for (int i = 0; i < kV; ++i) mx = fmaxf(mx, z[i]);
            mx = of(__reduce_max_sync(~0u, key_of(mx)));
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                val[i] = z[i] > kNone ? (kAside ? __expf(z[i] - mx) : expf(z[i] - mx)) : 0.f;
                sum += val[i];
            }
            sum = warp_sum(sum);
            err = 0x1.9p-19f / sum;
        }
        if (scored) {
            if (p.sigmoid) {
#pragma unroll
                for (int i = 0; i < kV; ++i) val[i] = fast_sigmoid(z[i]);
            } else {
                const float inv_sum = 1.f / sum;
#pragma unroll
                for (int i = 0; i < kV; ++i) val[i] *= inv_sum;
            }
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                if (kBias) val[i] += bias[i];
                // a bias of -inf (or NaN) takes its expert out too
                val[i] = z[i] > kNone && val[i] > kNone ? val[i] : kNone;
            }
        }
        float choice[kV];  // -inf: no candidate
#pragma unroll
        for (int i = 0; i < kV; ++i) choice[i] = kBias ? val[i] : z[i];
        bool doubt = false, groups_doubt = false;
        int g = 0, place = 0;  // this lane's group and its place
        if (kGroups && limited) {
            const int n = pool.n, top = pool.top, size = E / n, seg = lanes_of_group<kV>(size);
            float by[kV];  // what groups count by
#pragma unroll
            for (int i = 0; i < kV; ++i) by[i] = p.top2 ? val[i] : choice[i];
            float a;    // a group's value: its lanes', or lane g's of group g
            if (seg) {  // every group at once: its lanes hold its two best after log2(seg) exchanges
                float b = kNone;
                a = kNone;
#pragma unroll
                for (int i = 0; i < kV; ++i) add_two(a, b, by[i]);
                for (int off = 1; off < seg; off <<= 1) {
                    const float oa = __shfl_xor_sync(~0u, a, off), ob = __shfl_xor_sync(~0u, b, off);
                    add_two(a, b, oa);
                    add_two(a, b, ob);
                }
                if (p.top2 && b > kNone) a = fmaxf(a + b, -kLargest);  // two of the lowest value are still candidates
                g = lane / seg;
                for (int q = 0; q < n; ++q) {
                    const float o = __shfl_sync(~0u, a, q * seg);
                    place += o > a || (o == a && q < g) ? 1 : 0;
                }
#pragma unroll
                for (int i = 0; i < kV; ++i) choice[i] = place < top ? choice[i] : kNone;
            } else {
                uint32_t key[kV];
#pragma unroll
                for (int i = 0; i < kV; ++i) key[i] = by[i] > kNone ? key_of(by[i]) : 0u;
                a = group_value<uint32_t, kV>(key, n, size, p.top2, lane);
                g = lane;
                for (int q = 0; q < n; ++q) {
                    const float o = __shfl_sync(~0u, a, q);
                    place += o > a || (o == a && q < lane) ? 1 : 0;
                }
                const uint32_t kept = __ballot_sync(~0u, g < n && place < top);
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    const int e = lane * kV + i;
                    if (e < E && !((kept >> (e / size)) & 1u)) choice[i] = kNone;
                }
            }
            if (scored) {  // the last group kept and the first one dropped: sums of two values each, and their own rounding
                float top_value = 0.f;
#pragma unroll
                for (int i = 0; i < kV; ++i) top_value = fmaxf(top_value, val[i] > kNone ? fabsf(val[i]) : 0.f);
                top_value = of(__reduce_max_sync(~0u, key_of(top_value)));
                const float x = __shfl_sync(~0u, a, __ffs(__ballot_sync(~0u, g < n && place == top - 1)) - 1);
                const float y = __shfl_sync(~0u, a, __ffs(__ballot_sync(~0u, g < n && place == top)) - 1);
                groups_doubt = y > kNone && !(x - y > 4.f * err + 0x1p-20f * top_value);
                // A row of equal logits (padding) and biases is nothing but true
                // ties, settled by the ids: T = 8192 of them 24 us, put aside 274.
                if (groups_doubt) {
                    bool alike = true;
#pragma unroll 1
                    for (int e0 = 0; alike && e0 < E; e0 += 32) {
                        const int e = min(e0 + lane, E - 1);
                        const bool same_z = to_f32(pool.row[e]) == to_f32(pool.row[0]), same_b = !kBias || pool.bias[e] == pool.bias[0];
                        alike = __all_sync(~0u, same_z && same_b);
                    }
                    groups_doubt = !alike;
                }
            }
        }
        // Neighbours in the order, the last one's being the first not chosen
        // (which lane k holds, and e_next), are in doubt where their packed
        // choices are equal (again from the whole ones) or their FP32 choices
        // closer than those are exact, unless their logits and biases are the
        // same: a true tie.  16-bit logits without a bias are packed whole.
        // (Comparisons are written so that an infinite bias means doubt.)
        constexpr bool inexact = kBias || sizeof(T) == 4;
        int e_mine, e_next;
        bool whole;
        float above;  // no choice of the next one's packed word is larger
        {
            uint32_t v[kV], mine;
#pragma unroll
            for (int i = 0; i < kV; ++i) v[i] = (key_of(choice[i]) & ~255u) | (uint32_t)(255 - lane * kV - i);
            const uint32_t last = pick_packed<kV>(v, inexact ? p.k + 1 : p.k, lane, mine, whole);
            e_mine = mine >= kLeast ? 255 - (int)(mine & 255u) : -1;
            e_next = last >= kLeast ? 255 - (int)(last & 255u) : -1;
            above = of(last | 255u);
            if (inexact) {
                uint32_t after = __shfl_down_sync(~0u, mine, 1);
                if (lane == 31) after = last;  // of use where k = 32
                whole = whole || __any_sync(~0u, lane < p.k && after >= kLeast && (mine ^ after) < 256u);
            }
        }
        if (whole) {
            uint32_t key[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) key[i] = choice[i] > kNone ? key_of(choice[i]) : 0u;
            pick_whole<uint32_t, kV>(key, p.k, lane, e_mine, e_next);
        }
        auto score = [&](float zz) { return p.sigmoid ? 1.f / (1.f + expf(-zz)) : expf(zz - mx) / sum; };
        float zj = kNone, sj = 0.f, c0 = kNone;
        if (e_mine >= 0) {
            zj = logit(pool, e_mine);
            if (p.sigmoid || !p.renorm || kBias) sj = score(zj);
        }
        if (kBias) {
            const float b0 = e_mine >= 0 ? pool.bias[e_mine] : 0.f;
            c0 = e_mine >= 0 ? sj + b0 : kNone;
            float z1 = __shfl_down_sync(~0u, zj, 1), b1 = __shfl_down_sync(~0u, b0, 1), c1 = __shfl_down_sync(~0u, c0, 1);
            if (p.k == 32 && lane == 31) {  // no lane holds the 33rd
                z1 = e_next >= 0 ? logit(pool, e_next) : kNone;
                b1 = e_next >= 0 ? pool.bias[e_next] : 0.f;
                c1 = e_next >= 0 ? score(z1) + b1 : kNone;
            }
            // A pick against the next one down, whose own FP32 choice may be low
            // by as much: twice err, and four roundings.
            doubt = lane < p.k && c1 > kNone && !(c0 - c1 > 2.f * err + 0x1.8p-23f * (fabsf(c0) + fabsf(c1))) &&
                    !(b0 == b1 && zj == z1);
            // The k-th against what else may share the next one's packed word.
            if (!whole && lane == p.k - 1 && e_next >= 0)
                doubt = doubt || !(c0 - above > err + 0x1.8p-23f * (fabsf(c0) + fabsf(above)));
            // The k-th and the next one a true tie: against all that is not one.
            // (From memory again: choices kept for this took 24 registers.)
            if (__any_sync(~0u, lane == p.k - 1 && c1 > kNone && b0 == b1 && zj == z1)) {
                const float ck = __shfl_sync(~0u, c0, p.k - 1), zk = __shfl_sync(~0u, zj, p.k - 1), bk = __shfl_sync(~0u, b0, p.k - 1);
#pragma unroll 1
                for (int e = lane; e < E; e += 32) {
                    const float ze = to_f32(pool.row[e]) > kNone ? logit(pool, e) : kNone, be = pool.bias[e];
                    const float c = (p.sigmoid ? fast_sigmoid(ze) : __expf(ze - mx) * (1.f / sum)) + be;
                    doubt = doubt || (ze > kNone && c > kNone && !(ze == zk && be == bk) &&
                                      !(fabsf(ck - c) > err + 0x1.8p-23f * (fabsf(ck) + fabsf(c))));
                }
            }
        }
        if (kAside && __any_sync(~0u, doubt || groups_doubt)) {
            // the k-th choice: an expert further below it than A + 3 F (the picks
            // before it, itself and that expert) and their roundings is none
            const float c = __shfl_sync(~0u, c0, p.k - 1);
            const uint32_t kept = limited ? __reduce_or_sync(~0u, g < pool.n && place < pool.top ? 1u << g : 0u) : ~0u;
            if (lane == 0)
                s_tokens[atomicAdd(&s_aside, 1)] = {t, groups_doubt ? 0u : kept, c - (3.f * err + 0x1.8p-22f * fabsf(c))};
            continue;
        }
        const bool mine = lane < p.k && e_mine >= 0;
        const float w = weight_of(mine, zj, sj, p.sigmoid, p.renorm, !kBias);
        if (lane < p.k) {
            p.idx[(long long)t * p.k + lane] = mine ? base + e_mine : -1;
            p.w[(long long)t * p.k + lane] = w * p.scale;
            if (p.load && mine) atomicAdd(s_load + base + e_mine, 1);
        }
    }
    if constexpr (kAside) {
        __syncthreads();
        const int aside = s_aside;  // in any order: each token's result is its own
        for (int i = 0; i < aside; ++i) select_exactly<T, kV>(p, s_tokens[i], s_key, s_load);
    }
    if (p.load) {  // whole numbers: the order of the additions does not matter
        __syncthreads();
        for (int e = threadIdx.x; e < E_all; e += blockDim.x)
            if (s_load[e]) atomicAdd(p.load + e, s_load[e]);
    }
}

// ------------------------------------------------------------- backward

struct ScoreBwdParams {
    const void *logits;
    const uint8_t *policy;
    const int32_t *idx;
    const float *dw;
    void *d_logits;
    long long ld;
    int T, E_pub, E_priv, k, renorm, sigmoid;
    float scale;
};

// d_logits of a token, a warp each.  With s the scores, S the sum of the k
// chosen ones and D_j = scale dL/dw_j:
//   renormalised: ds_j = (D_j - sum_i D_i s_i / S) / S,  else ds_j = D_j
//   sigmoid: dz_j = ds_j s_j (1 - s_j)
//   softmax: dz_e = p_e (ds_e - sum_i ds_i p_i); renormalised the sum is zero
//   and only the k chosen remain: dz_j = w_j (D_j - sum_i D_i w_i)
// The selection is piecewise constant, and the bias only selects: neither has
// a gradient.  An id outside the token's pool contributes nothing.
template <typename T, int kV> __global__ void __launch_bounds__(32 * kRouteWarps) route_scores_bwd_kernel(const ScoreBwdParams p)
{
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E_all = p.E_pub + p.E_priv;
    for (int t = blockIdx.x * kRouteWarps + warp; t < p.T; t += gridDim.x * kRouteWarps) {
        const int priv = p.policy != nullptr && p.policy[t] == 0x01 ? 1 : 0;
        const int base = priv ? p.E_pub : 0, E = priv ? p.E_priv : p.E_pub;
        const T *row = (const T *)p.logits + t * p.ld + base;
        T *out = (T *)p.d_logits + (long long)t * E_all;
        int e = -1;
        float D = 0.f, zj = kNone;
        if (lane < p.k) {
            e = p.idx[(long long)t * p.k + lane];  // any value
            D = p.dw[(long long)t * p.k + lane] * p.scale;
        }
        // the whole row at once, beside the ids, not the picks' logits after them (4.08 us, so 3.9)
        float z[kV];
        load_logits<T, kV>(z, row, lane, E, ((uintptr_t)row & (sizeof(T) * kV - 1)) == 0);
        e = e >= base && e < base + E ? e - base : -1;
#pragma unroll
        for (int i = 0; i < kV; ++i) {  // a pick's logit from the lane that holds it
            const float o = __shfl_sync(~0u, z[i], max(e, 0) / kV);
            if (e >= 0 && e % kV == i) zj = o;
        }
        if (!(zj > kNone)) e = -1;  // never chosen
        if (e < 0) D = 0.f;
        zj = e >= 0 ? fminf(zj, kLargest) : kNone;
        const bool mine = e >= 0;
        float g = 0.f;  // what lane j adds to its expert's gradient
        float d[kV];
        const bool dense = !p.sigmoid && !p.renorm;
        // the other pool's logits have no gradient
        const int other = priv ? 0 : p.E_pub, n_other = priv ? p.E_pub : p.E_priv;
        for (int i = lane; i < n_other; i += 32) out[other + i] = from_f32<T>(0.f);
        if (p.sigmoid) {
            const float s = mine ? 1.f / (1.f + expf(-zj)) : 0.f;
            float ds = D;
            if (p.renorm) {
                const float S = warp_sum(s) + 1e-20f;
                ds = (D - warp_sum(mine ? D * s : 0.f) / S) / S;
            }
            // s (1 - s), 1 - s as the sigmoid of -z: no cancellation near s = 1
            if (mine) g = ds * s * (1.f / (1.f + expf(zj)));
        } else if (p.renorm) {
            const float m = of(__reduce_max_sync(~0u, key_of(mine ? zj : kNone)));
            const float ex = mine ? expf(zj - m) : 0.f;
            const float total = warp_sum(ex);
            const float w = mine ? ex / total : 0.f;
            const float mean = warp_sum(mine ? D * w : 0.f);
            if (mine) g = w * (D - mean);
        }
#pragma unroll
        for (int i = 0; i < kV; ++i) d[i] = 0.f;
        if (dense) {
            float mx = kNone, sum = 0.f;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                z[i] = z[i] > kNone ? fminf(z[i], kLargest) : kNone;
                mx = fmaxf(mx, z[i]);
            }
            mx = of(__reduce_max_sync(~0u, key_of(mx)));
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                d[i] = z[i] > kNone ? expf(z[i] - mx) : 0.f;
                sum += d[i];
            }
            sum = warp_sum(sum);
            const float pj = mine ? expf(zj - mx) / sum : 0.f;
            const float total = warp_sum(mine ? D * pj : 0.f);
#pragma unroll
            for (int i = 0; i < kV; ++i) d[i] = sum > 0.f ? -(d[i] / sum) * total : 0.f;
            g = pj * D;
        }
        for (int j = 0; j < p.k; ++j) {
            const int ej = __shfl_sync(~0u, mine ? e : -1, j);
            const float gj = __shfl_sync(~0u, g, j);
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (ej == lane * kV + i) d[i] += gj;
        }
        struct alignas(sizeof(T) * kV) Pack { T v[kV]; };
        T *o = out + base + lane * kV;
        if (lane * kV + kV <= E && ((uintptr_t)(out + base) & (sizeof(T) * kV - 1)) == 0) {
            Pack q;
#pragma unroll
            for (int i = 0; i < kV; ++i) q.v[i] = from_f32<T>(d[i]);
            *reinterpret_cast<Pack *>(o) = q;
        } else {
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (lane * kV + i < E) o[i] = from_f32<T>(d[i]);
        }
    }
}

// Calls go(T(), experts a lane) for the logits' type and the larger pool.
template <typename Go> cudaError_t dispatch(int type, int pool, Go go)
{
    auto by_size = [&](auto t) {
        if (pool <= 64) return go(t, std::integral_constant<int, 2>());
        if (pool <= 128) return go(t, std::integral_constant<int, 4>());
        return go(t, std::integral_constant<int, 8>());
    };
    if (type == PMPE_F32) return by_size(float());
    if (type == PMPE_BF16) return by_size(bf16());
    return by_size(__half());
}

// CTAs for T tokens: up to per_sm an SM, and not more than kMostTokens tokens
// each.  Eight where a token is short (T = 16384, 128 + 32 experts 8.0 us, with
// five 8.2); with biases or groups as many as are resident at once, so that no
// CTA starts late with a token to settle at its end (T = 8192, 256 experts in
// groups with biases 17.0 us, with eight 18.3; 128 + 32 with biases 14.6, 15.0).
constexpr int kMostTokens = 1024;
constexpr int kCtasPerSm = 8;
int grid_of(int T, int num_sms, int per_sm)
{
    const int all = (T + kRouteWarps - 1) / kRouteWarps;
    return std::max(1, std::min(all, std::max(per_sm * num_sms, (T + kMostTokens - 1) / kMostTokens)));
}

}  // namespace

cudaError_t launch_route_scores(const pmpe_route_desc &d, int num_sms, cudaStream_t st)
{
    ScoreParams p;
    p.logits = d.logits; p.policy = d.E_priv > 0 ? d.policy : nullptr; p.bias = d.bias;
    p.idx = d.topk_idx; p.w = d.topk_w; p.load = d.load; p.ld = d.ld;
    p.T = d.T; p.E_pub = d.E_pub; p.E_priv = d.E_priv; p.k = d.k; p.renorm = d.renormalize;
    p.sigmoid = d.score == PMPE_SCORE_SIGMOID; p.top2 = d.group_score == PMPE_GROUP_TOP2;
    p.groups[0] = d.groups_pub; p.groups[1] = d.groups_priv;
    p.top_groups[0] = d.top_groups_pub; p.top_groups[1] = d.top_groups_priv;
    p.scale = d.scale;
    const bool limited = d.top_groups_pub < d.groups_pub || (d.E_priv > 0 && d.top_groups_priv < d.groups_priv);
    // registers: 80 above 128 experts, at most 64 below
    const int resident = std::max(d.E_pub, d.E_priv) > 128 ? 3 : 4;
    const dim3 grid(grid_of(d.T, num_sms, limited || d.bias ? resident : kCtasPerSm)), block(32 * kRouteWarps);
    p.tokens = (d.T + (int)grid.x * kRouteWarps - 1) / ((int)grid.x * kRouteWarps) * kRouteWarps;
    const size_t smem = (limited || d.bias ? p.tokens * sizeof(Aside) : 0) + (d.load ? (d.E_pub + d.E_priv) * sizeof(int) : 0);
    return dispatch(d.logits_type, std::max(d.E_pub, d.E_priv), [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int kV = decltype(v)::value;
        if (d.bias)
            return limited ? launch_pdl(route_scores_kernel<T, kV, true, true>, grid, block, smem, st, p)
                           : launch_pdl(route_scores_kernel<T, kV, true, false>, grid, block, smem, st, p);
        return limited ? launch_pdl(route_scores_kernel<T, kV, false, true>, grid, block, smem, st, p)
                       : launch_pdl(route_scores_kernel<T, kV, false, false>, grid, block, smem, st, p);
    });
}

cudaError_t launch_route_scores_backward(const pmpe_route_desc &d, const float *dw, void *d_logits, int num_sms,
                                         cudaStream_t st)
{
    ScoreBwdParams p;
    p.logits = d.logits; p.policy = d.E_priv > 0 ? d.policy : nullptr; p.idx = d.topk_idx; p.dw = dw;
    p.d_logits = d_logits; p.ld = d.ld;
    p.T = d.T; p.E_pub = d.E_pub; p.E_priv = d.E_priv; p.k = d.k; p.renorm = d.renormalize;
    p.sigmoid = d.score == PMPE_SCORE_SIGMOID;
    p.scale = d.scale;
    const dim3 grid(grid_of(d.T, num_sms, kCtasPerSm)), block(32 * kRouteWarps);
    return dispatch(d.logits_type, std::max(d.E_pub, d.E_priv), [&](auto t, auto v) {
        return launch_pdl(route_scores_bwd_kernel<decltype(t), decltype(v)::value>, grid, block, 0, st, p);
    });
}

}  // namespace pmpe
