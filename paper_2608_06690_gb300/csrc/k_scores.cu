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
// row is read once with one vector load a lane, and each of the k rounds is
// one redux over order-preserving 32-bit keys, a ballot and an update in the
// winner's lane.
//
// The selection is that of exact arithmetic.  Logits compare exactly.
// Choices with a bias are FP32, a few 2^-24 off: where two choices that
// follow one another in the order (or two groups at the limit) lie within
// the bound of that error, the warp selects again with 64-bit choices.  That
// is about one token in a thousand; a 64-bit exponential for every expert
// would cost more than everything else here (2 FP64 operations a clock and SM).
#include <algorithm>

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
    float scale;
};

// Unsigned keys in the order of the floats; 0 is below every float, and -0 and
// +0 are one key.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t key)
{
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

constexpr float kNone = -INFINITY;
constexpr float kLargest = 3.402823466e38f;  // stands for a logit of +inf

// The largest value over the warp and the lowest expert that has it.
__device__ __forceinline__ void warp_best(float &v, int &e)
{
    const uint32_t key = e < 0 ? 0u : key_of(v);
    const uint32_t best = __reduce_max_sync(~0u, key);
    // experts ascend with the lanes, so the lowest lane holds the lowest expert
    const int src = __ffs(__ballot_sync(~0u, key == best)) - 1;
    e = __shfl_sync(~0u, best ? e : -1, src);
    v = best ? of_key(best) : kNone;
}
__device__ __forceinline__ void warp_best(double &v, int &e)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const double ov = __shfl_xor_sync(~0u, v, off);
        const int oe = __shfl_xor_sync(~0u, e, off);
        const bool take = oe >= 0 && (e < 0 || ov > v || (ov == v && oe < e));
        v = take ? ov : v;
        e = take ? oe : e;
    }
}

// Whether a group's value a of group i ranks above b of group j.
template <typename V> __device__ __forceinline__ bool group_above(V a, int i, V b, int j)
{
    return a > b || (a == b && i < j);
}

// The two largest values seen, best first; kNone where there are fewer.
template <typename V> __device__ __forceinline__ void add_two(V &first, V &second, V v)
{
    second = v > first ? first : (v > second ? v : second);
    first = v > first ? v : first;
}

// Clears the candidates (choice -> -inf) outside the best `top` of n groups of
// `size` experts.  val: score + bias, what two-best sums are made of.  Lane l
// computes group l's value (n <= 32).  gap: the distance between the last
// group kept and the first one dropped (+inf where nothing is dropped).
template <typename V, int kV>
__device__ __forceinline__ void limit_groups(V (&choice)[kV], const V (&val)[kV], int n, int size, int top, int top2, int lane,
                                             V &gap)
{
    const V none = (V)kNone;
    V mine = none;
    for (int g = 0; g < n; ++g) {
        V a = none, b = none;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const int e = lane * kV + i;
            const V c = e >= g * size && e < (g + 1) * size && choice[i] > none ? (top2 ? val[i] : choice[i]) : none;
            add_two(a, b, c);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            const V oa = __shfl_xor_sync(~0u, a, off), ob = __shfl_xor_sync(~0u, b, off);
            add_two(a, b, oa);
            add_two(a, b, ob);
        }
        if (top2 && b > none) a += b;
        if (lane == g) mine = a;
    }
    // rank of each group; the smallest kept and the largest dropped value
    int rank = 0;
    for (int g = 0; g < n; ++g) {
        const V o = __shfl_sync(~0u, mine, g);
        rank += group_above(o, g, mine, lane) ? 1 : 0;
    }
    const uint32_t kept = __ballot_sync(~0u, lane < n && rank < top);
    const uint32_t last = __ballot_sync(~0u, lane < n && rank == top - 1);
    const uint32_t next = __ballot_sync(~0u, lane < n && rank == top);
    gap = (V)INFINITY;
    if (next) {
        const V a = __shfl_sync(~0u, mine, __ffs(last) - 1), b = __shfl_sync(~0u, mine, __ffs(next) - 1);
        if (b > none) gap = a - b;
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        const int e = lane * kV + i;
        if (e < n * size && !((kept >> (e / size)) & 1u)) choice[i] = none;
    }
}

// The k best choices in order: lane j < k gets the j-th's expert (-1: none)
// and choice; next: the (k + 1)-th's (asked for by want_next).
template <typename V, int kV>
__device__ __forceinline__ void pick(V (&choice)[kV], int k, bool want_next, int lane, int &e_mine, V &c_mine, int &e_next,
                                     V &c_next)
{
    const V none = (V)kNone;
    e_mine = e_next = -1;
    c_mine = c_next = none;
    for (int j = 0; j < k + (want_next ? 1 : 0); ++j) {
        V c = none;
        int e = -1;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const bool take = choice[i] > c;
            c = take ? choice[i] : c;
            e = take ? lane * kV + i : e;
        }
        warp_best(c, e);
        if (e < 0) return;  // uniform: no candidate is left
        if (j < k) {
            if (lane == j) {
                e_mine = e;
                c_mine = c;
            }
        } else {
            e_next = e;
            c_next = c;
        }
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (e == lane * kV + i) choice[i] = none;
    }
}

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

// The selection in 64 bits, for the tokens whose FP32 choices are too close.
template <typename T, int kV>
__device__ __noinline__ int pick64(const T *row, const float *bias, int E, int sigmoid, int n, int top, int top2, int k, int lane)
{
    double z[kV], choice[kV], val[kV];
    double mx = (double)kNone, sum = 0.;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        const int e = lane * kV + i;
        const float f = e < E ? to_f32(row[e]) : kNone;
        z[i] = f > kNone ? (double)fminf(f, kLargest) : (double)kNone;
        mx = fmax(mx, z[i]);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mx = fmax(mx, __shfl_xor_sync(~0u, mx, off));
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        val[i] = 0.;
        if (z[i] > (double)kNone) val[i] = sigmoid ? 1. / (1. + exp(-z[i])) : exp(z[i] - mx);
        sum += val[i];
    }
    sum = warp_sum(sum);
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        choice[i] = z[i];
        if (z[i] > (double)kNone) {
            if (!sigmoid) val[i] /= sum;
            if (bias) choice[i] = val[i] += bias[lane * kV + i];
        }
    }
    double gap, c_mine, c_next;
    int e_mine, e_next;
    if (top < n) limit_groups<double, kV>(choice, val, n, E / n, top, top2, lane, gap);
    pick<double, kV>(choice, k, false, lane, e_mine, c_mine, e_next, c_next);
    return e_mine;
}

template <typename T, int kV> __global__ void __launch_bounds__(32 * kRouteWarps) route_scores_kernel(const ScoreParams p)
{
    extern __shared__ int s_load[];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E_all = p.E_pub + p.E_priv;
    if (p.load) {
        for (int e = threadIdx.x; e < E_all; e += blockDim.x) s_load[e] = 0;
        __syncthreads();
    }
    for (int t = blockIdx.x * kRouteWarps + warp; t < p.T; t += gridDim.x * kRouteWarps) {
        const int priv = p.policy != nullptr && p.policy[t] == 0x01 ? 1 : 0;
        const int base = priv ? p.E_pub : 0, E = priv ? p.E_priv : p.E_pub;
        const T *row = (const T *)p.logits + t * p.ld + base;
        float z[kV], choice[kV], val[kV];
        load_logits<T, kV>(z, row, lane, E, ((uintptr_t)row & (sizeof(T) * kV - 1)) == 0);
        const int n = p.groups[priv], top = p.top_groups[priv], size = E / n;
        const bool limited = top < n, scored = p.bias != nullptr || (limited && p.top2);
        uint32_t live = 0;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            live |= z[i] > kNone ? 1u << i : 0u;
            z[i] = fminf(z[i], kLargest);
        }
        float mx = kNone, sum = 0.f;
        if (!p.sigmoid && (!p.renorm || scored)) {  // the pool's softmax
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if ((live >> i) & 1u) mx = fmaxf(mx, z[i]);
            mx = of_key(__reduce_max_sync(~0u, key_of(mx)));
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if ((live >> i) & 1u) sum += expf(z[i] - mx);
            sum = warp_sum(sum);
        }
        // Error of an FP32 score, relative to it (twice it covers a pair).
        // Sigmoid: expf 2 ulp (2^-22), the sum and the quotient half an ulp
        // each.  Softmax: the difference z - max rounds by up to 2^-24 x 104
        // where exp does not underflow, which the exponential turns into a
        // relative error; the sum of 256 terms 13 x 2^-24 besides.
        const float rel = p.sigmoid ? 0x1p-21f : 0x1p-16f;
        float top_score = 0.f, top_value = 0.f;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const bool on = (live >> i) & 1u;
            val[i] = 0.f;
            choice[i] = on ? z[i] : kNone;
            if (scored && on) {
                val[i] = p.sigmoid ? 1.f / (1.f + expf(-z[i])) : expf(z[i] - mx) / sum;
                top_score = fmaxf(top_score, val[i]);
                if (p.bias) choice[i] = val[i] += __ldg(p.bias + base + lane * kV + i);
                top_value = fmaxf(top_value, fabsf(val[i]));
            }
        }
        bool again = false;
        if (limited) {
            float gap;
            limit_groups<float, kV>(choice, val, n, size, top, p.top2, lane, gap);
            if (scored) {  // sums of up to two values on either side
                top_score = of_key(__reduce_max_sync(~0u, key_of(top_score)));
                top_value = of_key(__reduce_max_sync(~0u, key_of(top_value)));
                again = gap <= 4.f * (rel * top_score + 0x1p-23f * top_value);
            }
        }
        int e_mine, e_next;
        float c_mine, c_next;
        pick<float, kV>(choice, p.k, p.bias != nullptr, lane, e_mine, c_mine, e_next, c_next);
        if (p.bias) {
            // neighbours in the order that are close, unless both their logits
            // and their biases are the same: a true tie
            int e_after = __shfl_down_sync(~0u, e_mine, 1);
            float c_after = __shfl_down_sync(~0u, c_mine, 1);
            if (lane == p.k - 1) {
                e_after = e_next;
                c_after = c_next;
            }
            bool doubt = false;
            if (lane < p.k && e_after >= 0) {
                const float b0 = p.bias[base + e_mine], b1 = p.bias[base + e_after];
                doubt = c_mine - c_after <= rel * (fabsf(c_mine - b0) + fabsf(c_after - b1)) +
                                                0x1p-22f * (fabsf(c_mine) + fabsf(c_after)) &&
                        !(b0 == b1 && to_f32(row[e_mine]) == to_f32(row[e_after]));
            }
            again = again || __any_sync(~0u, doubt);
        }
        if (again)
            e_mine = pick64<T, kV>(row, p.bias ? p.bias + base : nullptr, E, p.sigmoid, n, top, p.top2, p.k, lane);
        // lane j's weight
        const bool mine = lane < p.k && e_mine >= 0;
        float w = 0.f;
        const float zj = mine ? fminf(to_f32(row[e_mine]), kLargest) : kNone;
        if (p.sigmoid) {
            if (mine) w = 1.f / (1.f + expf(-zj));
            if (p.renorm) w = w / (warp_sum(w) + 1e-20f);
        } else if (p.renorm) {  // softmax over the k
            const float m = of_key(__reduce_max_sync(~0u, key_of(zj)));
            if (mine) w = expf(zj - m);
            const float s = warp_sum(w);
            if (mine) w = w / s;
        } else if (mine) {
            w = expf(zj - mx) / sum;
        }
        if (lane < p.k) {
            p.idx[(long long)t * p.k + lane] = mine ? base + e_mine : -1;
            p.w[(long long)t * p.k + lane] = w * p.scale;
            if (p.load && mine) atomicAdd(s_load + base + e_mine, 1);
        }
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
            e = p.idx[(long long)t * p.k + lane] - base;
            if (e < 0 || e >= E) e = -1;
            if (e >= 0) {
                zj = to_f32(row[e]);
                if (zj > kNone) D = p.dw[(long long)t * p.k + lane] * p.scale;
                else e = -1;  // never chosen
                zj = fminf(zj, kLargest);
            }
        }
        const bool mine = e >= 0;
        float g = 0.f;  // what lane j adds to its expert's gradient
        float d[kV];
        const bool dense = !p.sigmoid && !p.renorm;
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
            const float m = of_key(__reduce_max_sync(~0u, key_of(mine ? zj : kNone)));
            const float ex = mine ? expf(zj - m) : 0.f;
            const float total = warp_sum(ex);
            const float w = mine ? ex / total : 0.f;
            const float mean = warp_sum(mine ? D * w : 0.f);
            if (mine) g = w * (D - mean);
        }
#pragma unroll
        for (int i = 0; i < kV; ++i) d[i] = 0.f;
        if (dense) {
            float z[kV];
            load_logits<T, kV>(z, row, lane, E, ((uintptr_t)row & (sizeof(T) * kV - 1)) == 0);
            float mx = kNone, sum = 0.f;
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                z[i] = z[i] > kNone ? fminf(z[i], kLargest) : kNone;
                mx = fmaxf(mx, z[i]);
            }
            mx = of_key(__reduce_max_sync(~0u, key_of(mx)));
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
        // the other pool's logits have no gradient
        const int other = priv ? 0 : p.E_pub, n_other = priv ? p.E_pub : p.E_priv;
        for (int i = lane; i < n_other; i += 32) out[other + i] = from_f32<T>(0.f);
    }
}

template <template <typename, int> class Launch, typename P> cudaError_t dispatch(int type, int pool, const P &p, int grid, int smem, cudaStream_t st)
{
    const int per = (pool + 31) / 32;
    auto by_size = [&](auto tag) {
        using T = decltype(tag);
        if (per <= 1) return Launch<T, 1>::go(p, grid, smem, st);
        if (per <= 2) return Launch<T, 2>::go(p, grid, smem, st);
        if (per <= 4) return Launch<T, 4>::go(p, grid, smem, st);
        return Launch<T, 8>::go(p, grid, smem, st);
    };
    if (type == PMPE_F32) return by_size(float());
    if (type == PMPE_BF16) return by_size(bf16());
    return by_size(__half());
}

template <typename T, int kV> struct LaunchScores {
    static cudaError_t go(const ScoreParams &p, int grid, int smem, cudaStream_t st)
    {
        return launch_pdl(route_scores_kernel<T, kV>, dim3(grid), dim3(32 * kRouteWarps), (size_t)smem, st, p);
    }
};
template <typename T, int kV> struct LaunchScoresBwd {
    static cudaError_t go(const ScoreBwdParams &p, int grid, int smem, cudaStream_t st)
    {
        return launch_pdl(route_scores_bwd_kernel<T, kV>, dim3(grid), dim3(32 * kRouteWarps), (size_t)smem, st, p);
    }
};

int grid_of(int T, int num_sms) { return std::max(1, std::min((T + kRouteWarps - 1) / kRouteWarps, 4 * num_sms)); }

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
    return dispatch<LaunchScores>(d.logits_type, std::max(d.E_pub, d.E_priv), p, grid_of(d.T, num_sms),
                                  d.load ? (d.E_pub + d.E_priv) * 4 : 0, st);
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
    return dispatch<LaunchScoresBwd>(d.logits_type, std::max(d.E_pub, d.E_priv), p, grid_of(d.T, num_sms), 0, st);
}

}  // namespace pmpe
