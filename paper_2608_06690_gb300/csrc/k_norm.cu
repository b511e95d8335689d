// Root-mean-square norm of the residual stream with the residual's addition,
// optionally into 8 bits with scales, and its backward.
//
//   h = round(x + residual)            (x itself without a residual)
//   r = 1 / sqrt(mean_c h_c^2 + eps)
//   y = h r w                          in the input's type, or
//   s = max(amax |y| / 448, 2^-126),  q = e4m3(y / s)   per 128 columns or per row
//
//   g = dy w,  m = mean_c g_c h_c
//   dx = d_h + r g - h r^3 m           (d_h: the gradient that reaches h itself)
//   dw_c = sum_t dy_{t,c} h_{t,c} r_t
//
// h is rounded to its type before the norm, so that the backward, which reads
// the stored h, differentiates what the forward computed.  Everything between
// the loads and the stores is FP32.
//
// Bytes bound both, instructions follow closely (a row of 2048 columns is 8 KB
// in and 8 KB out and some 700 warp instructions): 16-bit sums and FP32
// products take two elements an instruction, and a thread holds 16 columns, so
// that the row's sum over the threads is a small part.
#include <algorithm>

#include <cuda_fp8.h>

#include "elem.cuh"

namespace pmpe {
namespace {

constexpr int kWarpRows = 8;      // rows of a CTA where a warp takes a row
constexpr int kMaxThreads = 512;  // of a CTA that takes a row of up to 8192 columns; twice that above

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
__device__ __forceinline__ float2 pair(const float (&v)[8], int j) { return make_float2(v[2 * j], v[2 * j + 1]); }
__device__ __forceinline__ void set(float (&v)[8], int j, float2 x)
{
    v[2 * j] = x.x;
    v[2 * j + 1] = x.y;
}

// The sum over the row's threads, in every one of them, in a fixed order: a
// warp's row by shuffles, a CTA's through s_red, one entry a warp.
template <bool kWarpRow, typename V> __device__ __forceinline__ V row_sum(V v, V *s_red)
{
    v = warp_sum(v);
    if (kWarpRow) return v;
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0) s_red[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum(lane < warps ? s_red[lane] : V(0));
}

constexpr float kMinScale = 1.17549435e-38f;  // 2^-126: the smallest scale, so that its reciprocal is finite

// A factor in two words: v times 448 / amax with one rounding in all, so that
// a value goes to the e4m3 neighbour of the exact quotient but within 2^-24 of
// the middle between two.
struct Divide {
    float hi, lo;
};
// For values u of a block whose largest is amax and which stand for u m:
// the scale s = max(amax m / 448, 2^-126) and the factor u -> u m / s.
__device__ __forceinline__ Divide divide_by(float amax, float m, float &s)
{
    s = max_nan(amax * m / 448.f, kMinScale);
    if (!(s > kMinScale)) return {m * 0x1p126f, 0.f};  // zeros (or NaN)
    const float hi = 448.f / amax;
    return {hi, hi > 0.f ? fmaf(-hi, amax, 448.f) / amax : 0.f};
}
__device__ __forceinline__ uint32_t e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

struct NormParams {
    const void *x, *res, *w;
    void *h, *y;
    float *scale, *rstd;
    long long x_ld, res_ld;
    int T, H, w_f32, quant;  // quant: PMPE_QUANT_*
    float eps;
};

template <typename T, int kNC, bool kWarpRow, bool kVec, int kThreads>
__global__ void __launch_bounds__(kThreads) rms_norm_kernel(const NormParams p)
{
    __shared__ double s_red64[32];
    __shared__ float s_red[32], s_max[32];
    pdl_trigger();
    pdl_wait();
    const Place<kWarpRow, kVec> at;
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const long long row = kWarpRow ? (long long)blockIdx.x * kWarpRows + (threadIdx.x >> 5) : (long long)blockIdx.x;
    if (row >= p.T) return;  // a whole warp; a CTA's row always exists
    Raw8<T> rx[kNC], rr[kNC];
#pragma unroll
    for (int i = 0; i < kNC; ++i) load8<kVec>(rx[i], (const T *)p.x + row * p.x_ld + at.col(i), p.H - at.col(i));
    if (p.res) {
#pragma unroll
        for (int i = 0; i < kNC; ++i) load8<kVec>(rr[i], (const T *)p.res + row * p.res_ld + at.col(i), p.H - at.col(i));
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            add8(rx[i], rr[i]);
            if (p.h) store_raw<kVec>((T *)p.h + row * p.H + at.col(i), rx[i], p.H - at.col(i));
        }
    } else if (p.h) {
#pragma unroll
        for (int i = 0; i < kNC; ++i) store_raw<kVec>((T *)p.h + row * p.H + at.col(i), rx[i], p.H - at.col(i));
    }
    float v[kNC][8];
    float2 two = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        unpack(rx[i], v[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) two = fma2(pair(v[i], j), pair(v[i], j), two);
    }
    const float ss = row_sum<kWarpRow>(two.x + two.y, s_red);
    float r;
    if (ss < 1e37f) {
        r = rsqrtf(ss / (float)p.H + p.eps);
    } else {  // squares past FP32's range (or NaN): again in 64 bits
        double s64 = 0.;
#pragma unroll
        for (int i = 0; i < kNC; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s64 += (double)v[i][j] * v[i][j];
        r = (float)rsqrt(row_sum<kWarpRow>(s64, s_red64) / p.H + p.eps);
    }
    if (p.rstd && at.t == 0) p.rstd[row] = r;
    // An 8-bit y divides by its block's largest value, and r cancels: only
    // the power of two of r enters y here (exact, and it keeps the products
    // in range), its significand m goes to the scale alone.
    float pre = r, m = 1.f;
    if (p.quant != PMPE_QUANT_NONE && r >= kMinScale) {
        pre = __uint_as_float(__float_as_uint(r) & 0x7f800000u);
        m = __uint_as_float((__float_as_uint(r) & 0x007fffffu) | 0x3f800000u);
    }
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        const int c = at.col(i);
        Raw8<float> rw;
        float w[8];
        load_any<kVec, T>(rw, p.w, p.w_f32, c, p.H - c);
        unpack_any<T>(rw, p.w_f32, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) set(v[i], j, mul2(mul2(pair(v[i], j), make_float2(pre, pre)), pair(w, j)));
        if (p.quant == PMPE_QUANT_NONE) {
            store8<kVec>((T *)p.y + row * p.H + c, v[i], p.H - c);
        } else if (p.quant == PMPE_QUANT_ROW) {
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = max_nan(amax, fabsf(v[i][j]));
        }
    }
    if (p.quant == PMPE_QUANT_NONE) return;
    Divide by = {0.f, 0.f};
    if (p.quant == PMPE_QUANT_ROW) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) amax = max_nan(amax, __shfl_xor_sync(~0u, amax, off));
        if (!kWarpRow) {
            if (lane == 0) s_max[threadIdx.x >> 5] = amax;
            __syncthreads();
            amax = lane < warps ? s_max[lane] : 0.f;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) amax = max_nan(amax, __shfl_xor_sync(~0u, amax, off));
        }
        float s;
        by = divide_by(amax, m, s);
        if (at.t == 0) p.scale[row] = s;
    }
    const int nb = (p.H + 127) / 128;
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        const int c = at.col(i), n = p.H - c;
        uint8_t *o = (uint8_t *)p.y + row * p.H + c;
        if (kVec) {
            if (p.quant == PMPE_QUANT_BLOCK) {  // 16 threads hold a block; columns past H hold zeros
                float a = 0.f, s;
#pragma unroll
                for (int j = 0; j < 8; ++j) a = max_nan(a, fabsf(v[i][j]));
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) a = max_nan(a, __shfl_xor_sync(~0u, a, off));
                by = divide_by(a, m, s);
                if ((at.t & 15) == 0 && n > 0) p.scale[row * nb + c / 128] = s;
            }
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = fmaf(v[i][j], by.hi, v[i][j] * by.lo);
            if (n > 0)
                *reinterpret_cast<uint2 *>(o) =
                    make_uint2(e4m3x2(e[0], e[1]) | e4m3x2(e[2], e[3]) << 16, e4m3x2(e[4], e[5]) | e4m3x2(e[6], e[7]) << 16);
        } else {
#pragma unroll
            for (int b = 0; b < 2; ++b) {  // a warp holds two blocks, four elements a lane each
                if (p.quant == PMPE_QUANT_BLOCK) {
                    float a = 0.f, s;
#pragma unroll
                    for (int j = 0; j < 4; ++j) a = max_nan(a, fabsf(v[i][4 * b + j]));
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) a = max_nan(a, __shfl_xor_sync(~0u, a, off));
                    by = divide_by(a, m, s);
                    if (lane == 0 && n > 128 * b) p.scale[row * nb + c / 128 + b] = s;
                }
#pragma unroll
                for (int j = 4 * b; j < 4 * b + 4; ++j)
                    if (32 * j < n) o[32 * j] = (uint8_t)e4m3x2(fmaf(v[i][j], by.hi, v[i][j] * by.lo), 0.f);
            }
        }
    }
}

// ------------------------------------------------------------- backward

struct NormBwdParams {
    const void *h, *dy, *d_h, *w;
    const float *rstd;
    void *dx;
    float *part;  // [CTAs, H] sums of dy h r over a CTA's rows; null: no dw
    int T, H, w_f32, dy_f32, dx_f32;
};

// Rows a grid apart, the next row's words requested before a row is reduced.
// A thread keeps its columns' sums of dy h r over all its rows in registers.
template <typename T, int kNC, bool kWarpRow, bool kVec, int kThreads>
__global__ void __launch_bounds__(kThreads) rms_norm_bwd_kernel(const NormBwdParams p)
{
    __shared__ float s_red[2][32];
    __shared__ float s_dw[kWarpRow ? kWarpRows * 256 * kNC : 1];
    pdl_trigger();
    pdl_wait();
    const Place<kWarpRow, kVec> at;
    const int warp = threadIdx.x >> 5;
    const long long step = kWarpRow ? (long long)gridDim.x * kWarpRows : (long long)gridDim.x;
    long long row = kWarpRow ? (long long)blockIdx.x * kWarpRows + warp : (long long)blockIdx.x;
    Raw8<T> rh[kNC];
    Raw8<float> rg[kNC], rd[kNC], rw[kNC];
    float r_next = 0.f;
    auto fetch = [&](long long q) {
        r_next = p.rstd[q];
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            const int c = at.col(i);
            load8<kVec>(rh[i], (const T *)p.h + q * p.H + c, p.H - c);
            load_any<kVec, T>(rg[i], p.dy, p.dy_f32, q * p.H + c, p.H - c);
            if (p.d_h) load_any<kVec, T>(rd[i], p.d_h, p.dx_f32, q * p.H + c, p.H - c);
        }
    };
    if (row < p.T) fetch(row);
    float acc[kNC][8];
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        load_any<kVec, T>(rw[i], p.w, p.w_f32, at.col(i), p.H - at.col(i));
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
    }
    for (int flip = 0; row < p.T; row += step, flip ^= 1) {
        const float r = r_next;
        const float2 r2 = make_float2(r, r);
        float h[kNC][8], g[kNC][8], d[kNC][8];
        float2 two = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            float w[8];
            unpack(rh[i], h[i]);
            unpack_any<T>(rg[i], p.dy_f32, g[i]);
            unpack_any<T>(rw[i], p.w_f32, w);
            if (p.d_h) unpack_any<T>(rd[i], p.dx_f32, d[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 n = mul2(pair(h[i], j), r2);  // the normed row
                set(acc[i], j, fma2(pair(g[i], j), n, pair(acc[i], j)));
                const float2 gw = mul2(pair(g[i], j), pair(w, j));
                two = fma2(gw, n, two);
                set(h[i], j, n);
                set(g[i], j, gw);
            }
        }
        if (row + step < p.T) fetch(row + step);
        // two buffers in turn: a warp may be a row ahead of the slowest reader
        const float m = row_sum<kWarpRow>(two.x + two.y, s_red[flip]) / (float)p.H;
        const float2 m2 = make_float2(-m, -m);
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            const int c = at.col(i);
            float o[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 q = fma2(pair(h[i], j), m2, pair(g[i], j));
                set(o, j, p.d_h ? fma2(q, r2, pair(d[i], j)) : mul2(q, r2));
            }
            if (p.dx_f32) store8<kVec>((float *)p.dx + row * p.H + c, o, p.H - c);
            else store8<kVec>((T *)p.dx + row * p.H + c, o, p.H - c);
        }
    }
    if (!p.part) return;
    float *part = p.part + (long long)blockIdx.x * p.H;
    if (kWarpRow) {  // the warps' sums in warp order
#pragma unroll
        for (int i = 0; i < kNC; ++i) store8<kVec>(s_dw + warp * 256 * kNC + at.col(i), acc[i], 256 * kNC - at.col(i));
        __syncthreads();
        for (int c = threadIdx.x; c < p.H; c += blockDim.x) {
            float a = 0.f;
#pragma unroll
            for (int q = 0; q < kWarpRows; ++q) a += s_dw[q * 256 * kNC + c];
            part[c] = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kNC; ++i) store8<kVec>(part + at.col(i), acc[i], p.H - at.col(i));
    }
}

// dw_c = the CTAs' partials of column c summed in a fixed order: kStrands
// strands of rows (a warp each), then the strands.
constexpr int kStrands = 32;
__global__ void __launch_bounds__(32 * kStrands) rms_norm_dw_kernel(const float *part, int n, int H, float *dw)
{
    __shared__ float s[kStrands][33];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float a = 0.f;
    if (c < H) {
#pragma unroll 8
        for (int i = strand; i < n; i += kStrands) a += part[(long long)i * H + c];
    }
    s[strand][lane] = a;
    __syncthreads();
    a = warp_sum(s[lane][strand]);  // column `strand` of the block
    if (lane == 0 && blockIdx.x * 32 + strand < H) dw[blockIdx.x * 32 + strand] = a;
}

// -------------------------------------------------------------- launches

// Up to 512 columns a warp takes a row, 8 or 16 columns a lane; above, a CTA
// does, 16 columns a thread.
constexpr int kWarpWidth = 512;
int threads_for(int H) { return H <= kWarpWidth ? 32 * kWarpRows : (H + 511) / 512 * 32; }
int ctas_for(int T, int H) { return H <= kWarpWidth ? (T + kWarpRows - 1) / kWarpRows : T; }

template <typename T, bool kVec> cudaError_t dispatch_fwd(const NormParams &p, cudaStream_t st)
{
    const int threads = threads_for(p.H), grid = ctas_for(p.T, p.H);
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(threads), 0, st, p); };
    if (p.H <= 256) return go(rms_norm_kernel<T, 1, true, kVec, 32 * kWarpRows>);
    if (p.H <= kWarpWidth) return go(rms_norm_kernel<T, 2, true, kVec, 32 * kWarpRows>);
    if (threads <= kMaxThreads) return go(rms_norm_kernel<T, 2, false, kVec, kMaxThreads>);
    return go(rms_norm_kernel<T, 2, false, kVec, 2 * kMaxThreads>);
}

// CTAs of the backward: 512 threads an SM of 152, what about 110 registers a
// thread allow.  Independent of the device, so that the workspace's size and
// the order of dw's sums are too.
int bwd_ctas(int T, int H) { return std::max(1, std::min(ctas_for(T, H), 152 * std::max(1, 512 / threads_for(H)))); }

template <typename T, bool kVec> cudaError_t dispatch_bwd(const NormBwdParams &p, cudaStream_t st)
{
    const int threads = threads_for(p.H), grid = bwd_ctas(p.T, p.H);
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(threads), 0, st, p); };
    if (p.H <= 256) return go(rms_norm_bwd_kernel<T, 1, true, kVec, 32 * kWarpRows>);
    if (p.H <= kWarpWidth) return go(rms_norm_bwd_kernel<T, 2, true, kVec, 32 * kWarpRows>);
    if (threads <= kMaxThreads) return go(rms_norm_bwd_kernel<T, 2, false, kVec, kMaxThreads>);
    return go(rms_norm_bwd_kernel<T, 2, false, kVec, 2 * kMaxThreads>);
}

bool multiple16(const void *q) { return ((uintptr_t)q & 15u) == 0; }

}  // namespace

cudaError_t launch_rms_norm(const pmpe_rms_norm_desc &d, cudaStream_t st)
{
    NormParams p;
    p.x = d.x; p.res = d.residual; p.w = d.weight; p.h = d.h; p.y = d.y; p.scale = d.scale; p.rstd = d.rstd;
    p.x_ld = d.x_ld; p.res_ld = d.residual_ld;
    p.T = d.T; p.H = d.H; p.w_f32 = d.weight_type == PMPE_F32; p.quant = d.quant;
    p.eps = d.eps;
    // 16-byte accesses: every row of every operand starts on a 16-byte
    // boundary and holds whole chunks (8-bit rows: an 8-byte boundary)
    const int per16 = d.type == PMPE_F32 ? 4 : 8;
    const bool vec = d.H % 8 == 0 && d.x_ld % per16 == 0 && (!d.residual || d.residual_ld % per16 == 0) &&
                     multiple16(d.x) && multiple16(d.residual) && multiple16(d.weight) && multiple16(d.h) && multiple16(d.y);
    if (d.type == PMPE_F32) return vec ? dispatch_fwd<float, true>(p, st) : dispatch_fwd<float, false>(p, st);
    if (d.type == PMPE_BF16) return vec ? dispatch_fwd<bf16, true>(p, st) : dispatch_fwd<bf16, false>(p, st);
    return vec ? dispatch_fwd<__half, true>(p, st) : dispatch_fwd<__half, false>(p, st);
}

size_t rms_norm_backward_workspace_bytes(int T, int H) { return (size_t)bwd_ctas(T, H) * H * sizeof(float); }

cudaError_t launch_rms_norm_backward(const pmpe_rms_norm_backward_desc &d, float *part, cudaStream_t st)
{
    NormBwdParams p;
    p.h = d.h; p.dy = d.dy; p.d_h = d.d_h; p.w = d.weight; p.rstd = d.rstd; p.dx = d.dx;
    p.part = d.dw ? part : nullptr;
    p.T = d.T; p.H = d.H; p.w_f32 = d.weight_type == PMPE_F32; p.dy_f32 = d.dy_type == PMPE_F32;
    p.dx_f32 = d.dx_type == PMPE_F32;
    const bool vec = d.H % 8 == 0 && multiple16(d.dy) && multiple16(d.h) && multiple16(d.weight) && multiple16(d.d_h) &&
                     multiple16(d.dx) && multiple16(part);
    cudaError_t err;
    if (d.type == PMPE_F32) err = vec ? dispatch_bwd<float, true>(p, st) : dispatch_bwd<float, false>(p, st);
    else if (d.type == PMPE_BF16) err = vec ? dispatch_bwd<bf16, true>(p, st) : dispatch_bwd<bf16, false>(p, st);
    else err = vec ? dispatch_bwd<__half, true>(p, st) : dispatch_bwd<__half, false>(p, st);
    if (err != cudaSuccess || !d.dw) return err;
    return launch_pdl(rms_norm_dw_kernel, dim3((d.H + 31) / 32), dim3(32 * kStrands), 0, st, (const float *)part,
                      bwd_ctas(d.T, d.H), d.H, d.dw);
}

}  // namespace pmpe
