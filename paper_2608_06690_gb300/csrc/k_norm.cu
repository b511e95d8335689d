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
// Bytes bound both: a forward row is loaded once into registers (eight
// elements a thread and chunk), reduced and written.
#include <algorithm>

#include <cuda_fp8.h>

#include "elem.cuh"

namespace pmpe {
namespace {

constexpr int kWarpRows = 8;  // rows of a CTA where a warp takes a row

struct NormParams {
    const void *x, *res, *w;
    void *h, *y;
    float *scale, *rstd;
    long long x_ld, res_ld;
    int T, H, w_f32, quant;  // quant: PMPE_QUANT_*
    float eps;
};

// The sum over the row's threads, in every one of them, in a fixed order:
// a warp's row by shuffles, a CTA's row through s_red (one entry a warp).
template <bool kWarpRow, typename V> __device__ __forceinline__ V row_sum(V v, V *s_red)
{
    v = warp_sum(v);
    if (kWarpRow) return v;
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0) s_red[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum(lane < warps ? s_red[lane] : V(0));
}

template <bool kVec> __device__ __forceinline__ void load_weight(float (&v)[8], const void *w, int f32, long long at, int n,
                                                                  bf16)
{
    if (f32) {
        Raw8<float> r;
        load8<kVec>(r, (const float *)w + at, n);
        unpack(r, v);
    } else {
        Raw8<bf16> r;
        load8<kVec>(r, (const bf16 *)w + at, n);
        unpack(r, v);
    }
}
template <bool kVec> __device__ __forceinline__ void load_weight(float (&v)[8], const void *w, int f32, long long at, int n,
                                                                  __half)
{
    if (f32) {
        Raw8<float> r;
        load8<kVec>(r, (const float *)w + at, n);
        unpack(r, v);
    } else {
        Raw8<__half> r;
        load8<kVec>(r, (const __half *)w + at, n);
        unpack(r, v);
    }
}
template <bool kVec> __device__ __forceinline__ void load_weight(float (&v)[8], const void *w, int, long long at, int n,
                                                                  float)
{
    Raw8<float> r;
    load8<kVec>(r, (const float *)w + at, n);
    unpack(r, v);
}

// A thread holds kNC chunks of eight consecutive elements: chunk i of thread
// t is columns 8 (i G + t) .. + 7, G the row's threads, so a warp's accesses
// are contiguous and 16 neighbouring threads hold one 128-column block.
template <typename T, int kNC, bool kWarpRow, bool kVec>
__global__ void __launch_bounds__(kWarpRow ? 32 * kWarpRows : 1024) rms_norm_kernel(const NormParams p)
{
    __shared__ double s_red64[32];
    __shared__ float s_red[32], s_max[32];
    pdl_trigger();
    pdl_wait();
    const int G = kWarpRow ? 32 : (int)blockDim.x, t = kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
    const int row = kWarpRow ? (int)blockIdx.x * kWarpRows + (int)(threadIdx.x >> 5) : (int)blockIdx.x;
    if (row >= p.T) return;  // a whole warp; a CTA's row always exists
    const T *x = (const T *)p.x + row * p.x_ld;
    Raw8<T> rx[kNC], rr[kNC];
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        const int c = 8 * (i * G + t);
        load8<kVec>(rx[i], x + c, p.H - c);
    }
    if (p.res) {
        const T *res = (const T *)p.res + row * p.res_ld;
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            const int c = 8 * (i * G + t);
            load8<kVec>(rr[i], res + c, p.H - c);
        }
    }
    float v[kNC][8];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        unpack(rx[i], v[i]);
        if (p.res) {
            float a[8];
            unpack(rr[i], a);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = to_f32(from_f32<T>(v[i][j] + a[j]));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += v[i][j] * v[i][j];
    }
    if (p.h) {
        T *h = (T *)p.h + (long long)row * p.H;
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            const int c = 8 * (i * G + t);
            store8<kVec>(h + c, v[i], p.H - c);
        }
    }
    ss = row_sum<kWarpRow>(ss, s_red);
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
    if (p.rstd && t == 0) p.rstd[row] = r;
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        const int c = 8 * (i * G + t);
        float w[8];
        load_weight<kVec>(w, p.w, p.w_f32, c, p.H - c, T());
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[i][j] *= r;
            v[i][j] *= w[j];
        }
        if (p.quant == PMPE_QUANT_NONE) {
            store8<kVec>((T *)p.y + (long long)row * p.H + c, v[i], p.H - c);
        } else if (p.quant == PMPE_QUANT_ROW) {
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = max_nan(amax, fabsf(v[i][j]));
        }
    }
    if (p.quant == PMPE_QUANT_NONE) return;
    float s = 0.f;
    if (p.quant == PMPE_QUANT_ROW) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) amax = max_nan(amax, __shfl_xor_sync(~0u, amax, off));
        if (!kWarpRow) {
            const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
            if (lane == 0) s_max[threadIdx.x >> 5] = amax;
            __syncthreads();
            amax = lane < warps ? s_max[lane] : 0.f;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) amax = max_nan(amax, __shfl_xor_sync(~0u, amax, off));
        }
        s = max_nan(amax / 448.f, 1.17549435e-38f);
        if (t == 0) p.scale[row] = s;
    }
    const int nb = (p.H + 127) / 128;
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        const int c = 8 * (i * G + t), n = p.H - c;
        if (p.quant == PMPE_QUANT_BLOCK) {  // columns past H hold zeros
            float m = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max_nan(m, fabsf(v[i][j]));
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) m = max_nan(m, __shfl_xor_sync(~0u, m, off));
            s = max_nan(m / 448.f, 1.17549435e-38f);
            if ((t & 15) == 0 && n > 0) p.scale[(long long)row * nb + c / 128] = s;
        }
        // y / s as y times the rounded reciprocal: two roundings of 2^-24 in
        // place of one, beside e4m3's 2^-4
        const float inv = 1.f / s;
        uint32_t q[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[i][4 * j] * inv, v[i][4 * j + 1] * inv),
                                                         __NV_SATFINITE, __NV_E4M3);
            const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[i][4 * j + 2] * inv, v[i][4 * j + 3] * inv),
                                                         __NV_SATFINITE, __NV_E4M3);
            q[j] = lo | hi << 16;
        }
        uint8_t *o = (uint8_t *)p.y + (long long)row * p.H + c;
        if (kVec) {
            if (n > 0) *reinterpret_cast<uint2 *>(o) = make_uint2(q[0], q[1]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) o[j] = (uint8_t)(q[j >> 2] >> 8 * (j & 3));
        }
    }
}

// ------------------------------------------------------------- backward

struct NormBwdParams {
    const void *dy, *h, *w, *d_h;
    const float *rstd;
    void *dx;
    float *part;  // [CTAs, H] sums of dy h r over a CTA's rows
    int T, H, w_f32, dy_f32, dx_f32;
};

template <bool kVec, typename T> __device__ __forceinline__ void load_either(float (&v)[8], const void *p, int f32,
                                                                              long long at, int n)
{
    if (f32) {
        Raw8<float> r;
        load8<kVec>(r, (const float *)p + at, n);
        unpack(r, v);
    } else {
        Raw8<T> r;
        load8<kVec>(r, (const T *)p + at, n);
        unpack(r, v);
    }
}

// Rows blockIdx.x, blockIdx.x + gridDim.x, ... (kWarpRow: kWarpRows of them at
// a time, a warp each).  A thread keeps its columns' sums of dy h r over all
// its rows in registers.
template <typename T, int kNC, bool kWarpRow, bool kVec>
__global__ void __launch_bounds__(kWarpRow ? 32 * kWarpRows : 1024) rms_norm_bwd_kernel(const NormBwdParams p)
{
    __shared__ float s_red[2][32];
    __shared__ float s_dw[kWarpRow ? kWarpRows * kNC * 256 : 1];
    pdl_trigger();
    pdl_wait();
    const int G = kWarpRow ? 32 : (int)blockDim.x, t = kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    float w[kNC][8], acc[kNC][8];
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        const int c = 8 * (i * G + t);
        load_weight<kVec>(w[i], p.w, p.w_f32, c, p.H - c, T());
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
    }
    const int step = kWarpRow ? (int)gridDim.x * kWarpRows : (int)gridDim.x;
    int flip = 0;
    for (int row = kWarpRow ? (int)blockIdx.x * kWarpRows + warp : (int)blockIdx.x; row < p.T; row += step, flip ^= 1) {
        const long long at = (long long)row * p.H;
        const float r = p.rstd[row];
        float h[kNC][8], g[kNC][8], d[kNC][8];
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            const int c = 8 * (i * G + t);
            load_either<kVec, T>(h[i], p.h, 0, at + c, p.H - c);
            load_either<kVec, T>(g[i], p.dy, p.dy_f32, at + c, p.H - c);
            if (p.d_h) load_either<kVec, T>(d[i], p.d_h, p.dx_f32, at + c, p.H - c);
        }
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < kNC; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[i][j] *= r;  // the normed row
                acc[i][j] += g[i][j] * h[i][j];
                g[i][j] *= w[i][j];
                m += g[i][j] * h[i][j];
            }
        m = warp_sum(m);
        if (!kWarpRow) {  // two buffers: a warp may be a row ahead of the slowest reader
            if (lane == 0) s_red[flip][warp] = m;
            __syncthreads();
            m = warp_sum(lane < warps ? s_red[flip][lane] : 0.f);
        }
        m /= (float)p.H;
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            const int c = 8 * (i * G + t);
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = r * (g[i][j] - h[i][j] * m);
                if (p.d_h) o[j] += d[i][j];
            }
            if (p.dx_f32) store8<kVec>((float *)p.dx + at + c, o, p.H - c);
            else store8<kVec>((T *)p.dx + at + c, o, p.H - c);
        }
    }
    if (!p.part) return;
    float *part = p.part + (long long)blockIdx.x * p.H;
    if (kWarpRow) {  // the warps' sums in warp order
#pragma unroll
        for (int i = 0; i < kNC; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s_dw[warp * kNC * 256 + 8 * (i * 32 + t) + j] = acc[i][j];
        __syncthreads();
        for (int c = threadIdx.x; c < p.H; c += blockDim.x) {
            float a = 0.f;
#pragma unroll
            for (int q = 0; q < kWarpRows; ++q) a += s_dw[q * kNC * 256 + c];
            part[c] = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            const int c = 8 * (i * G + t);
            if (kVec) {
                store8<true>(part + c, acc[i], p.H - c);
            } else {
                store8<false>(part + c, acc[i], p.H - c);
            }
        }
    }
}

// dw_c = the CTAs' partials of column c summed in a fixed order: eight
// strands of rows (a warp each), then the strands.
__global__ void __launch_bounds__(256) rms_norm_dw_kernel(const float *part, int n, int H, float *dw)
{
    __shared__ float s[8][32];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, strand = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float a = 0.f;
    if (c < H) {
#pragma unroll 8
        for (int i = strand; i < n; i += 8) a += part[(long long)i * H + c];
    }
    s[strand][lane] = a;
    __syncthreads();
    if (strand == 0 && c < H) {
        float b = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) b += s[i][lane];
        dw[c] = b;
    }
}

// Rows per CTA's worth of SMs that the backward's grid holds at most.
constexpr int kBwdCtasPerSm = 4;

template <typename T, int kNC, bool kWarpRow, bool kVec>
cudaError_t launch_fwd(const NormParams &p, int threads, cudaStream_t st)
{
    const int grid = kWarpRow ? (p.T + kWarpRows - 1) / kWarpRows : p.T;
    return launch_pdl(rms_norm_kernel<T, kNC, kWarpRow, kVec>, dim3(grid), dim3(threads), 0, st, p);
}

template <typename T> cudaError_t dispatch_fwd(const NormParams &p, bool vec, cudaStream_t st)
{
    const int chunks = (p.H + 7) / 8;
    if (vec && p.T >= 1024 && chunks <= 256) {
        const int threads = 32 * kWarpRows;
        if (chunks <= 32) return launch_fwd<T, 1, true, true>(p, threads, st);
        if (chunks <= 64) return launch_fwd<T, 2, true, true>(p, threads, st);
        if (chunks <= 128) return launch_fwd<T, 4, true, true>(p, threads, st);
        return launch_fwd<T, 8, true, true>(p, threads, st);
    }
    auto threads = [&](int nc) { return std::max(32, (chunks + 32 * nc - 1) / (32 * nc) * 32); };
    if (chunks <= 1024) return vec ? launch_fwd<T, 1, false, true>(p, threads(1), st) : launch_fwd<T, 1, false, false>(p, threads(1), st);
    return vec ? launch_fwd<T, 2, false, true>(p, threads(2), st) : launch_fwd<T, 2, false, false>(p, threads(2), st);
}

template <typename T, int kNC, bool kWarpRow, bool kVec>
cudaError_t launch_bwd(const NormBwdParams &p, int grid, int threads, cudaStream_t st)
{
    return launch_pdl(rms_norm_bwd_kernel<T, kNC, kWarpRow, kVec>, dim3(grid), dim3(threads), 0, st, p);
}

template <typename T> cudaError_t dispatch_bwd(const NormBwdParams &p, bool vec, int grid, cudaStream_t st)
{
    const int chunks = (p.H + 7) / 8;
    if (chunks <= 32) {
        const int threads = 32 * kWarpRows;
        return vec ? launch_bwd<T, 1, true, true>(p, grid, threads, st) : launch_bwd<T, 1, true, false>(p, grid, threads, st);
    }
    auto threads = [&](int nc) { return (chunks + 32 * nc - 1) / (32 * nc) * 32; };
    if (chunks <= 1024) return vec ? launch_bwd<T, 1, false, true>(p, grid, threads(1), st) : launch_bwd<T, 1, false, false>(p, grid, threads(1), st);
    return vec ? launch_bwd<T, 2, false, true>(p, grid, threads(2), st) : launch_bwd<T, 2, false, false>(p, grid, threads(2), st);
}

// CTAs of the backward: independent of the device, so that the workspace's
// size and the order of dw's sums are too.
constexpr int kBwdMaxCtas = 152 * kBwdCtasPerSm;

int bwd_ctas(int T, int H)
{
    const int rows = (H + 7) / 8 <= 32 ? kWarpRows : 1;
    return std::max(1, std::min((T + rows - 1) / rows, kBwdMaxCtas));
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
    if (d.type == PMPE_F32) return dispatch_fwd<float>(p, vec, st);
    if (d.type == PMPE_BF16) return dispatch_fwd<bf16>(p, vec, st);
    return dispatch_fwd<__half>(p, vec, st);
}

size_t rms_norm_backward_workspace_bytes(int T, int H) { return (size_t)bwd_ctas(T, H) * H * sizeof(float); }

cudaError_t launch_rms_norm_backward(const pmpe_rms_norm_backward_desc &d, float *part, cudaStream_t st)
{
    NormBwdParams p;
    p.dy = d.dy; p.h = d.h; p.w = d.weight; p.d_h = d.d_h; p.rstd = d.rstd; p.dx = d.dx;
    p.part = d.dw ? part : nullptr;
    p.T = d.T; p.H = d.H; p.w_f32 = d.weight_type == PMPE_F32; p.dy_f32 = d.dy_type == PMPE_F32;
    p.dx_f32 = d.dx_type == PMPE_F32;
    const bool vec = d.H % 8 == 0 && multiple16(d.dy) && multiple16(d.h) && multiple16(d.weight) && multiple16(d.d_h) &&
                     multiple16(d.dx) && multiple16(part);
    const int grid = bwd_ctas(d.T, d.H);
    cudaError_t err;
    if (d.type == PMPE_F32) err = dispatch_bwd<float>(p, vec, grid, st);
    else if (d.type == PMPE_BF16) err = dispatch_bwd<bf16>(p, vec, grid, st);
    else err = dispatch_bwd<__half>(p, vec, grid, st);
    if (err != cudaSuccess || !d.dw) return err;
    return launch_pdl(rms_norm_dw_kernel, dim3((d.H + 31) / 32), dim3(256), 0, st, (const float *)part, grid, d.H, d.dw);
}

}  // namespace pmpe
