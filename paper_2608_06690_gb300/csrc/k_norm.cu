// Root-mean-square norm of the residual stream with the residual's addition,
// optionally into 8 bits with scales (its backward: k_norm_bwd.cu).
//
//   h = round(x + residual)            (x itself without a residual)
//   r = 1 / sqrt(mean_c h_c^2 + eps)
//   y = h r w                          in the input's type, or
//   s = max(amax |y| / 448, 2^-126),  q = e4m3(y / s)   per 128 columns or per row,
//   the quotient by s before its rounding to FP32
//
// h is rounded to its type before the norm, so that the backward, which reads
// the stored h, differentiates what the forward computed.  Everything between
// the loads and the stores is FP32.
//
// Bytes bound it (16384 x 2048 BF16: 40.5 us, 6.6 TB/s; into e4m3, T = 4096,
// 12.6 us where the bytes take 8.7, start and end the rest), instructions
// follow (a row of 2048 columns is 8 KB in and 8 KB out): 16-bit sums take two
// elements an instruction, and a thread holds 16 columns, so that the row's sum
// over the threads is a small part.  (Two FP32 products an instruction, f32x2,
// changed nothing; CTAs that go on to further rows, the next one's loads ahead,
// took 14.6 to 17.7 us for the 12.6.)
#include <algorithm>

#include <cuda_fp8.h>

#include "norm_rows.cuh"

namespace pmpe {
namespace {

constexpr int kWarpRows = 8;      // rows of a CTA where a warp takes a row
constexpr int kMaxThreads = 512;  // of a CTA that takes a row of up to 8192 columns; twice that above

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
// For values u of a block whose largest is amax in magnitude and which stand
// for u m: the scale s = max(amax m / 448, 2^-126) and the factor u -> u m / s.
__device__ __forceinline__ Divide divide_by(float amax, float m, float &s)
{
    amax = fabsf(amax);
    s = max_nan(amax * m * (1.f / 448.f), kMinScale);
    if (!(s > kMinScale)) return {m * 0x1p126f, 0.f};  // zeros (or NaN)
    // the product's remainder is exact in one fused operation
    const float inv = __frcp_rn(amax), hi = 448.f * inv;
    return {hi, hi > 0.f ? fmaf(-hi, amax, 448.f) * inv : 0.f};
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

// kQuant: y in 8 bits, by p.quant.  (One kernel for both took 52 registers in
// place of 40 and 47: e4m3, T = 4096 13.0 us, apart 12.6.)
template <typename T, int kNC, bool kWarpRow, bool kVec, int kThreads, bool kQuant>
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
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        unpack(rx[i], v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += v[i][j] * v[i][j];
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
    if (p.rstd && at.t == 0) p.rstd[row] = r;
    // An 8-bit y divides by its block's largest value, and r cancels: only
    // the power of two of r enters y here (exact, and it keeps the products
    // in range), its significand m goes to the scale alone.
    float pre = r, m = 1.f;
    if (kQuant && r >= kMinScale) {
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
        for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * pre * w[j];
        if (!kQuant) {
            store8<kVec>((T *)p.y + row * p.H + c, v[i], p.H - c);
        } else if (p.quant == PMPE_QUANT_ROW) {
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = max_magnitude(amax, v[i][j]);
        }
    }
    if (!kQuant) return;
    Divide by = {0.f, 0.f};
    if (p.quant == PMPE_QUANT_ROW) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) amax = max_magnitude(amax, __shfl_xor_sync(~0u, amax, off));
        if (!kWarpRow) {
            if (lane == 0) s_max[threadIdx.x >> 5] = amax;
            __syncthreads();
            amax = lane < warps ? s_max[lane] : 0.f;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) amax = max_magnitude(amax, __shfl_xor_sync(~0u, amax, off));
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
                for (int j = 0; j < 8; ++j) a = max_magnitude(a, v[i][j]);
#pragma unroll
                for (int off = 8; off > 0; off >>= 1) a = max_magnitude(a, __shfl_xor_sync(~0u, a, off));
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
                    for (int j = 0; j < 4; ++j) a = max_magnitude(a, v[i][4 * b + j]);
#pragma unroll
                    for (int off = 16; off > 0; off >>= 1) a = max_magnitude(a, __shfl_xor_sync(~0u, a, off));
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

// -------------------------------------------------------------- launches

// Up to 512 columns a warp takes a row, 8 or 16 columns a lane; above, a CTA
// does, 16 columns a thread.
constexpr int kWarpWidth = 512;
int threads_for(int H) { return H <= kWarpWidth ? 32 * kWarpRows : (H + 511) / 512 * 32; }
int ctas_for(int T, int H) { return H <= kWarpWidth ? (T + kWarpRows - 1) / kWarpRows : T; }

template <typename T, bool kVec, bool kQuant> cudaError_t dispatch_q(const NormParams &p, cudaStream_t st)
{
    const int threads = threads_for(p.H), grid = ctas_for(p.T, p.H);
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(threads), 0, st, p); };
    if (p.H <= 256) return go(rms_norm_kernel<T, 1, true, kVec, 32 * kWarpRows, kQuant>);
    if (p.H <= kWarpWidth) return go(rms_norm_kernel<T, 2, true, kVec, 32 * kWarpRows, kQuant>);
    if (threads <= kMaxThreads) return go(rms_norm_kernel<T, 2, false, kVec, kMaxThreads, kQuant>);
    return go(rms_norm_kernel<T, 2, false, kVec, 2 * kMaxThreads, kQuant>);
}

template <typename T, bool kVec> cudaError_t dispatch_fwd(const NormParams &p, cudaStream_t st)
{
    return p.quant == PMPE_QUANT_NONE ? dispatch_q<T, kVec, false>(p, st) : dispatch_q<T, kVec, true>(p, st);
}

}  // namespace

cudaError_t launch_rms_norm(const pmpe_rms_norm_desc &d, cudaStream_t st)
{
    NormParams p;
    p.x = d.x; p.res = d.residual; p.w = d.weight; p.h = d.h; p.y = d.y; p.scale = d.scale; p.rstd = d.rstd;
    p.x_ld = d.x_ld; p.res_ld = d.residual_ld;
    p.T = d.T; p.H = d.H; p.w_f32 = d.weight_type == PMPE_F32; p.quant = d.quant;
    p.eps = d.eps;
    // eight elements an access: every row of every operand is aligned for it
    // and holds whole chunks (8-bit rows: 8 bytes)
    const bool f32 = d.type == PMPE_F32;
    const bool vec = d.H % 8 == 0 && d.x_ld % 8 == 0 && (!d.residual || d.residual_ld % 8 == 0) && aligned8(d.x, f32) &&
                     aligned8(d.residual, f32) && aligned8(d.weight, p.w_f32) && aligned8(d.h, f32) &&
                     aligned8(d.y, f32 && d.quant == PMPE_QUANT_NONE);
    if (d.type == PMPE_F32) return vec ? dispatch_fwd<float, true>(p, st) : dispatch_fwd<float, false>(p, st);
    if (d.type == PMPE_BF16) return vec ? dispatch_fwd<bf16, true>(p, st) : dispatch_fwd<bf16, false>(p, st);
    return vec ? dispatch_fwd<__half, true>(p, st) : dispatch_fwd<__half, false>(p, st);
}

}  // namespace pmpe
