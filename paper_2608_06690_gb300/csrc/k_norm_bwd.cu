// Backward of the root-mean-square norm (k_norm.cu): with r the rows' stored
// 1 / sqrt(mean h^2 + eps),
//
//   n = h r,  g = dy w,  m = mean_c g_c n_c
//   dx = d_h + r (g - n m)             (d_h: the gradient that reaches h itself)
//   dw_c = sum_t dy_{t,c} n_{t,c}
//
// FP32 throughout.  Bytes bound it, and close to them the instructions of a
// row, so types are template parameters and a thread's pointers only advance.
// A CTA takes a row, 8 columns a thread up to 6144 columns (up to 256 columns a
// warp does, eight of them a CTA), and goes on to the rows a grid further, the next of which is
// on its way into registers meanwhile.  16 columns a thread need more than 128
// registers for that and spill (27 us where 8 columns take 20).  Bytes that a
// thread spills: up to 256 columns 0 to 32 (48 to 84 where accesses are element
// by element and a type is FP32), from 6145 columns 0 to 64 (8 to 144), above
// 8192, where 1024 threads have 64 registers each, 476 to 700; FP32 rows of odd
// width 16 elsewhere.
#include <algorithm>

#include "norm_rows.cuh"

namespace pmpe {
namespace {

constexpr int kSms = 152;     // the grid does not go by the device: dw's sums keep their order
constexpr int kWarpRows = 8;  // rows of a CTA where a warp takes a row

struct NormBwdParams {
    const void *h, *dy, *d_h, *w;
    const float *rstd;
    void *dx;
    float *part;  // [CTAs, H] sums of dy n over a CTA's rows; null: no dw
    int T, H, w_f32;
};

// T: h, G: dy, X: dx and d_h.
template <typename T, typename G, typename X, int kNC, bool kWarpRow, bool kVec, int kThreads, int kCtas>
__global__ void __launch_bounds__(kThreads, kCtas) rms_norm_bwd_kernel(const NormBwdParams p)
{
    __shared__ float s_red[2][32];
    __shared__ float s_dw[kWarpRow ? kWarpRows * 256 * kNC : 1];
    pdl_wait();  // no early trigger: the sums' CTAs would take this grid's place (18.4 us, without 18.1)
    const Place<kWarpRow, kVec> at;
    const int warp = threadIdx.x >> 5;
    const long long step = kWarpRow ? (long long)gridDim.x * kWarpRows : (long long)gridDim.x;
    long long row = kWarpRow ? (long long)blockIdx.x * kWarpRows + warp : (long long)blockIdx.x;
    // chunk i is `apart` columns after the first, n[i] of its elements exist
    const int c0 = at.col(0), apart = at.col(1) - c0;
    int n[kNC];
#pragma unroll
    for (int i = 0; i < kNC; ++i) n[i] = p.H - c0 - i * apart;
    const long long first = row * p.H + c0, advance = step * p.H;
    const T *h_at = (const T *)p.h + first;
    const G *g_at = (const G *)p.dy + first;
    const X *d_at = p.d_h ? (const X *)p.d_h + first : nullptr;
    X *x_at = (X *)p.dx + first;
    Raw8<T> rh[kNC];
    Raw8<G> rg[kNC];
    Raw8<X> rd[kNC];
    float r_next = 0.f;
    auto fetch = [&](long long q) {
        r_next = p.rstd[q];
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            load8<kVec>(rh[i], h_at + i * apart, n[i]);
            load8<kVec>(rg[i], g_at + i * apart, n[i]);
            if (d_at) load8<kVec>(rd[i], d_at + i * apart, n[i]);
        }
        h_at += advance;
        g_at += advance;
        if (d_at) d_at += advance;
    };
    if (row < p.T) fetch(row);
    float acc[kNC][8], w[kNC][8];
#pragma unroll
    for (int i = 0; i < kNC; ++i) {
        Raw8<float> rw;
        load_any<kVec, T>(rw, p.w, p.w_f32, c0 + i * apart, n[i]);
        unpack_any<T>(rw, p.w_f32, w[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
    }
    const float inv_h = 1.f / (float)p.H;
    for (int flip = 0; row < p.T; row += step, flip ^= 1) {
        const float r = r_next;
        float h[kNC][8], g[kNC][8], d[kNC][8];
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            unpack(rh[i], h[i]);
            unpack(rg[i], g[i]);
            if (d_at) unpack(rd[i], d[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[i][j] *= r;
                acc[i][j] += g[i][j] * h[i][j];
                g[i][j] *= w[i][j];
                m += g[i][j] * h[i][j];
            }
        }
        if (row + step < p.T) fetch(row + step);
        m = warp_sum(m);
        if (!kWarpRow) {  // two buffers in turn: a warp may be a row ahead of the slowest reader
            const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
            if (lane == 0) s_red[flip][warp] = m;
            __syncthreads();
            m = warp_sum(lane < warps ? s_red[flip][lane] : 0.f);
        }
        m *= inv_h;
#pragma unroll
        for (int i = 0; i < kNC; ++i) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = g[i][j] - h[i][j] * m;
            if (d_at) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = r * o[j] + d[i][j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] *= r;
            }
            store8<kVec>(x_at + i * apart, o, n[i]);
        }
        x_at += advance;
    }
    if (!p.part) return;
    float *part = p.part + (long long)blockIdx.x * p.H;
    if (kWarpRow) {  // the warps' sums in warp order
#pragma unroll
        for (int i = 0; i < kNC; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int q = kVec ? j : 32 * j;
                if (q < n[i]) s_dw[warp * 256 * kNC + c0 + i * apart + q] = acc[i][j];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < p.H; c += blockDim.x) {
            float a = 0.f;
#pragma unroll
            for (int q = 0; q < kWarpRows; ++q) a += s_dw[q * 256 * kNC + c];
            part[c] = a;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kNC; ++i) store8<kVec>(part + c0 + i * apart, acc[i], n[i]);
    }
}

// dw_c = the CTAs' partials of column c summed in a fixed order: kStrands
// strands of rows, kDeep of them on the way at once, then the strands.  16
// columns a CTA spread the sums over the SMs (T = 4096, 2048 columns, the whole
// backward: 17.2 us, with 32 columns 17.9, with 8 17.2; a loop that loads one
// row after another where fewer than kDeep are left 18.1).
// pair: null, or [2, H], the sum of the earlier row blocks and what its
// roundings lost, to which this block's sum is added; dw then is written with
// the last block.
constexpr int kDwCols = 16, kStrands = 1024 / kDwCols, kDeep = 8;
__global__ void __launch_bounds__(kDwCols * kStrands) rms_norm_dw_kernel(const float *part, int n, int H, float *dw, float *pair,
                                                                       int first, int last)
{
    __shared__ float s[kStrands][kDwCols + 1];
    pdl_trigger();
    pdl_wait();
    const int strand = threadIdx.x / kDwCols, col = threadIdx.x % kDwCols, c = blockIdx.x * kDwCols + col;
    float a = 0.f;
    for (int i = strand; i < n; i += kDeep * kStrands) {
        float v[kDeep];
#pragma unroll
        for (int q = 0; q < kDeep; ++q) v[q] = c < H && i + q * kStrands < n ? part[(long long)(i + q * kStrands) * H + c] : 0.f;
#pragma unroll
        for (int q = 0; q < kDeep; ++q) a += v[q];
    }
    s[strand][col] = a;
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (warp < kDwCols) {  // a warp a column
        a = 0.f;
#pragma unroll
        for (int q = 0; q < kStrands; q += 32) a += s[q + lane][warp];
        a = warp_sum(a);
        const int at = blockIdx.x * kDwCols + warp;
        if (lane == 0 && at < H) {
            if (pair) {
                const float hi = first ? 0.f : pair[at], lo = first ? 0.f : pair[H + at];
                const float sum = hi + a, bb = sum - hi, lost = lo + ((hi - (sum - bb)) + (a - bb));
                a = sum + lost;
                pair[at] = sum;
                pair[H + at] = lost;
            }
            if (last) dw[at] = a;
        }
    }
}

// Threads of a CTA, and the CTAs that an SM holds: 768 threads at 80 registers
// (T = 4096, 2048 columns, BF16 with an FP32 dy: 18.6 us (17.2 now), with 512 19.9, with
// 1024 at 64 registers 21.3); wider rows' kernels take about 96, from 6145
// columns on, with 16 columns a thread, 128.  A grid beyond them would run its
// last CTAs in a second wave.  T = 3276, 5120 columns, BF16: 32.4 us
// with 8 columns, 43.5 with 16 (now, with 8 columns and d_h, 34.5 with an FP32
// dy and 42.7 with a BF16 one).  At 6400 to 8192 columns, 16 columns against 8
// (1024 threads at 64 registers): FP32 rows 55 to 58 us against 60 to 63 (45 to 48
// and 49 to 50 without d_h), BF16 rows 27 to 28 against 29 to 30 without d_h, but
// 35 to 36 against 32 to 33 with it (FP32 dy 40 to 42, 38 to 39): one rule for
// all, as the kernels of 8 columns would be as many again.
int sm_threads(int H) { return H <= 2048 ? 768 : H <= 4096 ? 640 : 512; }
int threads_for(int H)
{
    if (H <= 256) return 32 * kWarpRows;
    const int columns = H <= 6144 ? 256 : 512;  // a warp's
    return (H + columns - 1) / columns * 32;
}
int bwd_ctas(int T, int H)
{
    const int rows = H <= 256 ? kWarpRows : 1;
    return std::max(1, std::min((T + rows - 1) / rows, kSms * std::max(1, sm_threads(H) / threads_for(H))));
}

// Rows of a launch at most: a thread sums its rows' part of dw one after
// another, kChain of them, so that dw's error does not grow with T.  (Pairs
// kept in the row kernel, joined every 64 rows, took its registers: 60000 x
// 2048 194 -> 208 us, 1000 x 16384 77 -> 88.)
constexpr int kChain = 256;
long long block_rows(int H) { return (long long)kChain * bwd_ctas(1 << 30, H) * (H <= 256 ? kWarpRows : 1); }

template <typename T, typename G, typename X, bool kVec> cudaError_t launch(const NormBwdParams &p, cudaStream_t st)
{
    const int threads = threads_for(p.H), grid = bwd_ctas(p.T, p.H);
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(threads), 0, st, p); };
    if (p.H <= 256) return go(rms_norm_bwd_kernel<T, G, X, 1, true, kVec, 32 * kWarpRows, 3>);
    if (threads <= 256) return go(rms_norm_bwd_kernel<T, G, X, 1, false, kVec, 256, 3>);
    if (threads <= 512 && p.H <= 4096) return go(rms_norm_bwd_kernel<T, G, X, 1, false, kVec, 512, 1>);
    if (p.H <= 6144) return go(rms_norm_bwd_kernel<T, G, X, 1, false, kVec, 768, 1>);
    if (threads <= 512) return go(rms_norm_bwd_kernel<T, G, X, 2, false, kVec, 512, 1>);
    return go(rms_norm_bwd_kernel<T, G, X, 2, false, kVec, 1024, 1>);
}

template <typename T, bool kVec> cudaError_t by_types(const NormBwdParams &p, bool g32, bool x32, cudaStream_t st)
{
    if (g32) return x32 ? launch<T, float, float, kVec>(p, st) : launch<T, float, T, kVec>(p, st);
    return x32 ? launch<T, T, float, kVec>(p, st) : launch<T, T, T, kVec>(p, st);
}

}  // namespace

// The partial sums, aligned for eight of them at a time wherever the workspace
// starts (what is computed how does not depend on its address), and the row
// blocks' pair.
constexpr size_t kPartAlign = 32, kWorkspaceAlign = 16;
size_t rms_norm_backward_workspace_bytes(int T, int H)
{
    return ((size_t)bwd_ctas(T, H) + (T > block_rows(H) ? 2 : 0)) * H * sizeof(float) + (kPartAlign - kWorkspaceAlign);
}

cudaError_t launch_rms_norm_backward(const pmpe_rms_norm_backward_desc &d, cudaStream_t st)
{
    float *part = reinterpret_cast<float *>(((uintptr_t)d.workspace + (kPartAlign - 1)) & ~(uintptr_t)(kPartAlign - 1));
    const bool g32 = d.dy_type == PMPE_F32, x32 = d.dx_type == PMPE_F32, h32 = d.type == PMPE_F32, w32 = d.weight_type == PMPE_F32;
    // eight elements an access where every row of every operand allows it
    const bool vec = d.H % 8 == 0 && aligned8(d.dy, g32) && aligned8(d.h, h32) && aligned8(d.weight, w32) && aligned8(d.d_h, x32) &&
                     aligned8(d.dx, x32);
    const long long rows = d.dw ? std::min<long long>(d.T, block_rows(d.H)) : d.T;
    float *pair = rows < d.T ? part + (size_t)bwd_ctas(d.T, d.H) * d.H : nullptr;
    for (long long t = 0; t < d.T; t += rows) {
        auto from = [&](auto *p, bool f32) { return p ? (decltype(p))((uintptr_t)p + (size_t)t * d.H * (f32 ? 4 : 2)) : p; };
        NormBwdParams p;
        p.h = from(d.h, h32); p.dy = from(d.dy, g32); p.d_h = from(d.d_h, x32); p.dx = from(d.dx, x32);
        p.w = d.weight; p.rstd = d.rstd + t;
        p.part = d.dw ? part : nullptr;
        p.T = (int)std::min<long long>(rows, d.T - t); p.H = d.H; p.w_f32 = w32;
        cudaError_t err;
        if (d.type == PMPE_F32) err = vec ? launch<float, float, float, true>(p, st) : launch<float, float, float, false>(p, st);
        else if (d.type == PMPE_BF16) err = vec ? by_types<bf16, true>(p, g32, x32, st) : by_types<bf16, false>(p, g32, x32, st);
        else err = vec ? by_types<__half, true>(p, g32, x32, st) : by_types<__half, false>(p, g32, x32, st);
        if (err == cudaSuccess && d.dw)
            err = launch_pdl(rms_norm_dw_kernel, dim3((d.H + kDwCols - 1) / kDwCols), dim3(kDwCols * kStrands), 0, st, (const float *)part,
                             bwd_ctas(p.T, d.H), d.H, d.dw, pair, t == 0 ? 1 : 0, t + rows >= d.T ? 1 : 0);
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

}  // namespace pmpe
