// Attention of one query of each sequence over its paged cache:
//
//   s_p = scale q . k_p,   out = sum_p e^(s_p - m) v_p / sum_p e^(s_p - m),   lse = m + ln sum_p e^(s_p - m)
//
// in one pass over the cache with the running maximum m.  The cache's bytes
// bound it: of a key and its value (512 bytes with 128 columns of 16 bits)
// every query head of a group takes 512 operations, 8 an octet of heads and
// byte, a tenth of what mma.sync gives at the rate of DRAM.  (tcgen05 would
// hold 128 keys by eight heads in TMEM; there is no product here whose time
// shows.)  So each warp works by itself: it copies 16 keys and their values
// into a ring of its own, asynchronously, and no barrier stands between tiles.
//
//   S^T = K Q^T    16 keys by 8 heads: keys are the rows, so that a group of up
//                  to eight heads fills the tile; FP32
//   O^T += V^T P^T 16 columns by 8 heads; P in two 16-bit words (hi + lo), so
//                  that its rounding (2^-17 or less) vanishes beside the output's
//   8 bits         e4m3 to FP16 is exact; a key's scale multiplies its row of
//                  S, a value's scale its weight, over the largest scale so far
//                  (a power of two) to stay inside FP16
//
// Work is cut by length, not by sequence: tiles of 64 positions of all
// (sequence, key head) pairs in a row, an equal run of them for each CTA (two
// an SM), whose bounds each CTA derives from the lengths on the device.  A pair
// that one CTA holds whole is finished there; of the others each CTA leaves its
// sums (FP32) in the workspace, and a second launch joins them in order.
#include <algorithm>

#include "kv_cache.cuh"

namespace pmpe {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kKeys = 16;                // of a warp and tile
constexpr int kTile = kKeys * kWarps;    // positions of a tile
constexpr int kMaxCtas = 320;
constexpr int kJoinThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

enum Kind { kBf16, kF16, kE4m3Bf16, kE4m3F16 };  // cache (and queries)

struct AttendParams {
    KvView kv;
    const void *q;
    void *out;
    float *lse;
    long long q_ld, q_head_ld;
    int heads, group, blocks;  // query heads of a key head, and blocks of 8 kNT of them
    int window;
    float scale_log2;
    float *part;               // [CTAs][2][8 kNT][kDP + 2]: sums, maxima, totals
    long long *plan;           // [0] tiles a CTA, [1 + b] tiles before sequence b
};

template <int kDP, int kNT, int kKind> struct AttendShape {
    static constexpr bool k8 = kKind >= kE4m3Bf16;
    static constexpr int kE = k8 ? 1 : 2;
    static constexpr int kRow = kDP * kE, kCpr = kRow / 16;  // bytes, 16-byte chunks of a row
    static constexpr int kStage = 2 * kKeys * kRow + (k8 ? 2 * kKeys * 4 : 0) + 16;
    static constexpr int kCtas = kDP * kE <= 256 ? 2 : 1;   // of an SM
    static constexpr int kHeads = 8 * kNT;
    static constexpr int kBuf = kHeads * (kDP + 4) * 4, kStats = 2 * kWarps * kHeads * 4;
    static constexpr int kRoom = 228 * 1024 / kCtas - 1024 - 128 - kBuf - kStats;  // 1 KB a CTA is the system's, 128 bytes static
    static constexpr int kStages = kRoom / (kWarps * kStage) < 8 ? kRoom / (kWarps * kStage) : 8;
    static constexpr int kSmem = kWarps * kStages * kStage + kBuf + kStats;
    static_assert(kStages >= 3 && kStage % 16 == 0, "shared memory");
};

// Chunk c of row r of a tile: no two of eight rows' equal chunks in the same
// 16 bytes of a 128-byte bank line.
template <int kCpr> __device__ __forceinline__ int chunk_at(int r, int c)
{
    return r * kCpr + (kCpr % 8 == 0 ? c ^ (r & 7) : c ^ ((r >> 1) & 3));
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
template <bool kBf> __device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (kBf)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two e4m3 (the low half) as two FP16.
__device__ __forceinline__ uint32_t widen(uint32_t two)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    return (uint32_t)h.x | (uint32_t)h.y << 16;
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <bool kBf> __device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (kBf) return pack_bf16x2(a, b);
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <bool kBf> __device__ __forceinline__ float2 unpack2(uint32_t u)
{
    if constexpr (kBf) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&u));
}

// The positions of a sequence that its query sees, in tiles from a multiple of
// kTile on.
struct Span {
    int len, lo, first, tiles;
    __device__ __forceinline__ Span(const AttendParams &p, int b)
    {
        len = b < p.kv.B ? p.kv.length(b) : 0;
        lo = p.window > 0 ? max(0, len - p.window) : 0;
        first = lo / kTile * kTile;
        tiles = (int)(((unsigned)(len - first) + kTile - 1) / kTile);
    }
};

// A place in the row of all tiles: tile `tile` of the positions of sequence b,
// for block `block` of the queries of key head `head`.
struct Walk {
    int b, head, block, tile;
    Span s;
    __device__ __forceinline__ bool advance(const AttendParams &p)  // whether another pair begins
    {
        if (++tile < s.tiles) return false;
        tile = 0;
        if (++block == p.blocks) {
            block = 0;
            if (++head == p.kv.kv_heads) {
                head = 0;
                do s = Span(p, ++b);
                while (s.tiles == 0 && b < p.kv.B);
            }
        }
        return true;
    }
};

// The sum over the CTA's threads before this one, and over all.
__device__ __forceinline__ long long scan_before(long long v, long long *s_warp, long long &all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long sum = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long o = __shfl_up_sync(~0u, sum, off);
        if (lane >= off) sum += o;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    long long before = sum - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += s_warp[w];
        all += s_warp[w];
    }
    return before;
}

template <int kDP, int kNT, int kKind>
__global__ void __launch_bounds__(kThreads, (AttendShape<kDP, kNT, kKind>::kCtas)) attend_kernel(const __grid_constant__ AttendParams p)
{
    using S = AttendShape<kDP, kNT, kKind>;
    constexpr bool k8 = S::k8, kBf = kKind == kBf16;  // kBf: of the products
    constexpr bool kQBf = kKind == kBf16 || kKind == kE4m3Bf16;
    using Q = typename std::conditional<kQBf, bf16, __half>::type;
    constexpr int kSteps = kDP / 16;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long s_warp[kWarps], s_start;
    __shared__ int s_seq;
    uint8_t *ring = smem + (threadIdx.x >> 5) * S::kStages * S::kStage;
    float *all = (float *)(smem + kWarps * S::kStages * S::kStage);
    float *s_m = all + S::kBuf / 4, *s_l = s_m + kWarps * S::kHeads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane & 3, g = lane >> 2;
    pdl_trigger();
    pdl_wait();

    // ---- this CTA's run of tiles
    const int pairs = p.kv.kv_heads * p.blocks;
    long long total = 0, mine = 0, before0 = 0;
    for (int b0 = 0; b0 < p.kv.B; b0 += kThreads) {
        const int b = b0 + threadIdx.x;
        const long long n = (long long)Span(p, b).tiles * pairs;
        long long all;
        const long long before = total + scan_before(n, s_warp, all);
        if (b0 == 0) mine = n, before0 = before;
        if (blockIdx.x == 0 && b < p.kv.B) p.plan[1 + b] = before;
        total += all;
    }
    const long long per = (total + gridDim.x - 1) / gridDim.x;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.plan[0] = per;
        p.plan[1 + p.kv.B] = total;
    }
    // sequences that see nothing
    for (int b = blockIdx.x; b < p.kv.B; b += gridDim.x) {
        if (Span(p, b).tiles > 0) continue;
        const int n = p.heads * p.kv.head_dim;
        for (int i = threadIdx.x; i < n; i += kThreads) ((uint16_t *)p.out)[(long long)b * n + i] = 0;
        if (p.lse)
            for (int i = threadIdx.x; i < p.heads; i += kThreads) p.lse[(long long)b * p.heads + i] = -INFINITY;
    }
    const long long start = blockIdx.x * per, left = min(total, start + per) - start;
    if (left <= 0) return;
    if (p.kv.B <= kThreads) {
        if (start >= before0 && start < before0 + mine) {
            s_seq = threadIdx.x;
            s_start = start - before0;
        }
    } else {
        long long sum = 0;
        for (int b0 = 0; b0 < p.kv.B; b0 += kThreads) {
            const long long n = (long long)Span(p, b0 + threadIdx.x).tiles * pairs;
            long long all;
            const long long before = sum + scan_before(n, s_warp, all);
            if (start >= before && start < before + n) {
                s_seq = b0 + threadIdx.x;
                s_start = start - before;
            }
            sum += all;
        }
    }
    __syncthreads();
    Walk at = {s_seq, 0, 0, 0, Span(p, s_seq)};
    {
        const long long pair = s_start / at.s.tiles;
        at.tile = (int)(s_start - pair * at.s.tiles);
        at.head = (int)(pair / p.blocks);
        at.block = (int)(pair - (long long)at.head * p.blocks);
    }

    // ---- copies: lane r < 16 (and r + 16) finds row r's entry, one tile ahead
    Walk ahead = at;
    long long to_copy = left;
    int page = -1, place = 0;
    auto look_up = [&]() {
        const int pos = ahead.s.first + ahead.tile * kTile + warp * kKeys + (lane & 15);
        page = -1;
        if (to_copy > 0 && pos >= ahead.s.lo && pos < ahead.s.len) {
            const int j = p.kv.by_page.quotient(pos);
            place = pos - j * p.kv.page_size;
            page = __ldg(p.kv.table + ahead.b * p.kv.table_ld + j);
        }
    };
    const int row_bytes = p.kv.head_dim * S::kE;
    auto copy = [&](int stage) {
        if (to_copy > 0) {
            uint8_t *to = ring + stage * S::kStage;
            const uint32_t to32 = smem_u32(to);
            const bool there = (unsigned)page < (unsigned)p.kv.pages;
            const uint32_t mask = __ballot_sync(~0u, there) & 0xffffu;
            const long long entry = there ? ((long long)page * p.kv.kv_heads + ahead.head) * p.kv.page_size + place : 0;
            if (mask) {
#pragma unroll
                for (int i = 0; i < S::kCpr / 2; ++i) {
                    const int n = i * 32 + lane, r = n / S::kCpr, ch = n % S::kCpr;
                    const long long off = __shfl_sync(~0u, entry, r) * row_bytes + ch * 16;
                    const bool live = (mask >> r & 1) && ch * 16 < row_bytes;
                    const uint32_t dst = to32 + chunk_at<S::kCpr>(r, ch) * 16;
                    cp_async16(dst, p.kv.k + (live ? off : 0), live ? 16 : 0);
                    cp_async16(dst + kKeys * S::kRow, p.kv.v + (live ? off : 0), live ? 16 : 0);
                }
                if constexpr (k8) {
                    const float *src = lane < 16 ? p.kv.k_scale : p.kv.v_scale;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(to32 + 2 * kKeys * S::kRow + lane * 4), "l"(src + entry),
                                 "r"(there ? 4 : 0));
                }
            }
            if (lane == 0) *(uint32_t *)(to + S::kStage - 16) = mask;
            --to_copy;
            ahead.advance(p);
            look_up();
        }
        asm volatile("cp.async.commit_group;\n");
    };
    look_up();
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) copy(i);

    // ---- tiles
    uint32_t qf[kSteps][kNT][2];
    float o[kSteps][kNT][4], m[kNT][2], l[kNT][2], cs[kNT][2];
    float r_max = 0x1p-100f;  // 8 bits: the power of two that the weights are relative to
    int stage = 0, fill = S::kStages - 1, pieces = 0;
    bool fresh = true;
    int first_tile = at.tile;
    for (long long t = 0; t < left; ++t) {
        if (fresh) {
            fresh = false;
            first_tile = at.tile;
            const int live = min(p.group - at.block * S::kHeads, S::kHeads);
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) {
                const int h = nt * 8 + g;
                const Q *q = (const Q *)p.q + at.b * p.q_ld + (long long)(at.head * p.group + at.block * S::kHeads + h) * p.q_head_ld;
                float x[kSteps][4], top = 0.f;
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int d = ks * 16 + (k8 ? 4 * c + i : 2 * c + (i & 1) + 8 * (i >> 1));
                        x[ks][i] = h < live && d < p.kv.head_dim ? to_f32<Q>(q[d]) : 0.f;
                        top = fmaxf(top, fabsf(x[ks][i]));
                    }
                float up = 1.f;
                if constexpr (kKind == kE4m3Bf16) {  // into FP16's range, by a power of two
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
                    const int e = (int)(__float_as_uint(top) >> 23) - 127;  // -127 for zeros and subnormals, 128: not finite
                    if (e < 128) up = __uint_as_float((uint32_t)(min(14 - e, 100) + 127) << 23);
                }
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks) {
                    qf[ks][nt][0] = pack2<kBf>(x[ks][0] * up, x[ks][1] * up);
                    qf[ks][nt][1] = pack2<kBf>(x[ks][2] * up, x[ks][3] * up);
                }
                const float f = p.scale_log2 / up;
                cs[nt][0] = k8 ? __shfl_sync(~0u, f, 8 * c) : f;  // of heads 2c and 2c + 1
                cs[nt][1] = k8 ? __shfl_sync(~0u, f, 8 * c + 4) : f;
                m[nt][0] = m[nt][1] = -INFINITY;
                l[nt][0] = l[nt][1] = 0.f;
            }
            r_max = 0x1p-100f;
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[j][nt][i] = 0.f;
        }
        cp_async_wait<S::kStages - 2>();
        __syncwarp();
        copy(fill);
        fill = stage;
        const uint8_t *from = ring + stage * S::kStage;
        stage = stage + 1 == S::kStages ? 0 : stage + 1;
        const uint32_t mask = *(const uint32_t *)(from + S::kStage - 16);
        if (mask) {
            const uint32_t k_at = smem_u32(from), v_at = k_at + kKeys * S::kRow;
            float s[kNT][4];
            {
                float a[2][kNT][4] = {};
#pragma unroll
                for (int ks = 0; ks < kSteps; ks += k8 ? 2 : 1) {
                    uint32_t f[4];
                    ldsm4(f, k_at + chunk_at<S::kCpr>(lane & 15, (k8 ? ks : 2 * ks) + (lane >> 4)) * 16);
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) {
                        if constexpr (k8) {
                            mma16816<kBf>(a[0][nt], widen(f[0] & 0xffffu), widen(f[1] & 0xffffu), widen(f[0] >> 16), widen(f[1] >> 16), qf[ks][nt][0], qf[ks][nt][1]);
                            mma16816<kBf>(a[1][nt], widen(f[2] & 0xffffu), widen(f[3] & 0xffffu), widen(f[2] >> 16), widen(f[3] >> 16), qf[ks + 1][nt][0],
                                          qf[ks + 1][nt][1]);
                        } else {
                            mma16816<kBf>(a[ks & 1][nt], f[0], f[1], f[2], f[3], qf[ks][nt][0], qf[ks][nt][1]);
                        }
                    }
                }
                float k0 = 1.f, k1 = 1.f;
                if constexpr (k8) {
                    const float *sc = (const float *)(from + 2 * kKeys * S::kRow);
                    k0 = sc[g];
                    k1 = sc[g + 8];
                }
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nt][i] = (a[0][nt][i] + a[1][nt][i]) * (cs[nt][i & 1] * (i < 2 ? k0 : k1));
            }
            if (mask != 0xffffu) {
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(mask >> (g + (i < 2 ? 0 : 8)) & 1)) s[nt][i] = -INFINITY;
            }
            float top[kNT][2];
            bool grown = false;
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    top[nt][i] = fmaxf(s[nt][i], s[nt][i + 2]);
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1) top[nt][i] = fmaxf(top[nt][i], __shfl_xor_sync(~0u, top[nt][i], off));
                    grown |= top[nt][i] > m[nt][i];
                }
            float v0 = 1.f, v1 = 1.f;
            if constexpr (k8) {
                const float *sc = (const float *)(from + 2 * kKeys * S::kRow) + kKeys;
                v0 = sc[g];
                v1 = sc[g + 8];
                grown |= fmaxf(v0, v1) > r_max;
            }
            if (__any_sync(~0u, grown)) {
                float by = 1.f;
                if constexpr (k8) {
                    float r = fmaxf(v0, v1);
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1) r = fmaxf(r, __shfl_xor_sync(~0u, r, off));
                    if (r > r_max) {
                        const float to = __uint_as_float(min((__float_as_uint(r) & 0x7f800000u) + 0x00800000u, 0x7f000000u));
                        by = r_max / to;
                        r_max = to;
                    }
                }
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    float f[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float now = fmaxf(m[nt][i], top[nt][i]);
                        f[i] = ex2(m[nt][i] - (now == -INFINITY ? 0.f : now));
                        m[nt][i] = now;
                        l[nt][i] *= f[i];
                        f[i] *= by;
                    }
#pragma unroll
                    for (int j = 0; j < kSteps; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[j][nt][i] *= f[i & 1];
                }
            }
            const float w0 = k8 ? v0 * (0x1p14f / r_max) : 1.f, w1 = k8 ? v1 * (0x1p14f / r_max) : 1.f;
            uint32_t hi[kNT][2], lo[kNT][2];
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float base = m[nt][i & 1] == -INFINITY ? 0.f : m[nt][i & 1];
                    e[i] = ex2(s[nt][i] - base);
                    l[nt][i & 1] += e[i];
                    if (k8) e[i] *= i < 2 ? w0 : w1;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t h = pack2<kBf>(e[2 * i], e[2 * i + 1]);
                    const float2 back = unpack2<kBf>(h);
                    hi[nt][i] = transposed(h);
                    lo[nt][i] = transposed(pack2<kBf>(e[2 * i] - back.x, e[2 * i + 1] - back.y));
                }
            }
#pragma unroll
            for (int j = 0; j < kSteps; j += k8 ? 2 : 1) {
                uint32_t f[4];
                if constexpr (k8) {
                    ldsm4t(f, v_at + chunk_at<S::kCpr>(lane & 15, j + (lane >> 4)) * 16);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {  // bytes of a register: two columns of one key, two of the next
                        const uint32_t x = __byte_perm(f[2 * u], 0, 0x3120), y = __byte_perm(f[2 * u + 1], 0, 0x3120);
                        const uint32_t a0 = widen(x & 0xffffu), a1 = widen(x >> 16), a2 = widen(y & 0xffffu), a3 = widen(y >> 16);
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt) {
                            mma16816<kBf>(o[j + u][nt], a0, a1, a2, a3, hi[nt][0], hi[nt][1]);
                            mma16816<kBf>(o[j + u][nt], a0, a1, a2, a3, lo[nt][0], lo[nt][1]);
                        }
                    }
                } else {
                    ldsm4t(f, v_at + chunk_at<S::kCpr>((lane & 7) + (lane >> 4) * 8, 2 * j + ((lane >> 3) & 1)) * 16);
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) {
                        mma16816<kBf>(o[j][nt], f[0], f[1], f[2], f[3], hi[nt][0], hi[nt][1]);
                        mma16816<kBf>(o[j][nt], f[0], f[1], f[2], f[3], lo[nt][0], lo[nt][1]);
                    }
                }
            }
        }

        // ---- the end of a pair, or of this CTA's part of it
        const int b = at.b, head = at.head, block = at.block, tile = at.tile, tiles = at.s.tiles;
        fresh = at.advance(p);
        if (!fresh && t + 1 < left) continue;
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) l[nt][i] += __shfl_xor_sync(~0u, l[nt][i], off);
                if (g == 0) {
                    s_m[warp * S::kHeads + nt * 8 + 2 * c + i] = m[nt][i];
                    s_l[warp * S::kHeads + nt * 8 + 2 * c + i] = l[nt][i];
                }
            }
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w * S::kHeads + nt * 8 + 2 * c + i]);
                const float f = ex2(m[nt][i] - (top == -INFINITY ? 0.f : top)) * (k8 ? r_max * 0x1p-14f : 1.f);
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    o[j][nt][i] *= f;
                    o[j][nt][i + 2] *= f;
                }
            }
        // the warps' sums, one warp after another
        constexpr int kLd = kDP + 4;  // eight columns and four pairs of heads in different banks
#pragma unroll 1
        for (int w = 0; w < kWarps; ++w) {
            if (warp == w) {
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int d = j * 16 + (k8 ? 2 * g + (i >> 1) : g + 8 * (i >> 1));
                            float *at_d = all + (nt * 8 + 2 * c + (i & 1)) * kLd + d;
                            *at_d = w == 0 ? o[j][nt][i] : *at_d + o[j][nt][i];
                        }
            }
            __syncthreads();
        }
        auto totals = [&](int h, float &top, float &sum) {
            top = -INFINITY;
            sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w * S::kHeads + h]);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) sum += s_l[w * S::kHeads + h] * ex2(s_m[w * S::kHeads + h] - (top == -INFINITY ? 0.f : top));
        };
        const int live = min(p.group - block * S::kHeads, S::kHeads);
        if (first_tile == 0 && tile + 1 == tiles) {
            const long long h0 = (long long)b * p.heads + head * p.group + block * S::kHeads;
            for (int h = warp; h < live; h += kWarps) {
                float top, sum;
                totals(h, top, sum);
                const float f = sum == 0.f ? 0.f : 1.f / sum;
                for (int d = lane; d < p.kv.head_dim; d += 32) ((Q *)p.out)[(h0 + h) * p.kv.head_dim + d] = from_f32<Q>(all[h * kLd + d] * f);
                if (p.lse && lane == 0) p.lse[h0 + h] = (top + log2f(sum)) * kLn2;
            }
        } else {
            float *part = p.part + (blockIdx.x * 2 + (pieces > 0)) * (long long)(S::kHeads * (kDP + 2));
            for (int h = warp; h < live; h += kWarps) {
                float top, sum;
                totals(h, top, sum);
                for (int d = lane; d < kDP; d += 32) part[h * kDP + d] = all[h * kLd + d];
                if (lane == 0) {
                    part[S::kHeads * kDP + h] = top;
                    part[S::kHeads * (kDP + 1) + h] = sum;
                }
            }
        }
        ++pieces;
        __syncthreads();
    }
    cp_async_wait<0>();
}

// The parts of one head of one sequence, in the CTAs' order.
template <typename Q>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ AttendParams p, int dp, int block_heads)
{
    constexpr int kJoinWarps = kJoinThreads / 32;
    __shared__ float s_w[kMaxCtas], s_red[kJoinWarps], s_sum[kJoinWarps][PMPE_MAX_HEAD_DIM];
    pdl_trigger();
    pdl_wait();
    const int head = blockIdx.x, b = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long per = p.plan[0], first = p.plan[1 + b], tiles = (p.plan[2 + b] - first) / (p.kv.kv_heads * p.blocks);
    if (tiles == 0) return;
    const int kv_head = head / p.group, in_group = head - kv_head * p.group, block = in_group / block_heads, h = in_group - block * block_heads;
    const long long t0 = first + (long long)(kv_head * p.blocks + block) * tiles;
    const int c0 = (int)(t0 / per), c1 = (int)((t0 + tiles - 1) / per), n = c1 - c0 + 1;
    if (n == 1) return;
    // a CTA's first piece is in its first place
    auto part = [&](int i) { return p.part + ((c0 + i) * 2 + (i == 0 && t0 != c0 * per)) * (long long)(block_heads * (dp + 2)); };
    float top = -INFINITY;
    for (int i = threadIdx.x; i < n; i += kJoinThreads) {
        s_w[i] = part(i)[block_heads * dp + h];
        top = fmaxf(top, s_w[i]);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, off));
    if (lane == 0) s_red[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, s_red[w]);
    const float base = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    for (int i = threadIdx.x; i < n; i += kJoinThreads) {
        s_w[i] = ex2(s_w[i] - base);
        sum += s_w[i] * part(i)[block_heads * (dp + 1) + h];
    }
    sum = warp_sum(sum);
    __syncthreads();
    if (lane == 0) s_red[warp] = sum;
    float acc[PMPE_MAX_HEAD_DIM / 128][4] = {};
#pragma unroll 4
    for (int i = warp; i < n; i += kJoinWarps) {
        const float *from = part(i) + h * dp;
        const float w = s_w[i];
#pragma unroll
        for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k) {
            const int d = k * 128 + lane * 4;
            if (d >= dp) break;
            const float4 v = *reinterpret_cast<const float4 *>(from + d);
            acc[k][0] += w * v.x;
            acc[k][1] += w * v.y;
            acc[k][2] += w * v.z;
            acc[k][3] += w * v.w;
        }
    }
#pragma unroll
    for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k)
        if (k * 128 + lane * 4 < dp) *reinterpret_cast<float4 *>(&s_sum[warp][k * 128 + lane * 4]) = make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) sum += s_red[w];
    const long long row = (long long)b * p.heads + head;
    for (int d = threadIdx.x; d < p.kv.head_dim; d += kJoinThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) v += s_sum[w][d];
        ((Q *)p.out)[row * p.kv.head_dim + d] = from_f32<Q>(sum == 0.f ? 0.f : v / sum);
    }
    if (p.lse && threadIdx.x == 0) p.lse[row] = (top + log2f(sum)) * kLn2;
}

// -------------------------------------------------------------- launches

int padded(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : head_dim <= 192 ? 192 : 256; }
// Heads that share a pass over the keys: 8, or 16 where more share them and
// their sums fit the registers.
int block_heads_for(int group, int head_dim) { return group > 8 && head_dim <= 128 ? 16 : 8; }

template <int kDP, int kNT, int kKind> cudaError_t launch_shape(const AttendParams &p, int ctas, cudaStream_t st)
{
    using S = AttendShape<kDP, kNT, kKind>;
    static std::atomic<int> limit[64];
    cudaError_t err = ensure_dynamic_smem(attend_kernel<kDP, kNT, kKind>, S::kSmem, limit);
    if (err != cudaSuccess) return err;
    err = launch_pdl(attend_kernel<kDP, kNT, kKind>, dim3(std::min(ctas * S::kCtas, kMaxCtas)), dim3(kThreads), S::kSmem, st, p);
    if (err != cudaSuccess) return err;
    constexpr bool q_bf = kKind == kBf16 || kKind == kE4m3Bf16;
    return launch_pdl(join_kernel<typename std::conditional<q_bf, bf16, __half>::type>, dim3(p.heads, p.kv.B), dim3(kJoinThreads), 0, st, p, kDP, S::kHeads);
}
template <int kKind> cudaError_t launch_kind(const AttendParams &p, int ctas, cudaStream_t st)
{
    const int dp = padded(p.kv.head_dim);
    const bool wide = block_heads_for(p.group, p.kv.head_dim) == 16;
    if (dp == 64) return wide ? launch_shape<64, 2, kKind>(p, ctas, st) : launch_shape<64, 1, kKind>(p, ctas, st);
    if (dp == 128) return wide ? launch_shape<128, 2, kKind>(p, ctas, st) : launch_shape<128, 1, kKind>(p, ctas, st);
    return dp == 192 ? launch_shape<192, 1, kKind>(p, ctas, st) : launch_shape<256, 1, kKind>(p, ctas, st);
}

size_t part_bytes(int group, int head_dim) { return (size_t)kMaxCtas * 2 * block_heads_for(group, head_dim) * (padded(head_dim) + 2) * sizeof(float); }

}  // namespace

size_t kv_attend_workspace_bytes(int B, int heads, int kv_heads, int head_dim)
{
    return part_bytes(heads / kv_heads, head_dim) + ((size_t)B + 2) * sizeof(long long);
}

cudaError_t launch_kv_attend(const pmpe_kv_cache &c, const pmpe_kv_sequences &s, const pmpe_kv_attend_desc &d, int num_sms, cudaStream_t st)
{
    const int group = d.heads / c.kv_heads, bh = block_heads_for(group, c.head_dim);
    AttendParams p = {KvView(c, s), d.q, d.out, d.lse, d.q_ld, d.q_head_ld, d.heads, group, (group + bh - 1) / bh, d.window, d.scale * kLog2e,
                      (float *)d.workspace, (long long *)((uint8_t *)d.workspace + part_bytes(group, c.head_dim))};
    if (c.type == PMPE_BF16) return launch_kind<kBf16>(p, num_sms, st);
    if (c.type == PMPE_F16) return launch_kind<kF16>(p, num_sms, st);
    return d.type == PMPE_BF16 ? launch_kind<kE4m3Bf16>(p, num_sms, st) : launch_kind<kE4m3F16>(p, num_sms, st);
}

}  // namespace pmpe
