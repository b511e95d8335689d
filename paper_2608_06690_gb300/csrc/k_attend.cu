// Attention of one query of each sequence over its paged cache:
//
//   s_p = scale q . k_p,   out = sum_p e^(s_p - m) v_p / sum_p e^(s_p - m),   lse = m + ln sum_p e^(s_p - m)
//
// in one pass over the cache with the running maximum m.  The cache's bytes
// bound it (64 sequences of up to 8192 positions, 32 over 4 heads of 128, 538 MB
// of BF16: 87.6 us, 6.1 TB/s; 131072 positions of one sequence 50.2 us; in e4m3
// the 278 MB 60.2 us, where instructions count as much).  Of a key and its value (512 bytes in 16 bits) every query
// head of a group takes 512 operations: mma.sync is busy a sixth of the time
// (a fifth in e4m3).  tcgen05 would hold 128 keys by eight heads in TMEM and
// read them back for the maximum; no product here is long enough to show.
//
// Each warp works by itself, so that no barrier stands between tiles: it copies
// 16 keys and their values (32 of narrow ones) ahead into a ring of its own, by
// TMA where 16 positions lie one after another in a page (pages of a multiple of
// 16), by 16-byte copies of each row otherwise.  (The copies alone take 81 us of
// the 87.6, with the ones of each row 95.)  The more warps an SM has, the less
// each one's chain of dependent steps shows: 12 or 16 of them with two or three
// stages each; 8 with three took 107 us, and 97 in e4m3.
//
//   S^T = K Q^T    16 keys by 8 heads: keys are the rows, so that a group of up
//                  to eight heads fills the tile; FP32
//   O^T += V^T P^T 16 columns by 8 heads; P in three BF16 words, which hold all
//                  24 bits of an FP32 weight, or in two FP16 words.  (Two words of
//                  BF16, 2^-17 off, turned the rounding of one output in a thousand.)
//   8 bits         e4m3 to FP16 is exact; a key's scale multiplies its row of
//                  S, a value's scale its weight, over the largest scale so far
//                  (a power of two) to stay inside FP16
//
// Work is cut by length, not by sequence: tiles of 64 or 128 positions of all
// (sequence, block of heads) pairs in a row, an equal run of them for each CTA,
// whose bounds each CTA derives from the lengths on the device.  A pair that one
// CTA holds whole is finished there; of the others each CTA leaves its sums
// (FP32) in the workspace, and a second launch joins them in order.  That launch
// costs 2 to 5 us; sums joined by the last CTA of a pair would need counters that
// are zero before the call.
//
// Groups of more than 8 heads (16 up to 128 columns) are several blocks, each of
// which reads the keys and values again, and 16 heads side by side cost registers:
// the 64 ragged sequences with 16, 24, 64 heads a key head of 128 take 96, 159, 305
// us in BF16, 86, 146, 275 in e4m3 (102 bytes a thread spilled, 40 with heads of 64,
// 28 in 16 bits); with 24 heads of 256 246 and 146.
#include <algorithm>

#include "kv_cache.cuh"
#include "tc_ptx.cuh"

namespace pmpe {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kMaxCtas = 640;
constexpr int kJoinThreads = 256, kFew = 4;  // parts that a warp joins by itself
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;


enum Kind { kBf16, kF16, kE4m3Bf16, kE4m3F16 };  // cache (and queries)

struct AttendParams {
    KvView kv;
    const void *q;
    void *out;
    float *lse;
    long long q_ld, q_head_ld;
    int q_pairs;               // two elements of q an access
    int heads, group, blocks;  // query heads of a key head, and blocks of 8 kNT of them
    int window;
    float scale_log2;
    int box_rows;              // of a TMA copy: positions that lie one after another in a page; 0: copied one by one
    CUtensorMap k_map, v_map;  // the keys and values as rows of 16-bit words
    float *part;               // [CTAs][2]: [8 kNT][kDP] sums, [8 kNT][2] maxima and totals
};

template <int kDP, int kNT, int kKind> struct AttendShape {
    static constexpr bool k8 = kKind >= kE4m3Bf16;
    static constexpr int kE = k8 ? 1 : 2;
    // bytes of a row, its 16-byte chunks, and bytes of it in shared memory
    static constexpr int kRow = kDP * kE, kUsed = kRow / 16, kPitch = kRow <= 64 ? 64 : (kRow + 127) / 128 * 128;
    static constexpr int kBox = kPitch < 128 ? kPitch : 128, kBoxes = kPitch / kBox;  // bytes of a row that a TMA copy takes
    static constexpr int kHeads = 8 * kNT;
    // rows of 16 keys that a warp takes at a time: a stage of them holds the
    // warp's sums when a pair ends
    static constexpr int kMT = 2 * 16 * kPitch >= kHeads * kDP * 4 ? 1 : 2;
    static constexpr int kKeys = 16 * kMT, kTile = kKeys * kWarps;  // positions of a warp's part, of a tile
    static constexpr uint32_t kAll = kMT == 2 ? 0xffffffffu : 0xffffu;
    static constexpr int kData = 2 * kKeys * kPitch, kScales = k8 ? 2 * kKeys * 4 : 0;  // of a stage
    static constexpr int kSmall = kScales + 16;  // scales, barrier, mask
    static constexpr int kStats = 2 * kWarps * kHeads * 4;
    // CTAs of an SM: what their registers and two stages a warp allow
    static constexpr int kCtas = kDP * kNT <= 128 ? (kData <= 4096 ? 4 : 3) : kData <= 8192 ? (kDP <= 128 ? 3 : 2) : kData <= 12288 ? 2 : 1;
    // 1 KB a CTA is the system's, 128 bytes static, up to 1 KB goes to the rings' alignment
    static constexpr int kRoom = 228 * 1024 / kCtas - 2048 - 128 - kStats;
    static constexpr int kStages = kRoom / (kWarps * (kData + kSmall)) < 8 ? kRoom / (kWarps * (kData + kSmall)) : 8;
    static constexpr int kSmem = 1024 + kWarps * kStages * (kData + kSmall) + kStats;
    static_assert(kStages >= 2 && kData % 1024 == 0 && kSmall % 16 == 0 && kData >= kHeads * kDP * 4, "shared memory");
    // Chunk c of row r of a tile, as a TMA copy swizzles it: rows of kBox bytes,
    // no two of eight rows' equal chunks in the same 16 bytes of a 128-byte line.
    static __device__ __forceinline__ int chunk_at(int r, int c)
    {
        return kBox == 64 ? r * 4 + (c ^ ((r >> 1) & 3)) : (c >> 3) * kKeys * 8 + r * 8 + ((c & 7) ^ (r & 7));
    }
};

// 16 bytes into shared memory, asynchronously; zeros for bytes = 0.
__device__ __forceinline__ void fetch16(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(bytes));
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
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
template <int kTile> struct Span {
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
// for block `block` of the queries of key head `head`.  A warp's lanes go together.
template <int kTile> struct Walk {
    int b, head, block, tile;
    Span<kTile> s;
    __device__ __forceinline__ bool advance(const AttendParams &p)  // whether another pair begins
    {
        if (++tile < s.tiles) return false;
        tile = 0;
        if (++block == p.blocks) {
            block = 0;
            if (++head == p.kv.kv_heads) {
                head = 0;
                // the next sequence that sees something, by a look at 32 lengths
                // at once; B for none
                for (++b; b < p.kv.B; b += 32) {
                    const uint32_t any = __ballot_sync(~0u, Span<kTile>(p, b + (threadIdx.x & 31)).tiles > 0);
                    if (any) {
                        b += __ffs(any) - 1;
                        break;
                    }
                }
                b = min(b, p.kv.B);
                s = Span<kTile>(p, b);
            }
        }
        return true;
    }
};

// Work as the CTAs share it: a tile counts one, and each pair of a sequence and
// a block of heads kEnd more, for its queries and its end (64 sequences of 0 to
// 8192 positions in e4m3: CTAs of equal tiles ended 26 us apart, the ones with
// many short sequences last; kEnd = 1, 2, 3, 4 took 63.1, 63.6, 57.2, 56.7 us
// when 3 was chosen, in BF16 86.8 to 87.8, where a pair's end takes as long as 1.6 tiles).  Tile k of a
// pair that begins at cost P is at cost P + kEnd + k; CTA c has the costs c per ..
// (c + 1) per - 1.
constexpr long long kEnd = 3;
struct Cost {
    long long cost, tiles;
};
// The sum over the CTA's threads before this one, and over all.
template <int kN> __device__ __forceinline__ Cost scan_before(Cost v, Cost (&s_warp)[kN], Cost &all)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Cost sum = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long c = __shfl_up_sync(~0u, sum.cost, off), t = __shfl_up_sync(~0u, sum.tiles, off);
        if (lane >= off) sum.cost += c, sum.tiles += t;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    Cost before = {sum.cost - v.cost, sum.tiles - v.tiles};
    all = {0, 0};
#pragma unroll
    for (int w = 0; w < kN; ++w) {
        if (w < warp) before.cost += s_warp[w].cost, before.tiles += s_warp[w].tiles;
        all.cost += s_warp[w].cost, all.tiles += s_warp[w].tiles;
    }
    return before;
}
// Where a cost lies: the sequence, the pair of it, and what of it comes before;
// b = B past the end.
struct Spot {
    int b, pair, tile;         // the first tile from there on
    long long before, at;      // tiles before that one; the pair's cost
};
template <int kTile, int kN> struct Planner {
    const AttendParams &p;
    Cost (&s_warp)[kN];
    Spot (&s_spot)[2];
    int pairs;
    Cost all;
    __device__ __forceinline__ Cost of(int b) const
    {
        const int n = Span<kTile>(p, b).tiles;
        return {n > 0 ? (n + kEnd) * pairs : 0, (long long)n * pairs};
    }
    // The spots of the costs where(cost of all), two of them, in every thread.
    template <typename F> __device__ __forceinline__ void find(F where)
    {
        constexpr int kThreads = 32 * kN;
        Cost sum = {0, 0}, mine = {0, 0}, first = {0, 0};
        for (int b0 = 0; b0 < p.kv.B; b0 += kThreads) {
            const Cost n = of(b0 + threadIdx.x);
            Cost total;
            const Cost before = scan_before(n, s_warp, total);
            if (b0 == 0) mine = n, first = before;
            sum.cost += total.cost, sum.tiles += total.tiles;
        }
        all = sum;
        if (threadIdx.x < 2) s_spot[threadIdx.x] = {p.kv.B, 0, 0, all.tiles, all.cost};
        __syncthreads();
        sum = {0, 0};
        for (int b0 = 0; b0 < p.kv.B; b0 += kThreads) {
            if (b0 > 0 || p.kv.B > kThreads) {
                Cost total;
                mine = of(b0 + threadIdx.x);
                first = scan_before(mine, s_warp, total);
                first.cost += sum.cost, first.tiles += sum.tiles;
                sum.cost += total.cost, sum.tiles += total.tiles;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const long long x = where(all.cost, i) - first.cost;
                if (x >= 0 && x < mine.cost) {
                    const int tiles = (int)(mine.tiles / pairs), pair = (int)(x / (tiles + kEnd)), tile = max((int)(x - pair * (tiles + kEnd) - kEnd), 0);
                    s_spot[i] = {b0 + (int)threadIdx.x, pair, tile, first.tiles + (long long)pair * tiles + tile, first.cost + pair * (tiles + kEnd)};
                }
            }
        }
        __syncthreads();
    }
};

template <int kDP, int kNT, int kKind>
__global__ void __launch_bounds__(kThreads, (AttendShape<kDP, kNT, kKind>::kCtas)) attend_kernel(const __grid_constant__ AttendParams p)
{
    using S = AttendShape<kDP, kNT, kKind>;
    constexpr bool k8 = S::k8, kBf = kKind == kBf16;  // kBf: of the products
    constexpr bool kQBf = kKind == kBf16 || kKind == kE4m3Bf16;
    using Q = typename std::conditional<kQBf, bf16, __half>::type;
    constexpr int kSteps = kDP / 16, kMT = S::kMT, kKeys = S::kKeys, kTile = S::kTile;
    // Blocks of 16 columns whose products with the values go side by side: 1, 2, 4
    // take 95.8, 94.6, 89.0 us for heads of 256 in BF16 (where a scheduler has one
    // or two warps), 60.2, 60.2, 61.5 in e4m3 of 128, 95.1, 94.3, 98.6 with 16 heads of 64.
    constexpr int kCols = !k8 && kNT == 1 ? 4 : 2;
    constexpr int kWords = kBf ? 3 : 2;  // of a weight: all of its 24 bits, or 22
    // Powers of two that a score may be above the maximum that the weights are
    // relative to, and what they are multiplied by.  FP16's words end at 2^-24: they
    // use its range up to 2^15, so that a weight of 2^-22 of the largest keeps 16
    // bits and a smaller one is off by 2^-39 of the largest at most (over 8 bits, where
    // following the maximum more often costs time, 2^-19 and 2^-36: the 64 ragged
    // sequences take 58.1, 58.6, 59.0, 59.6 us with 8, 4, 3, 1 powers).
    constexpr float kAhead = kBf ? 8.f : k8 ? 3.f : 1.f, kUp = kBf ? 1.f : k8 ? 0x1p12f : 0x1p14f;
    using Span = Span<kTile>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Cost s_warp[kWarps];
    __shared__ Spot s_spot[2];
    __shared__ volatile int s_abort, s_left;  // a wait ran out; one for what was left behind did too
    uint8_t *rings = smem + (-smem_u32(smem) & 1023u), *smalls = rings + kWarps * S::kStages * S::kData;
    uint8_t *ring = rings + (threadIdx.x >> 5) * S::kStages * S::kData, *small = smalls + (threadIdx.x >> 5) * S::kStages * S::kSmall;
    float *s_m = (float *)(smalls + kWarps * S::kStages * S::kSmall), *s_l = s_m + kWarps * S::kHeads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane & 3, g = lane >> 2;
    const bool boxes = p.box_rows > 0;
    auto barrier = [&](int stage) { return smem_u32(small + stage * S::kSmall + S::kScales); };
    if (lane == 0) {  // a stage is full when its copies are: one arrival with their bytes, or every lane's
        for (int i = 0; i < S::kStages; ++i) mbar_init(barrier(i), boxes ? 1 : 32);
        if (warp == 0) s_abort = 0, s_left = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();  // not before: the second launch reads the lengths as soon as it starts

    // ---- this CTA's run of tiles
    Planner<kTile, kWarps> plan = {p, s_warp, s_spot, p.kv.kv_heads * p.blocks, {0, 0}};
    plan.find([&](long long all, int i) {
        const long long per = max((all + gridDim.x - 1) / gridDim.x, 1ll);
        return (blockIdx.x + i) * per;
    });
    // sequences that see nothing
    for (int b = blockIdx.x; b < p.kv.B; b += gridDim.x) {
        if (Span(p, b).tiles > 0) continue;
        const int n = p.heads * p.kv.head_dim;
        for (int i = threadIdx.x; i < n; i += kThreads) ((uint16_t *)p.out)[(long long)b * n + i] = 0;
        if (p.lse)
            for (int i = threadIdx.x; i < p.heads; i += kThreads) p.lse[(long long)b * p.heads + i] = -INFINITY;
    }
    const long long left = s_spot[1].before - s_spot[0].before;
    if (left <= 0) return;
    Walk<kTile> at = {s_spot[0].b, s_spot[0].pair / p.blocks, s_spot[0].pair % p.blocks, s_spot[0].tile, Span(p, s_spot[0].b)};

    // ---- copies
    Walk<kTile> ahead = at;
    long long to_copy = left;
    int copied = 0;
    // The entry of position pos (the first of `n` in one page); -1: none of
    // them is seen, or there is no page.
    auto entry_at = [&](int pos, int n) -> long long {
        if (pos + n <= ahead.s.lo || pos >= ahead.s.len) return -1;
        const int j = p.kv.by_page.quotient(pos), page = __ldg(p.kv.table + ahead.b * p.kv.table_ld + j);
        return (unsigned)page < (unsigned)p.kv.pages ? ((long long)page * p.kv.kv_heads + ahead.head) * p.kv.page_size + (pos - j * p.kv.page_size) : -1;
    };
    // In boxes a lane looks up 16 positions, for the pair's next tiles together,
    // so that the table's latency shows once in kBatch tiles.
    constexpr int kBatch = 32 / kMT;
    long long found = -1;  // boxes: of 16 positions of tile lane / kMT of the batch; else of one of the next tile's
    int in_batch = kBatch;
    auto look_up = [&]() {
        if (to_copy > 0) found = entry_at(ahead.s.first + ahead.tile * kTile + warp * kKeys + (lane & (kKeys - 1)), 1);
    };
    auto copy = [&](int stage) {
        if (to_copy <= 0) return;
        const uint32_t to = smem_u32(ring + stage * S::kData), bar = barrier(stage), scales = bar - S::kScales;
        uint32_t mask = 0;
        if (boxes) {
            const int pos = ahead.s.first + ahead.tile * kTile + warp * kKeys;
            if (in_batch == kBatch) {
                found = entry_at(pos + lane / kMT * kTile + lane % kMT * 16, 16);
                in_batch = 0;
            }
            long long entry[kMT];
            uint32_t bytes = 0;
#pragma unroll
            for (int h = 0; h < kMT; ++h) {
                entry[h] = __shfl_sync(~0u, found, in_batch * kMT + h);
                const int above = min(max(ahead.s.len - pos - 16 * h, 0), 16), below = min(max(ahead.s.lo - pos - 16 * h, 0), 16);
                mask |= (entry[h] >= 0 ? ((1u << above) - 1) & ~((1u << below) - 1) : 0u) << (16 * h);
                if (entry[h] >= 0) bytes += 2 * 16 * S::kPitch + S::kScales / kMT;
            }
            ++in_batch;
            if (lane == 0) {
                mbar_expect_tx(bar, bytes);
#pragma unroll
                for (int h = 0; h < kMT; ++h) {
                    if (entry[h] < 0) continue;
                    if (k8) {
                        bulk_load(scales + 64 * h, p.kv.k_scale + entry[h], 64, bar);
                        bulk_load(scales + kKeys * 4 + 64 * h, p.kv.v_scale + entry[h], 64, bar);
                    }
#pragma unroll
                    for (int x = 0; x < S::kBoxes; ++x) {
                        const uint32_t dst = to + x * kKeys * S::kBox + 16 * h * S::kBox;
                        tma_load_2d(dst, &p.k_map, bar, x * (S::kBox / 2), (int)entry[h]);
                        tma_load_2d(dst + kKeys * S::kPitch, &p.v_map, bar, x * (S::kBox / 2), (int)entry[h]);
                    }
                }
            }
        } else {
            const int row_bytes = p.kv.head_dim * S::kE;
            mask = __ballot_sync(~0u, found >= 0) & S::kAll;
            if (mask) {
#pragma unroll
                for (int i = 0; i < kKeys * S::kUsed / 32; ++i) {
                    const int n = i * 32 + lane, r = n / S::kUsed, ch = n % S::kUsed;
                    const long long off = __shfl_sync(~0u, found, r) * row_bytes + ch * 16;
                    const bool live = (mask >> r & 1) && ch * 16 < row_bytes;
                    const uint32_t dst = to + S::chunk_at(r, ch) * 16;
                    fetch16(dst, p.kv.k + (live ? off : 0), live ? 16 : 0);
                    fetch16(dst + kKeys * S::kPitch, p.kv.v + (live ? off : 0), live ? 16 : 0);
                }
                if constexpr (k8) {
                    const uint32_t dst = scales + (lane & (kKeys - 1)) * 4;
                    const long long e = max(found, 0ll);
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(p.kv.k_scale + e), "r"(found >= 0 ? 4 : 0));
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst + kKeys * 4), "l"(p.kv.v_scale + e), "r"(found >= 0 ? 4 : 0));
                }
            }
            cp_async_arrive_noinc(bar);
        }
        if (lane == 0) *(uint32_t *)(small + stage * S::kSmall + S::kScales + 8) = mask;
        --to_copy;
        ++copied;
        if (ahead.advance(p)) in_batch = kBatch;
        if (!boxes) look_up();
    };
    __syncwarp();
    if (!boxes) look_up();
#pragma unroll
    for (int i = 0; i < S::kStages - 1; ++i) copy(i);

    // ---- tiles
    uint32_t qf[kSteps][kNT][2];
    float o[kSteps][kNT][4], m[kNT][2], l[kNT][2], cs[kNT][2];
    float v_up = 0x1p126f;  // 8 bits: one over the power of two that the weights are relative to
    int stage = 0, fill = S::kStages - 1, pieces = 0;
    uint32_t parity = 0;
    bool fresh = true, lost = false;
    int first_tile = at.tile;
    // The queries of the pair at `at`, as stored: columns 2c, 2c + 1 and 8 on of
    // each 16 (8 bits: 4c to 4c + 3) of head g of eight; zeros where there are none.
    auto load_queries = [&]() {
        const int live = min(p.group - at.block * S::kHeads, S::kHeads);
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
            const int h = nt * 8 + g;
            const uint16_t *q = (const uint16_t *)p.q + at.b * p.q_ld + (long long)(at.head * p.group + at.block * S::kHeads + h) * p.q_head_ld;
#pragma unroll
            for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int d = ks * 16 + (k8 ? 4 * c + 2 * i : 2 * c + 8 * i);
                    uint32_t w = 0;
                    if (h < live && d < p.kv.head_dim) w = p.q_pairs ? *(const uint32_t *)(q + d) : q[d] | (uint32_t)q[d + 1] << 16;
                    qf[ks][nt][i] = w;
                }
        }
    };
    for (long long t = 0; t < left; ++t) {
        if (fresh) {
            fresh = false;
            first_tile = at.tile;
            if (t == 0) load_queries();
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) {
                float up = 1.f;
                if constexpr (kKind == kE4m3Bf16) {  // into FP16's range, by a power of two
                    float top = 0.f;
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 x = unpack2<true>(qf[ks][nt][i]);
                            top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));
                        }
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
                    const int e = (int)(__float_as_uint(top) >> 23) - 127;  // -127 for zeros and subnormals, 128: not finite
                    if (e < 128) up = __uint_as_float((uint32_t)(min(14 - e, 100) + 127) << 23);
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 x = unpack2<true>(qf[ks][nt][i]);
                            qf[ks][nt][i] = pack2<false>(x.x * up, x.y * up);
                        }
                }
                const float f = p.scale_log2 / up;
                cs[nt][0] = k8 ? __shfl_sync(~0u, f, 8 * c) : f;  // of heads 2c and 2c + 1
                cs[nt][1] = k8 ? __shfl_sync(~0u, f, 8 * c + 4) : f;
                m[nt][0] = m[nt][1] = -INFINITY;
                l[nt][0] = l[nt][1] = 0.f;
            }
            v_up = 0x1p126f;
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[j][nt][i] = 0.f;
        }
        if (!lost && __any_sync(~0u, !mbar_wait(barrier(stage), parity, &s_abort, nullptr))) {
            lost = true;  // (a copy that does not end: what this warp, all lanes of it, holds becomes NaN)
            to_copy = 0;
        }
        __syncwarp();
        copy(fill);
        fill = stage;
        const uint8_t *from = ring + stage * S::kData;
        const float *scales = (const float *)(small + stage * S::kSmall);
        const uint32_t mask = lost ? 0u : *(const uint32_t *)(small + stage * S::kSmall + S::kScales + 8);
        if (++stage == S::kStages) {
            stage = 0;
            parity ^= 1;
        }
        if (mask) {
            const uint32_t k_at = smem_u32(from), v_at = k_at + kKeys * S::kPitch;
            if (boxes && mask != S::kAll) {  // values that are not seen become zeros: 0 NaN is NaN
#pragma unroll 1
                for (int r = 0; r < kKeys; ++r)
                    if (!(mask >> r & 1) && lane < S::kUsed) st_shared_v4(v_at + S::chunk_at(r, lane) * 16, make_uint4(0u, 0u, 0u, 0u));
                fence_proxy_async_smem();  // before the next copy into this stage
                __syncwarp();
            }
            float s[kMT][kNT][4];
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt) {
                float a[2][kNT][4] = {};
#pragma unroll
                for (int ks = 0; ks < kSteps; ks += k8 ? 2 : 1) {
                    uint32_t f[4];
                    ldsm4(f, k_at + S::chunk_at(16 * mt + (lane & 15), (k8 ? ks : 2 * ks) + (lane >> 4)) * 16);
                    uint32_t w[8];
                    if constexpr (k8) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) e4m3x4_to_f16(f[i], w[2 * i], w[2 * i + 1]);
                    }
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) {
                        if constexpr (k8) {
                            mma16816<kBf>(a[0][nt], w[0], w[2], w[1], w[3], qf[ks][nt][0], qf[ks][nt][1]);
                            mma16816<kBf>(a[1][nt], w[4], w[6], w[5], w[7], qf[ks + 1][nt][0], qf[ks + 1][nt][1]);
                        } else {
                            mma16816<kBf>(a[ks & 1][nt], f[0], f[1], f[2], f[3], qf[ks][nt][0], qf[ks][nt][1]);
                        }
                    }
                }
                float k0 = 1.f, k1 = 1.f;
                if constexpr (k8) {
                    k0 = scales[16 * mt + g];
                    k1 = scales[16 * mt + g + 8];
                }
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[mt][nt][i] = (a[0][nt][i] + a[1][nt][i]) * (cs[nt][i & 1] * (i < 2 ? k0 : k1));
            }
            if (mask != S::kAll) {
#pragma unroll
                for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!(mask >> (16 * mt + g + (i < 2 ? 0 : 8)) & 1)) s[mt][nt][i] = -INFINITY;
            }
            // the maximum that powers are relative to follows the scores only
            // where one is 2^kAhead above it: no shuffles for most tiles
            bool grown = false;
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) grown |= s[mt][nt][i] > m[nt][i & 1] + kAhead;
            float v0[kMT], v1[kMT], v_top = 0.f;
            if constexpr (k8) {
#pragma unroll
                for (int mt = 0; mt < kMT; ++mt) {
                    v0[mt] = mask >> (16 * mt + g) & 1 ? scales[kKeys + 16 * mt + g] : 0.f;
                    v1[mt] = mask >> (16 * mt + g + 8) & 1 ? scales[kKeys + 16 * mt + g + 8] : 0.f;
                    v_top = fmaxf(v_top, fmaxf(v0[mt], v1[mt]));
                }
                grown |= v_top * v_up > 1.f;
            }
            if (__any_sync(~0u, grown)) {
                float by = 1.f;
                if constexpr (k8) {
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1) v_top = fmaxf(v_top, __shfl_xor_sync(~0u, v_top, off));
                    if (v_top * v_up > 1.f) {
                        const float to = 1.f / __uint_as_float(min((__float_as_uint(v_top) & 0x7f800000u) + 0x00800000u, 0x7f000000u));
                        by = to / v_up;
                        v_up = to;
                    }
                }
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    float f[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float now = fmaxf(s[0][nt][i], s[0][nt][i + 2]);
                        if (kMT == 2) now = fmaxf(now, fmaxf(s[kMT - 1][nt][i], s[kMT - 1][nt][i + 2]));
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) now = fmaxf(now, __shfl_xor_sync(~0u, now, off));
                        now = fmaxf(now, m[nt][i]);
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
            uint32_t pw[kMT][kNT][kWords][2];  // the weights' words, the largest first
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt) {
                const float w0 = k8 ? v0[mt] * v_up * kUp : kUp, w1 = k8 ? v1[mt] * v_up * kUp : kUp;
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float base = m[nt][i & 1] == -INFINITY ? 0.f : m[nt][i & 1];
                        e[i] = ex2(s[mt][nt][i] - base);
                        l[nt][i & 1] += e[i];
                        if (!kBf) e[i] *= i < 2 ? w0 : w1;
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int w = 0; w < kWords; ++w) {
                            const uint32_t h = pack2<kBf>(e[2 * i], e[2 * i + 1]);
                            const float2 back = unpack2<kBf>(h);
                            pw[mt][nt][w][i] = transposed(h);
                            e[2 * i] -= back.x;  // exactly
                            e[2 * i + 1] -= back.y;
                        }
                }
            }
            // 16 positions' sums, the smallest words first, then to the running
            // ones by additions that round: the matrix instructions cut their sums
            // off, always towards zero, which in running sums grew with the run
            // (1e-3 over 2^20 positions; without them 0.7 us of the 88, over
            // 8 bits 1.3 of the 60).
#pragma unroll
            for (int mt = 0; mt < kMT; ++mt)
#pragma unroll
                for (int j = 0; j < kSteps; j += kCols) {
                    uint32_t f[kCols][4];
                    if constexpr (k8) {
#pragma unroll
                        for (int u = 0; u < kCols; u += 2) {
                            uint32_t t[4];
                            ldsm4t(t, v_at + S::chunk_at(16 * mt + (lane & 15), j + u + (lane >> 4)) * 16);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {  // bytes of a register: two columns of one key, two of the next
                                e4m3x4_to_f16(__byte_perm(t[2 * h], 0, 0x3120), f[u + h][0], f[u + h][1]);
                                e4m3x4_to_f16(__byte_perm(t[2 * h + 1], 0, 0x3120), f[u + h][2], f[u + h][3]);
                            }
                        }
                    } else {
#pragma unroll
                        for (int u = 0; u < kCols; ++u) ldsm4t(f[u], v_at + S::chunk_at(16 * mt + (lane & 7) + (lane >> 4) * 8, 2 * (j + u) + ((lane >> 3) & 1)) * 16);
                    }
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) {
                        float sum[kCols][4] = {};
#pragma unroll
                        for (int w = kWords - 1; w >= 0; --w)
#pragma unroll
                            for (int u = 0; u < kCols; ++u) mma16816<kBf>(sum[u], f[u][0], f[u][1], f[u][2], f[u][3], pw[mt][nt][w][0], pw[mt][nt][w][1]);
#pragma unroll
                        for (int u = 0; u < kCols; ++u)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[j + u][nt][i] += sum[u][i];
                    }
                }
        }

        // ---- the end of a pair, or of this CTA's part of it
        const int b = at.b, head = at.head, block = at.block, tile = at.tile, tiles = at.s.tiles;
        fresh = at.advance(p);
        if (!fresh && t + 1 < left) continue;
        if (lost) {
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt) l[nt][0] = l[nt][1] = m[nt][0] = m[nt][1] = NAN;
        }
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
                const float f = ex2(m[nt][i] - (top == -INFINITY ? 0.f : top)) / kUp, down = k8 ? 1.f / v_up : 1.f;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {  // (two factors: their product may be too small)
                    o[j][nt][i] = o[j][nt][i] * f * down;
                    o[j][nt][i + 2] = o[j][nt][i + 2] * f * down;
                }
            }
        // the warps' sums, each in the stage that the warp has just read; a
        // head's columns turned by its number, so that few share a bank
        auto place = [](int h, int d) { return h * kDP + (d ^ ((h >> 1 & 3) << 3)); };
        {
            float *mine = (float *)const_cast<uint8_t *>(from);
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mine[place(nt * 8 + 2 * c + (i & 1), j * 16 + (k8 ? 2 * g + (i >> 1) : g + 8 * (i >> 1)))] = o[j][nt][i];
        }
        if (t + 1 < left) load_queries();  // of the next pair: on the way while this one ends
        __syncthreads();
        const float *sums = (const float *)(rings + (from - ring));  // of warp 0; the others' are a ring apart
        auto sum_of = [&](int h, int d) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) v += sums[w * (S::kStages * S::kData / 4) + place(h, d)];
            return v;
        };
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
                for (int d = lane; d < p.kv.head_dim; d += 32) ((Q *)p.out)[(h0 + h) * p.kv.head_dim + d] = from_f32<Q>(sum_of(h, d) * f);
                if (p.lse && lane == 0) p.lse[h0 + h] = (top + log2f(sum)) * kLn2;
            }
        } else {
            float *part = p.part + (blockIdx.x * 2 + (pieces > 0)) * (long long)(S::kHeads * (kDP + 2));
            for (int h = warp; h < live; h += kWarps) {
                float top, sum;
                totals(h, top, sum);
                for (int d = lane; d < kDP; d += 32) part[h * kDP + d] = sum_of(h, d);
                if (lane == 0) *reinterpret_cast<float2 *>(part + S::kHeads * kDP + 2 * h) = make_float2(top, sum);
            }
        }
        ++pieces;
        fence_proxy_async_smem();  // before the next copies into the stages
        __syncthreads();
    }
    if (lost)  // no copy is left behind: each stage's last one is waited for, again with a limit
        for (int n = max(copied - S::kStages, 0); n < copied; ++n) mbar_wait(barrier(n % S::kStages), n / S::kStages & 1, &s_left, nullptr);
    cp_async_wait<0>();
}

// The parts of a pair, joined in the CTAs' order.  A CTA for each border between
// two CTAs of the first launch; of a pair with a few parts the first border's
// does all, a warp a head; of one with many each border's does some heads.
// Which, and where the parts are, follows from the lengths, before the first
// launch is done.
template <typename Q, int kTile>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ AttendParams p, int dp, int block_heads, int ctas)
{
    constexpr int kJoinWarps = kJoinThreads / 32;
    __shared__ float s_top[kJoinWarps], s_total[kJoinWarps];
    __shared__ __align__(16) float s_sum[kJoinWarps][PMPE_MAX_HEAD_DIM];
    __shared__ Cost s_warp[kJoinWarps];
    __shared__ Spot s_spot[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Planner<kTile, kJoinWarps> plan = {p, s_warp, s_spot, p.kv.kv_heads * p.blocks, {0, 0}};
    long long per = 1;
    plan.find([&](long long all, int) {
        per = max((all + ctas - 1) / ctas, 1ll);
        return (blockIdx.x + 1) * per;
    });
    const Spot spot = s_spot[0];  // of what the border cuts
    const int b = spot.b, pair = spot.pair, tiles = b < p.kv.B ? Span<kTile>(p, b).tiles : 0;
    const int c0 = (int)((spot.at + kEnd) / per), n = tiles > 0 ? (int)((spot.at + kEnd + tiles - 1) / per) - c0 + 1 : 1;
    const int own = (int)blockIdx.x - c0;  // the own-th border of the pair
    const bool few = n <= kFew;
    pdl_trigger();
    pdl_wait();
    if (n == 1 || own < 0 || (few && own > 0)) return;
    const long long size = block_heads * (dp + 2);
    // a CTA's first piece is in its first place
    auto part = [&](int i) { return p.part + ((c0 + i) * 2 + (i == 0 && c0 * per < spot.at)) * size; };
    const int kv_head = pair / p.blocks, block = pair - kv_head * p.blocks, live = min(p.group - block * block_heads, block_heads);
    const long long row0 = (long long)b * p.heads + kv_head * p.group + block * block_heads;
    if (few) {
        for (int h = warp; h < live; h += kJoinWarps) {
            float4 v[kFew][PMPE_MAX_HEAD_DIM / 128];
            float2 ml[kFew];  // maximum and total
#pragma unroll
            for (int i = 0; i < kFew; ++i) {
                ml[i] = i < n ? *reinterpret_cast<const float2 *>(part(i) + block_heads * dp + 2 * h) : make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k) {
                    const int d = k * 128 + lane * 4;
                    v[i][k] = i < n && d < dp ? *reinterpret_cast<const float4 *>(part(i) + h * dp + d) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
            float top = -INFINITY, sum = 0.f, acc[PMPE_MAX_HEAD_DIM / 128][4] = {};
#pragma unroll
            for (int i = 0; i < kFew; ++i) top = fmaxf(top, ml[i].x);
#pragma unroll
            for (int i = 0; i < kFew; ++i) {
                const float w = ex2(ml[i].x - (top == -INFINITY ? 0.f : top));
                sum += w * ml[i].y;
#pragma unroll
                for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k) {
                    acc[k][0] += w * v[i][k].x;
                    acc[k][1] += w * v[i][k].y;
                    acc[k][2] += w * v[i][k].z;
                    acc[k][3] += w * v[i][k].w;
                }
            }
            const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int d = k * 128 + lane * 4 + e;
                    if (d < p.kv.head_dim) ((Q *)p.out)[(row0 + h) * p.kv.head_dim + d] = from_f32<Q>(acc[k][e] * f);
                }
            if (p.lse && lane == 0) p.lse[row0 + h] = (top + log2f(sum)) * kLn2;
        }
        return;
    }
    // every load of a part is on the way before one is waited for
    for (int h = own; h < live; h += n - 1) {
        constexpr int kAtOnce = 8;
        float acc[PMPE_MAX_HEAD_DIM / 128][4] = {}, top = -INFINITY, sum = 0.f;
        for (int i0 = warp; i0 < n; i0 += kJoinWarps * kAtOnce) {
            float4 v[kAtOnce][PMPE_MAX_HEAD_DIM / 128];
            float m[kAtOnce], l[kAtOnce], now = top;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const int i = i0 + j * kJoinWarps;
                m[j] = -INFINITY;
                l[j] = 0.f;
                if (i < n) {
                    const float2 ml = *reinterpret_cast<const float2 *>(part(i) + block_heads * dp + 2 * h);
                    m[j] = ml.x;
                    l[j] = ml.y;
                }
#pragma unroll
                for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k) {
                    const int d = k * 128 + lane * 4;
                    v[j][k] = i < n && d < dp ? *reinterpret_cast<const float4 *>(part(i) + h * dp + d) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) now = fmaxf(now, m[j]);
            const float base = now == -INFINITY ? 0.f : now, f = ex2(top - base);
            sum *= f;
#pragma unroll
            for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[k][e] *= f;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const float w = ex2(m[j] - base);
                sum += w * l[j];
#pragma unroll
                for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k) {
                    acc[k][0] += w * v[j][k].x;
                    acc[k][1] += w * v[j][k].y;
                    acc[k][2] += w * v[j][k].z;
                    acc[k][3] += w * v[j][k].w;
                }
            }
            top = now;
        }
        if (lane == 0) s_top[warp] = top, s_total[warp] = sum;
#pragma unroll
        for (int k = 0; k < PMPE_MAX_HEAD_DIM / 128; ++k)
            if (k * 128 + lane * 4 < dp) *reinterpret_cast<float4 *>(&s_sum[warp][k * 128 + lane * 4]) = make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
        __syncthreads();
        top = -INFINITY;
        sum = 0.f;
        float f[kJoinWarps];
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, s_top[w]);
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) {
            f[w] = ex2(s_top[w] - (top == -INFINITY ? 0.f : top));
            sum += f[w] * s_total[w];
        }
        for (int d = threadIdx.x; d < p.kv.head_dim; d += kJoinThreads) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kJoinWarps; ++w) v += f[w] * s_sum[w][d];
            ((Q *)p.out)[(row0 + h) * p.kv.head_dim + d] = from_f32<Q>(sum == 0.f ? 0.f : v / sum);
        }
        if (p.lse && threadIdx.x == 0) p.lse[row0 + h] = (top + log2f(sum)) * kLn2;
        __syncthreads();
    }
}

// -------------------------------------------------------------- launches

int padded(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : head_dim <= 192 ? 192 : 256; }
// Heads that share a pass over the keys: 8, or 16 where more share them and
// their sums fit the registers.
int block_heads_for(int group, int head_dim) { return group > 8 && head_dim <= 128 ? 16 : 8; }

template <int kDP, int kNT, int kKind> cudaError_t launch_shape(const AttendParams &p0, int ctas, cudaStream_t st)
{
    using S = AttendShape<kDP, kNT, kKind>;
    // copies in boxes: of kKeys rows, or of 16, that lie in one page
    AttendParams p = p0;
    const long long rows = (long long)p.kv.pages * p.kv.kv_heads * p.kv.page_size;
    const uint64_t words = (uint64_t)p.kv.head_dim * S::kE / 2;
    const CUtensorMapSwizzle swizzle = S::kBox == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
    p.box_rows = 0;
    if (p.kv.page_size % 16 == 0 && rows < (1ll << 31) && !(((uintptr_t)p.kv.k_scale | (uintptr_t)p.kv.v_scale) & 15u) &&
        encode_2d_box(&p.k_map, p.kv.k, words, rows, S::kBox / 2, 16, swizzle) && encode_2d_box(&p.v_map, p.kv.v, words, rows, S::kBox / 2, 16, swizzle))
        p.box_rows = 16;
    static std::atomic<int> limit[64];
    cudaError_t err = ensure_dynamic_smem(attend_kernel<kDP, kNT, kKind>, S::kSmem, limit);
    if (err != cudaSuccess) return err;
    ctas = std::min(ctas * S::kCtas, kMaxCtas);
    err = launch_pdl(attend_kernel<kDP, kNT, kKind>, dim3(ctas), dim3(kThreads), S::kSmem, st, p);
    if (err != cudaSuccess) return err;
    constexpr bool q_bf = kKind == kBf16 || kKind == kE4m3Bf16;
    return launch_pdl(join_kernel<typename std::conditional<q_bf, bf16, __half>::type, S::kTile>, dim3(std::max(ctas - 1, 1)), dim3(kJoinThreads), 0, st, p, kDP, S::kHeads, ctas);
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
    (void)B;
    return part_bytes(heads / kv_heads, head_dim);
}

cudaError_t launch_kv_attend(const pmpe_kv_cache &c, const pmpe_kv_sequences &s, const pmpe_kv_attend_desc &d, int num_sms, cudaStream_t st)
{
    const int group = d.heads / c.kv_heads, bh = block_heads_for(group, c.head_dim);
    AttendParams p = {KvView(c, s), d.q, d.out, d.lse, d.q_ld, d.q_head_ld,
                      ((uintptr_t)d.q & 3u) == 0 && d.q_ld % 2 == 0 && d.q_head_ld % 2 == 0, d.heads, group, (group + bh - 1) / bh, d.window, d.scale * kLog2e,
                      0, {}, {}, (float *)d.workspace};
    if (c.type == PMPE_BF16) return launch_kind<kBf16>(p, num_sms, st);
    if (c.type == PMPE_F16) return launch_kind<kF16>(p, num_sms, st);
    return d.type == PMPE_BF16 ? launch_kind<kE4m3Bf16>(p, num_sms, st) : launch_kind<kE4m3F16>(p, num_sms, st);
}

}  // namespace pmpe
