// The paged key-value cache as its kernels see it (k_cache.cu, k_attend.cu).
#pragma once

#include "elem.cuh"

namespace pmpe {

// n / d for 0 <= n < 2^31 by a multiplication: with l = ceil(log2 d) and
// m = ceil(2^(31+l) / d) < 2^32, floor(n m / 2^(31+l)) is the quotient, as
// n (m d - 2^(31+l)) < 2^(31+l) (Granlund and Montgomery 1994).
struct FastDiv {
    uint32_t d, m;
    int shift;  // l - 1; -1 for d = 1
    explicit FastDiv(int div) : d((uint32_t)div), m(0), shift(-1)
    {
        int l = 0;
        while (((int64_t)1 << l) < div) ++l;
        if (l > 0) {
            m = (uint32_t)((((uint64_t)1 << (31 + l)) + div - 1) / (uint64_t)div);
            shift = l - 1;
        }
    }
    __device__ __forceinline__ int quotient(int n) const { return shift < 0 ? n : (int)(__umulhi((uint32_t)n, m) >> shift); }
};

struct KvView {
    uint8_t *k, *v;
    float *k_scale, *v_scale;
    int pages, page_size, kv_heads, head_dim;
    FastDiv by_page;
    const int32_t *table, *lengths, *cu;
    long long table_ld;
    int B, capacity;  // capacity: positions that a table row holds
    KvView(const pmpe_kv_cache &c, const pmpe_kv_sequences &s)
        : k((uint8_t *)c.k), v((uint8_t *)c.v), k_scale(c.k_scale), v_scale(c.v_scale), pages(c.pages), page_size(c.page_size),
          kv_heads(c.kv_heads), head_dim(c.head_dim), by_page(c.page_size), table(s.table), lengths(s.lengths), cu(s.cu_seqlens),
          table_ld(s.table_ld), B(s.B), capacity(s.table_width * c.page_size)
    {
    }
    __device__ __forceinline__ int length(int b) const { return min(max(__ldg(lengths + b), 0), capacity); }
};

}  // namespace pmpe
