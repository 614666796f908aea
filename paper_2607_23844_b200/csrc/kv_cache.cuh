// The paged cache as the kernels see it: where a token's vectors lie, and what a vector of whole numbers stands for.
#pragma once
#include "rows.cuh"

namespace oc {

struct KvPages {
    const int32_t* table;            // null: pages in order
    long long table_stride;
    FastDiv page_rows;
    uint32_t n_pages, seq_pages;     // pages of the pool; of a sequence without a table
    uint32_t seq_rows, n_tokens;
    int heads, D;
    int* status;
};

inline KvPages kv_pages(const oc_kv_desc& d, const int32_t* table, int* status) {
    KvPages k;
    k.table = table; k.table_stride = d.table_stride; k.page_rows = FastDiv((uint32_t)d.page_rows);
    k.n_pages = (uint32_t)d.n_pages; k.seq_pages = (uint32_t)((d.seq_rows + d.page_rows - 1) / d.page_rows);
    k.seq_rows = (uint32_t)d.seq_rows; k.n_tokens = (uint32_t)(d.n_seqs * d.seq_rows);
    k.heads = d.heads; k.D = d.head_dim; k.status = status;
    return k;
}

#ifdef __CUDACC__
// The pool's page of a sequence's page number, or -1 (recorded) where the table names one outside the pool.
__device__ __forceinline__ int kv_page(const KvPages& K, uint32_t seq, uint32_t page) {
    if (!K.table) return (int)(seq * K.seq_pages + page);
    const int id = __ldg(K.table + (long long)seq * K.table_stride + page);
    if ((uint32_t)id < K.n_pages) return id;
    atomicCAS(K.status, 0, OC_ERR_INVALID_ARG);
    return -1;
}
// The vector of (page, head 0, row of the page); those of the other heads follow page_rows apart.
__device__ __forceinline__ uint32_t kv_vector(const KvPages& K, int page, uint32_t row) {
    return (uint32_t)page * (uint32_t)K.heads * K.page_rows.d + row;
}

// Whole numbers of a vector from its largest magnitude (bits of it): scale = max|x| / L, inv = L / max|x|.
struct KvQuant { float scale, inv, max; };
template <int L>
__device__ __forceinline__ KvQuant kv_quant(uint32_t max_bits) {
    KvQuant r;
    r.max = __uint_as_float(max_bits);
    if (max_bits >= 0x7F800000u) { r.scale = r.max; r.inv = 0.0f; }
    else if (r.max < 7.8886091e-31f) { r.scale = 0.0f; r.inv = 0.0f; }
    else { r.scale = r.max * (1.0f / L); r.inv = (float)L / r.max; }
    return r;
}
// rint(x * L / max), ties to even.  x * inv is off by up to two roundings, which only matters next to a border: there the
// remainder x * L - q * max, which a fused multiply-add gives with one rounding, is half of max or more.
template <int L>
__device__ __forceinline__ int kv_level(float x, const KvQuant& k) {
    int q = __float2int_rn(x * k.inv);
    if (k.inv != 0.0f) {
        const float xl = x * (float)L, lost = fmaf(x, (float)L, -xl);        // x * L = xl + lost
        const float rest = 2.0f * (fmaf(-(float)q, k.max, xl) + lost);
        if (rest > k.max || (rest == k.max && (q & 1))) ++q;
        else if (rest < -k.max || (rest == -k.max && (q & 1))) --q;
    } else {
        q = 0;
    }
    return q;
}
#endif

}  // namespace oc
