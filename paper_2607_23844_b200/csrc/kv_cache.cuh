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
// The scale is the nearest fp32 number, without a division (one costs fp32 rows 24 us of 174): max times a reciprocal of two
// parts, the smaller one first (Brisebarre, Muller and Raina, division by a divisor known in advance; equal to max / L for
// every mantissa with both L).
struct KvQuant { float scale, inv, max; };
template <int L>
__device__ __forceinline__ KvQuant kv_quant(uint32_t max_bits) {
    constexpr float high = 1.0f / L, low = (float)(1.0 / L - (double)high);
    KvQuant r;
    r.max = __uint_as_float(max_bits);
    if (max_bits >= 0x7F800000u) { r.scale = r.max; r.inv = 0.0f; }
    else if (r.max < 7.8886091e-31f) { r.scale = 0.0f; r.inv = 0.0f; }
    else { r.scale = fmaf(r.max, high, r.max * low); r.inv = r.max < 1e36f ? __fdividef((float)L, r.max) : (float)L / r.max; }     // (the former has no room above)
    return r;
}
// rint(x * L / max) exactly, ties to even, from a quotient that is off by less than 1.  x * L - (q +- 1/2) * max, doubled, decides.  x * L is a sum
// of two fp32 numbers; the larger less the product is exact where the two are close (a multiple of the smaller one's last
// place, and few of them), and a sum of two fp32 numbers always has the right sign.
template <int L>
__device__ __forceinline__ float kv_level_exact(float x, float q, float max) {
    if (max > 1e30f) { x *= 2.3283064e-10f; max *= 2.3283064e-10f; }         // (by 2^-32, exactly: twice x * L has no room above)
    const float xl = x * (float)L, lost = fmaf(x, (float)L, -xl);            // x * L = xl + lost
    const float above = fmaf(-(2.0f * q + 1.0f), max, 2.0f * xl) + 2.0f * lost, below = fmaf(-(2.0f * q - 1.0f), max, 2.0f * xl) + 2.0f * lost;
    const bool odd = ((int)q & 1) != 0;
    if (above > 0.0f || (above == 0.0f && odd)) return q + 1.0f;
    if (below < 0.0f || (below == 0.0f && odd)) return q - 1.0f;
    return q;
}
// 8 elements: their whole numbers in the low bits of 8 words.  A quotient + 1.5 * 2^23 rounds to one (the conversion
// instruction has a quarter of the rate); x * inv is off by less than 3e-5.
//   fp32  what lands within 1e-4 of a tie is looked at again
//   bf16  ties are common (x = max / 2 is one).  x and max being n 2^a and m 2^b with n, m < 256, a quotient that is no tie
//         differs from each by a share of 1 / (2 L n) at least, 1.5e-5: rounded with 1 / max 4e-6 too small and too large, the two
//         differ at a tie only, and their mean rounds to the even one
// inv = 0 gives 0 also where x is not finite.
template <int L, int DT>
__device__ __forceinline__ void kv_levels(const f32x2* f, const KvQuant& k, uint32_t* n) {
    const float magic = 12582912.0f;
    if (k.inv == 0.0f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) n[i] = 0u;
        return;
    }
    float worst = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f32x2 y;
        if (DT == OC_DTYPE_BF16) {
            const f32x2 a = f2_add(f2_fma(f[i], f2(k.inv * (1.0f - 4e-6f)), f2(magic)), f2(-magic));
            const f32x2 b = f2_add(f2_fma(f[i], f2(k.inv * (1.0f + 4e-6f)), f2(magic)), f2(-magic));
            y = f2_fma(f2_add(a, b), f2(0.5f), f2(magic));
        } else {
            y = f2_fma(f[i], f2(k.inv), f2(magic));
            const f32x2 t = f2_fma(f[i], f2(k.inv), f2_fma(y, f2(-1.0f), f2(magic)));
            worst = fmaxf(worst, fmaxf(fabsf(f2_lo(t)), fabsf(f2_hi(t))));
        }
        n[2 * i] = __float_as_uint(f2_lo(y)); n[2 * i + 1] = __float_as_uint(f2_hi(y));
    }
    if (DT == OC_DTYPE_F32 && worst > 0.4999f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a = kv_level_exact<L>(f2_lo(f[i]), __uint_as_float(n[2 * i]) - magic, k.max), b = kv_level_exact<L>(f2_hi(f[i]), __uint_as_float(n[2 * i + 1]) - magic, k.max);
            n[2 * i] = __float_as_uint(a + magic); n[2 * i + 1] = __float_as_uint(b + magic);
        }
    }
}
#endif

}  // namespace oc
