// What the attention kernels share: a call's parameters, the rows and keys of a sequence, which keys a row sees, and the
// joining of partial results of CTAs that split a sequence's keys.
#pragma once
#include "kv_cache.cuh"

namespace oc {

static constexpr int ATT_SPLIT_MAX = 16;         // CTAs of a cluster that share the keys of a tile of rows

struct AttnParams {
    KvPages pages;
    const int32_t *kv_len, *q_start, *idx;
    const void *q, *k_pool, *v_pool;
    const float *k_scale, *v_scale;
    void* out; float* lse;
    long long q_batch, q_row, q_head, o_batch, o_row, o_head;                 // elements
    uint32_t n_rows, rows_per_batch, n_seqs;
    int q_heads, group;                          // heads of q; those that share a head of the cache
    long long unit, back, ahead;                 // (64 bits: a window's end may leave 32)
    float scale, scale_log2;                     // of the scores; the same times log2(e)
    uint32_t tiles;                              // tiles of rows of a sequence and head of the cache
    int split;                                   // CTAs of a cluster
    bool wide_q, wide_out;                       // 16 bytes at a time
    bool long_first;                             // order of the tiles (attn_tile)
    int part_shift;                              // log2 of the keys of a 128th of a sequence, 7 or more
};

#ifdef __CUDACC__
// A CTA's work: a tile of rows of one sequence and head of the cache.  Neighbouring CTAs share their keys and values
// in L2, except where the tiles' work differs (windows, packed sequences): then the last tiles of all sequences, which
// have the most keys with a causal window and exist in the longest sequences only, come first.
struct AttnTile { uint32_t seq, head, tile; };
__device__ __forceinline__ AttnTile attn_tile(const AttnParams& P, uint32_t id) {
    AttnTile t;
    uint32_t problem;
    if (P.long_first) {
        const uint32_t problems = P.n_seqs * (uint32_t)P.pages.heads, back = id / problems;
        problem = id - back * problems;
        t.tile = P.tiles - 1 - back;
    } else {
        problem = id / P.tiles;
        t.tile = id - problem * P.tiles;
    }
    t.seq = problem / (uint32_t)P.pages.heads;
    t.head = problem - t.seq * (uint32_t)P.pages.heads;
    return t;
}

struct AttnSeq { long long row0; int n, len; };                               // first row, rows, tokens of the cache
__device__ __forceinline__ AttnSeq attn_seq(const AttnParams& P, uint32_t seq) {
    AttnSeq s;
    if (P.q_start) {
        const int a = __ldg(P.q_start + seq), b = __ldg(P.q_start + seq + 1);
        const bool good = a >= 0 && b >= a && (uint32_t)b <= P.n_rows && (uint32_t)(b - a) <= P.rows_per_batch;
        if (!good) atomicCAS(P.pages.status, 0, OC_ERR_INVALID_ARG);
        s.row0 = a; s.n = good ? b - a : 0;
    } else {
        s.row0 = (long long)seq * P.rows_per_batch;
        const long long left = (long long)P.n_rows - s.row0;
        s.n = left <= 0 ? 0 : (left < (long long)P.rows_per_batch ? (int)left : (int)P.rows_per_batch);
    }
    s.len = (int)P.pages.seq_rows;
    if (P.kv_len) {
        const int l = __ldg(P.kv_len + seq);
        if (l < 0 || l > s.len) atomicCAS(P.pages.status, 0, OC_ERR_INVALID_ARG);
        s.len = l < 0 ? 0 : min(l, s.len);
    }
    return s;
}

// Keys [lo, hi) that row i of the sequence sees; false if the row is left as it is.
__device__ __forceinline__ bool attn_bounds(const AttnParams& P, const AttnSeq& s, uint32_t seq, int i, int& lo, int& hi) {
    long long p = (long long)s.len - s.n + i;
    lo = 0; hi = s.len;
    if (P.idx) {
        const int t = __ldg(P.idx + s.row0 + i);
        if (t < 0) return false;
        p = (long long)t - (long long)seq * P.pages.seq_rows;
        if (p < 0 || p >= (long long)P.pages.seq_rows) { atomicCAS(P.pages.status, 0, OC_ERR_INVALID_ARG); return false; }
    }
    if (P.unit > 0) {
        const int un = (int)P.unit, pi = (int)p;                              // (both fit: unit was clamped to 2^31 - 1)
        const long long u = pi >= 0 ? pi / un : -(long long)((un - 1 - (long long)pi) / un);
        if (P.back >= 0) lo = (int)max(0ll, min((long long)s.len, (u - P.back) * P.unit));
        if (P.ahead >= 0) hi = (int)max(0ll, min((long long)s.len, (u + P.ahead + 1) * P.unit));
    }
    return true;
}
__device__ __forceinline__ long long attn_q_at(const AttnParams& P, const AttnSeq& s, uint32_t seq, int i, int head) {
    return (P.q_start ? (s.row0 + i) * P.q_row : (long long)seq * P.q_batch + (long long)i * P.q_row) + (long long)head * P.q_head;
}
__device__ __forceinline__ long long attn_out_at(const AttnParams& P, const AttnSeq& s, uint32_t seq, int i, int head) {
    return (P.q_start ? (s.row0 + i) * P.o_row : (long long)seq * P.o_batch + (long long)i * P.o_row) + (long long)head * P.o_head;
}

__device__ __forceinline__ uint32_t attn_fma2(uint32_t a, uint32_t b, uint32_t c) { uint32_t r; asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c)); return r; }
// Values that are no numbers are taken as zeros by the kernels, so that they stay away from rows that do not see them, and added
// at the end to those that do.  A CTA keeps the first and the last key that holds one, and of 128 parts of the sequence (of 128 keys
// and more) whether they hold any: rows look at those only.
static constexpr int ATT_BAD = 2 + 4;
// (of pairs of bf16: 0 times what is no number is NaN, and stays it in a sum that begins with zeros)
__device__ __forceinline__ uint32_t attn_zero2(uint32_t sum, uint32_t w) { return attn_fma2(w, 0u, sum); }
__device__ __forceinline__ bool attn_bad2(uint32_t sum) { return (sum & 0x7FFF7FFFu) != 0u; }
__device__ __forceinline__ void attn_bad_none(int* bad) {
    bad[0] = 0x7FFFFFFF;
    for (int i = 1; i < ATT_BAD; ++i) bad[i] = 0;
}
__device__ __forceinline__ void attn_bad_key(const AttnParams& P, int* bad, int key) {
    atomicMin(&bad[0], key); atomicMax(&bad[1], key + 1);
    atomicOr(&bad[2 + (key >> P.part_shift >> 5)], 1 << (key >> P.part_shift & 31));
}
// Elements d .. d + 3 of vector v of the values, as bits of floats
template <int KT>
__device__ __forceinline__ void attn_value4(const AttnParams& P, uint32_t v, int d, uint32_t* x) {
    const long long at = (long long)v * P.pages.D + d;
    if (KT == OC_DTYPE_F32) {
        const uint4 w = *(const uint4*)((const float*)P.v_pool + at);
        x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
    } else if (KT == OC_DTYPE_BF16) {
        const uint2 w = *(const uint2*)((const uint16_t*)P.v_pool + at);
        x[0] = w.x << 16; x[1] = w.x & 0xFFFF0000u; x[2] = w.y << 16; x[3] = w.y & 0xFFFF0000u;
    } else {
        const float s = P.v_scale[v];
        const uint32_t w = KT == OC_DTYPE_I8 ? *(const uint32_t*)((const uint8_t*)P.v_pool + at) : (uint32_t)*(const uint16_t*)((const uint8_t*)P.v_pool + (at >> 1));
#pragma unroll
        for (int e = 0; e < 4; ++e)
            x[e] = __float_as_uint(s * (float)(KT == OC_DTYPE_I8 ? (int)(w << (24 - 8 * e)) >> 24 : (int)(w << (28 - 4 * e)) >> 28));
    }
}
// The sums of what is no number in columns d .. d + 3 of the keys [lo, hi): 0 where there is nothing of the kind.
// (Sums of NaN stay what they are: the rest is not looked at.)
template <int KT>
__device__ __forceinline__ float4 attn_not_finite(const AttnParams& P, const int* bad, uint32_t seq, uint32_t head, int lo, int hi, int d) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int j = lo; j < hi;) {
        const int part = j >> P.part_shift;
        if (!(bad[2 + (part >> 5)] >> (part & 31) & 1)) {
            j = (int)min((long long)hi, (long long)(part + 1) << P.part_shift);
            continue;
        }
        const int end = min(hi, (j & ~15) + 16);                             // (pages have a multiple of 16 rows)
        const uint32_t pn = P.pages.page_rows.div((uint32_t)j);
        const int page = kv_page(P.pages, seq, pn);
        if (page < 0) { j = end; continue; }
        uint32_t v = kv_vector(P.pages, page, (uint32_t)j - pn * P.pages.page_rows.d) + head * P.pages.page_rows.d;
#pragma unroll 4
        for (; j < end; ++j, ++v) {
            uint32_t x[4];
            attn_value4<KT>(P, v, d, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) if ((x[e] & 0x7F800000u) == 0x7F800000u) sum[e] += __uint_as_float(x[e]);
        }
        if (isnan(sum[0]) && isnan(sum[1]) && isnan(sum[2]) && isnan(sum[3])) break;
    }
    return make_float4(sum[0], sum[1], sum[2], sum[3]);
}
__device__ __forceinline__ void attn_add4(float4& y, const float4& t) { y.x += t.x; y.y += t.y; y.z += t.z; y.w += t.w; }

// Whole numbers as pairs of bf16, which holds them exactly.
//   8 bits: u = x + 128 (the sign bit flipped) in the low byte of 0x4300 reads as 256 + x where x < 0, as 256 + 2x elsewhere (bit 7
//   falls on the exponent's last bit), so that with d = that - 256:  x = d - max(d, 0) / 2.  Three operations on the FMA
//   pipe, which the product's conversions leave idle; masks and subtractions that tell the cases apart take four on the integer
//   pipe, which has half its rate (single tokens over 8-bit caches: 185 us with those).
//   4 bits: u = x + 8 in the low bits of 0x4300 reads as 136 + x.
__device__ __forceinline__ uint32_t attn_i8_pair(uint32_t v) {                // 0x43uu 0x43uu
    uint32_t d = attn_fma2(v, 0x3F803F80u, 0xC380C380u), r;
    asm("fma.rn.relu.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(0x3F803F80u), "r"(0xC380C380u));
    return attn_fma2(r, 0xBF00BF00u, d);
}
__device__ __forceinline__ uint32_t attn_i4_pair(uint32_t v) { return attn_fma2((v & 0x000F000Fu) | 0x43004300u, 0x3F803F80u, 0xC308C308u); }

// Distributed shared memory of a cluster
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_map(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float cluster_ld(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 cluster_ld4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}

// The first and last of such keys of a cluster's CTAs; their parts join this CTA's
__device__ __forceinline__ void cluster_bad(int* bad, int ctas, int& first, int& end) {
    first = 0x7FFFFFFF; end = 0;
    for (int k = 0; k < ctas; ++k) {
        const uint32_t at = cluster_map(smem_u32(bad), (uint32_t)k);
        int a, b;
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(a) : "r"(at) : "memory");
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(b) : "r"(at + 4u) : "memory");
        first = min(first, a); end = max(end, b);
    }
    if (first >= end) return;
    for (int k = 0; k < ctas; ++k)
        for (int i = 2; i < ATT_BAD; ++i) {
            int w;
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(w) : "r"(cluster_map(smem_u32(bad + i), (uint32_t)k)) : "memory");
            atomicOr(&bad[i], w);
        }
}

// Four neighbouring elements of a row's result
template <int QT> __device__ __forceinline__ void attn_store4(const AttnParams& P, long long at, float4 v) {
    if (QT == OC_DTYPE_F32) {
        float* o = (float*)P.out + at;
        if (P.wide_out) st_v4(o, make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)));
        else { o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w; }
    } else {
        uint16_t* o = (uint16_t*)P.out + at;
        const uint32_t a = pack_bf16x2(v.x, v.y), b = pack_bf16x2(v.z, v.w);
        if (P.wide_out) *(uint2*)o = make_uint2(a, b);
        else { o[0] = (uint16_t)a; o[1] = (uint16_t)(a >> 16); o[2] = (uint16_t)b; o[3] = (uint16_t)(b >> 16); }
    }
}
#endif

}  // namespace oc
