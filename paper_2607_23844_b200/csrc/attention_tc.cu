// Attention over the paged cache on the tensor cores: bf16 queries, keys and values in bf16 or in 8 or 4 bits.
//     S = Q K^T,   P = exp2(S c - m c),   O = O + P V,   out = O / sum(P)          (c = scale * log2(e))
// A CTA takes NT tiles of 128 rows (a row is a query with one of the heads that share a head of the cache) and walks
// over the keys 128 at a time:
//   softmax warps   four for each tile of rows, a thread for each row: scores out of tensor memory, maximum, exponentials,
//                   sum, probabilities in bf16 back into tensor memory, where the second product reads them
//   copy warp       keys and values of the pages: TMA boxes (bf16), bulk copies (8 and 4 bits), into rings
//   MMA warps       tcgen05.mma, one for Q K^T from shared memory, one for P V with P in tensor memory and V as it lies (its
//                   rows are the product's inner axis)
//   helper warps    bf16: values that are no numbers become zeros (0 * NaN would reach the rows that do not see them), and their
//                   keys are kept for the rows that do; 8 and 4 bits: raw rows to bf16, which holds those whole
//                   numbers exactly, so that the scales join the scores and the probabilities
// Two tiles of rows take turns: while one's scores become probabilities the tensor cores work for the other.  With heads of up
// to 64 a third place for scores in tensor memory lets the products run ahead of the softmax warps.
// Measured (bf16): 25 x 4608 rows over 9216 keys, 5 heads of 64, 1359 GFLOP: 1.81 ms, 751 TFLOP/s; 2 x 2560 x 4096, 24 heads of 64:
// 214 us, 603 (480 CTAs are 3.2 rounds of the device's 148); 2 x 2048 x 4096, 16 heads of 128: 147 us, 935.  In 8 bits 330 us and 261.
// Probabilities are rounded to bf16: the second product takes both operands in one type, and values in bf16 as they are.
// What bounds heads of 64: a step (256 rows, 128 keys) takes 2500 to 2800 clocks, of which the products take 1024 and the
// exponentials 1790 (an eighth of them by polynomial), both warps of a scheduler together 1900 with all their instructions
// where nothing else runs; reading scores out of tensor memory beside running products costs 350, and each hand-over
// through a barrier 150 to 300.  Other splits were slower: P beside S with a place for each tile of rows (2.08 ms), one
// warp for both products (1.92), a pass for the maximum of its own (2.07), two CTAs of one tile on an SM (2.03).
// The maximum that a row subtracts only follows the running one when that is 2^8 ahead: rescaling O in tensor memory
// is then rare, and the sums lose nothing by it.
// Where there are few tiles, the CTAs of a cluster split the keys and join their sums through distributed shared memory.
#include <string.h>

#include <algorithm>
#include <numeric>
#include <type_traits>

#include "attention.cuh"
#include "attention_tc.cuh"
#include "tc_ptx.cuh"

namespace oc {

static constexpr int AT_ROWS = 128, AT_KEYS = 128, AT_SUB_BYTES = 128 * 128;   // a tile of 128 rows of 64 bf16
static constexpr int AT_SCALES = 4;                                             // stages of the ring of scales
// A row's maximum may lag behind by 8 powers of two and more: no more than this for the sum of a tile's exponentials.
static constexpr float AT_LAG = 8.0f, AT_SUM_MAX = 128.0f * 256.0f;

template <int NT, int SUB, int KT> struct At {
    static constexpr bool quant = KT == OC_DTYPE_I8 || KT == OC_DTYPE_I4;
    static constexpr int softmax_warps = 4 * NT, copy_warp = softmax_warps, score_warp = copy_warp + 1, output_warp = copy_warp + 2, helper0 = copy_warp + 3;
    static constexpr int helpers = quant ? 5 : 1, k_helpers = quant ? 3 : 0, v_helpers = helpers - k_helpers;         // of keys, of values
    static constexpr int warps = helper0 + helpers, threads = 32 * warps;
    // 8 and 4 bits: of the registers that a CTA is launched with (128 for each of 512 threads, 168 for each of 384) the softmax
    // warps take from the others: 2 x 128 x 176 + 2 x 128 x 80 = 512 x 128, 128 x 232 + 2 x 128 x 136 = 384 x 168.
    static constexpr int take_regs = !quant ? 0 : threads == 512 ? 176 : 232, give_regs = !quant ? 0 : threads == 512 ? 80 : 136;
    static_assert(!quant || threads == 512 || threads == 384, "registers of a CTA");
    // Which of 8 neighbouring pairs of exponentials come from the polynomial: what the FMA pipe has room for.  None, one, two:  25 x 4608 x
    // 9216, 5 heads of 64: 1809, 1735, 1760 us;  2 x 2560 x 4096, 24 heads of 64: 221, 214, 215;  2 x 2048 x 4096, 16 heads of 128:
    // 156, 152.  In 8 and 4 bits the scales take that pipe.
    static constexpr int poly = quant ? 0 : 0x01;
    static constexpr int chunk = 32;                                             // scores that a thread fetches at a time
    static constexpr int tile_bytes = SUB * AT_SUB_BYTES;                        // 128 keys (or rows) in bf16
    static constexpr int raw_bytes = KT == OC_DTYPE_I8 ? tile_bytes / 2 : tile_bytes / 4;        // (most) of 128 keys as they lie
    static constexpr int k_stages = quant ? (NT * SUB == 4 ? 1 : 2) : (SUB == 1 ? 3 : 2), v_stages = quant ? 2 : k_stages;
    static constexpr int rk_stages = quant ? 2 : 0, rv_stages = !quant ? 0 : (SUB == 2 && KT == OC_DTYPE_I8 ? 1 : 2), raw_stages = rk_stages + rv_stages;   // rows as they lie
    static constexpr int q_at = 0, k_at = NT * tile_bytes, v_at = k_at + k_stages * tile_bytes, raw_at = v_at + v_stages * tile_bytes;
    static constexpr int scale_at = raw_at + raw_stages * raw_bytes, rest_at = scale_at + (quant ? AT_SCALES * 2 * AT_KEYS * 4 : 0);
    // Tensor memory, all 512 columns: what is left beside O are places of 128 columns for scores, each taken over by its
    // probabilities.
    static constexpr int o_step = 64 * SUB, places = (512 - NT * o_step) / 128, o_col = places * 128;
    static constexpr bool one_warp = places == NT;                               // for both products
    static constexpr int n_bars = 2 * k_stages + 3 * v_stages + 2 * raw_stages + 3 * AT_SCALES + 3 * places + 3;
    static constexpr int smem = rest_at + n_bars * 8 + 64;
    static constexpr int out_stride = 64 * SUB + 4;                              // floats between rows where a cluster joins them
};

// A MN-major operand (V: rows of keys, the inner axis; 64 elements of N contiguous), 128-byte swizzle: groups of 8 keys
// 1024 bytes apart, the next 64 elements of N a sub-tile further.
__device__ __forceinline__ uint64_t at_desc_v(uint32_t addr) {
    const uint32_t lo = ((addr >> 4) & 0x3FFFu) | ((uint32_t)(AT_SUB_BYTES >> 4) << 16);
    const uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    return ((uint64_t)hi << 32) | lo;
}
// The products of one step of 64 elements or keys, 16 at a time, in one piece so that nothing the compiler schedules comes between
// them (the tensor cores take them faster than a warp computes operands).  Scores: both operands in shared memory, 32 bytes
// of their swizzled rows at a time, the first `steps` of the four.
__device__ __forceinline__ void at_mma_scores(uint32_t d, uint64_t q, uint64_t k, uint32_t idesc, uint32_t accumulate, int steps, uint32_t issue) {
    asm volatile(
        "{\n\t.reg .pred a, y, e;\n\t.reg .b64 q, k;\n\t"
        "setp.ne.b32 e, %6, 0;\n\tsetp.ne.b32 a, %4, 0;\n\tsetp.eq.b32 y, 0, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, a;\n\t"
        "setp.gt.and.s32 e, %5, 1, e;\n\tadd.u64 q, %1, 2;\n\tadd.u64 k, %2, 2;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], q, k, %3, y;\n\t"
        "setp.gt.and.s32 e, %5, 2, e;\n\tadd.u64 q, %1, 4;\n\tadd.u64 k, %2, 4;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], q, k, %3, y;\n\t"
        "setp.gt.and.s32 e, %5, 3, e;\n\tadd.u64 q, %1, 6;\n\tadd.u64 k, %2, 6;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], q, k, %3, y;\n\t}"
        :: "r"(d), "l"(q), "l"(k), "r"(idesc), "r"(accumulate), "r"(steps), "r"(issue) : "memory");
}
// Outputs: P in tensor memory, 8 columns for 16 keys; V 2048 bytes for them.
__device__ __forceinline__ void at_mma_outputs(uint32_t d, uint32_t p, uint64_t v, uint32_t idesc, uint32_t accumulate, uint32_t issue) {
    asm volatile(
        "{\n\t.reg .pred a, y, e;\n\t.reg .b64 v;\n\t.reg .b32 p;\n\t"
        "setp.ne.b32 e, %5, 0;\n\tsetp.ne.b32 a, %4, 0;\n\tsetp.eq.b32 y, 0, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, a;\n\t"
        "add.u32 p, %1, 8;\n\tadd.u64 v, %2, 128;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [p], v, %3, y;\n\t"
        "add.u32 p, %1, 16;\n\tadd.u64 v, %2, 256;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [p], v, %3, y;\n\t"
        "add.u32 p, %1, 24;\n\tadd.u64 v, %2, 384;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [p], v, %3, y;\n\t}"
        :: "r"(d), "r"(p), "l"(v), "r"(idesc), "r"(accumulate), "r"(issue) : "memory");
}
__device__ __forceinline__ void at_tmem_st16(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        :: "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
           "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void at_tmem_ld16(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void at_tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void at_tma_2d(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar, uint32_t issue) {
    asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %5, 0;\n\t"
                 "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
                 :: "r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar), "r"(issue) : "memory");
}
__device__ __forceinline__ void at_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint32_t issue) {
    asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %4, 0;\n\t"
                 "@e cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar), "r"(issue) : "memory");
}
__device__ __forceinline__ float at_max3(float a, float b, float c) {            // NaN if one of them is
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float at_exp2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// 2^x of two numbers without the special function unit, which gives 16 a clock and SM: x = n + f with n whole and
// 0 <= f < 1, 2^f = 1 + f (a + f (b + f (c + f (d + f e)))) (minimax for a polynomial through 1 by Remez' exchange, its
// coefficients rounded to fp32 one after the other; relative error in fp32 2.5e-7, that of the unit: the log-sum-exp is as good as
// the other form's, which it was not with two terms less, 8.6e-5).  n is added to the exponent.  What is below -127 becomes 0, what
// is above 127 2^127.
__device__ __forceinline__ float at_clamp(float x) {
    float r;
    asm("{\n\t.reg .f32 t;\n\tmax.NaN.f32 t, %1, 0fC2FE0000;\n\tmin.NaN.f32 %0, t, 0f42FE0000;\n\t}" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ f32x2 at_exp2_poly(f32x2 x) {
    x = f2(at_clamp(f2_lo(x)), at_clamp(f2_hi(x)));
    const f32x2 big = f2(12582912.0f);                                           // 1.5 * 2^23: the sum's last bits are n
    f32x2 y;
    asm("add.rm.f32x2 %0, %1, %2;" : "=l"(y) : "l"(x), "l"(big));
    const f32x2 f = f2_add(x, f2_fma(y, f2(-1.0f), big));
    f32x2 p = f2_fma(f, f2(0.0018613838f), f2(0.009022821f));
    p = f2_fma(p, f, f2(0.055799514f));
    p = f2_fma(p, f, f2(0.2401646f));
    p = f2_fma(p, f, f2(0.6931513f));
    p = f2_fma(p, f, f2(1.0f));
    return f2_bits(__float_as_uint(f2_lo(p)) + (__float_as_uint(f2_lo(y)) << 23), __float_as_uint(f2_hi(p)) + (__float_as_uint(f2_hi(y)) << 23));
}

// 8 whole numbers as bf16
__device__ __forceinline__ uint4 at_widen_i8(uint2 w) {
    w.x ^= 0x80808080u; w.y ^= 0x80808080u;
    return make_uint4(attn_i8_pair(__byte_perm(w.x, 0x43434343u, 0x4140u)), attn_i8_pair(__byte_perm(w.x, 0x43434343u, 0x4342u)),
                      attn_i8_pair(__byte_perm(w.y, 0x43434343u, 0x4140u)), attn_i8_pair(__byte_perm(w.y, 0x43434343u, 0x4342u)));
}
__device__ __forceinline__ uint4 at_widen_i4(uint32_t w) {
    w ^= 0x88888888u;
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const uint32_t x = __byte_perm(w, 0u, 0x4440u + i); o[i] = attn_i4_pair(x | x << 12); }      // elements 2i and 2i + 1
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// Registers that warps give back and that the softmax warps take (whole warpgroups do the same)
template <int REGS> __device__ __forceinline__ void at_give() { if constexpr (REGS > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(REGS)); }
template <int REGS> __device__ __forceinline__ void at_take() { if constexpr (REGS > 0) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(REGS)); }

struct AttnTcParams {
    AttnParams a;
    CUtensorMap mapK, mapV;          // bf16: {head_dim, vectors of the pool}, boxes {64, box_rows}
    int box_rows;                    // rows that a copy takes: the largest piece of 128 keys that no page boundary cuts
    int n_boxes, row_bytes;
    FastDiv group, units;
};

template <int NT, int SUB, int KT>
__global__ void __launch_bounds__((At<NT, SUB, KT>::threads), 1)
attention_tc_kernel(const __grid_constant__ AttnTcParams TP) {
    using A = At<NT, SUB, KT>;
    const AttnParams& P = TP.a;
    extern __shared__ __align__(1024) uint8_t at_smem[];
    __shared__ int s_range[NT][2];                                               // of each tile: first key seen, last
    __shared__ float s_stats[NT * AT_ROWS][2], s_share[NT * AT_ROWS];             // maxima and sums; weights of the cluster's parts
    __shared__ __align__(16) float s_ones[A::quant ? AT_KEYS : 4];
    __shared__ unsigned char s_there[NT * AT_ROWS];
    __shared__ int s_bad[ATT_BAD];                                                     // keys with values that are no numbers
    const uint32_t smem = smem_u32(at_smem);
    uint64_t* bars = (uint64_t*)(at_smem + A::rest_at);
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t k_full = bar0, k_empty = k_full + 8 * A::k_stages, v_full = k_empty + 8 * A::k_stages, v_ready = v_full + 8 * A::v_stages;
    const uint32_t v_empty = v_ready + 8 * A::v_stages, raw_full = v_empty + 8 * A::v_stages, raw_empty = raw_full + 8 * A::raw_stages;
    const uint32_t sc_full = raw_empty + 8 * A::raw_stages, sc_empty = sc_full + 8 * AT_SCALES;
    const uint32_t sc_ready = sc_empty + 8 * AT_SCALES, s_full = sc_ready + 8 * AT_SCALES, p_ready = s_full + 8 * A::places, p_done = p_ready + 8 * A::places, drain = p_done + 8 * A::places, q_ready = drain + 16;
    uint32_t* tmem_slot = (uint32_t*)(bars + A::n_bars);
    volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = P.pages.D;

    if (A::quant && threadIdx.x < AT_KEYS) s_ones[threadIdx.x] = 1.0f;
    if (smem & 1023u) {                                                          // never expected; refuse rather than compute garbage
        if (threadIdx.x == 0) atomicCAS(P.pages.status, 0, OC_ERR_ALIGNMENT);
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < A::k_stages; ++i) { mbar_init(k_full + 8 * i, A::quant ? A::k_helpers : 1); mbar_init(k_empty + 8 * i, 1); }
        for (int i = 0; i < A::v_stages; ++i) { mbar_init(v_full + 8 * i, 1); mbar_init(v_ready + 8 * i, A::v_helpers); mbar_init(v_empty + 8 * i, 1); }
        for (int i = 0; i < A::raw_stages; ++i) { mbar_init(raw_full + 8 * i, 1); mbar_init(raw_empty + 8 * i, i < A::rk_stages ? A::k_helpers : A::v_helpers); }
        for (int i = 0; i < AT_SCALES; ++i) { mbar_init(sc_full + 8 * i, 1); mbar_init(sc_ready + 8 * i, 1); mbar_init(sc_empty + 8 * i, A::softmax_warps); }
        for (int i = 0; i < A::places; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(p_ready + 8 * i, 4); mbar_init(p_done + 8 * i, 1); }
        mbar_init(drain, 1); mbar_init(drain + 8, 1); mbar_init(q_ready, A::softmax_warps);
        *abort_flag = 0;
        attn_bad_none(s_bad);
        for (int t = 0; t < NT; ++t) { s_range[t][0] = 0x7FFFFFFF; s_range[t][1] = 0; }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (!A::quant && P.pages.n_tokens > 0) { tma_prefetch_map(&TP.mapK); tma_prefetch_map(&TP.mapV); }      // (there are none for a cache of no tokens)
    }
    pdl_wait();
    const uint32_t rank = P.split > 1 ? cluster_rank() : 0u;
    const AttnTile T = attn_tile(P, blockIdx.x / (uint32_t)P.split);
    const AttnSeq S = attn_seq(P, T.seq);
    const uint32_t first = T.tile * (uint32_t)(NT * AT_ROWS), rows = (uint32_t)S.n * (uint32_t)P.group;
    if (first >= rows) return;                                                   // (the whole cluster; nothing is allocated yet)
    // (registers leave room for one CTA of this kernel on an SM, so no cluster waits here for what another cluster's CTA holds)
    if (warp == A::score_warp) tmem_alloc_cta1(smem_u32(tmem_slot), 512);
    __syncwarp();
    __syncthreads();                                                             // (the ranges are set up)
    // ---- rows: which keys they see ----
    const int my_tile = warp >> 2, my_row = (warp & 3) * 32 + lane;              // of a softmax thread
    bool exists = false;
    int lo = 0, hi = 0, qi = 0, qg = 0;
    if (warp < A::softmax_warps) {
        const uint32_t r = first + (uint32_t)(my_tile * AT_ROWS + my_row);
        if (r < rows) {
            qi = (int)TP.group.div(r); qg = (int)(r - (uint32_t)qi * TP.group.d);
            exists = attn_bounds(P, S, T.seq, qi, lo, hi);
            if (exists && lo < hi) {
                atomicMin(&s_range[my_tile][0], lo); atomicMax(&s_range[my_tile][1], hi);
            } else {
                lo = hi = 0;
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __reduce_max_sync(0xFFFFFFFFu, *tmem_slot);             // (known to be the same in all lanes)
    // (not before this CTA has its tensor memory: a kernel that takes its own before it waits for this one could have it)
    if (threadIdx.x == 0) pdl_launch_dependents();
    // Tiles of keys [a, b) of each tile of rows; this CTA's share of them all.
    int ka[NT], kb[NT], j0 = 0x7FFFFFFF, j1 = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const bool any = s_range[t][1] > 0;                                      // (some row sees a key)
        ka[t] = any ? s_range[t][0] / AT_KEYS : 0; kb[t] = any ? (s_range[t][1] + AT_KEYS - 1) / AT_KEYS : 0;
        if (any) { j0 = min(j0, ka[t]); j1 = max(j1, kb[t]); }
    }
    if (j1 == 0) j0 = 0;
    if (P.split > 1) {
        const int n = j1 - j0, a = (int)((long long)n * rank / P.split), b = (int)((long long)n * (rank + 1) / P.split);
        j1 = j0 + b; j0 += a;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) { ka[t] = max(ka[t], j0); kb[t] = max(min(kb[t], j1), ka[t]); }
    auto on = [&](int j, int t) { return j >= ka[t] && j < kb[t]; };
    // Products of scores in the order of their issue: tile of keys after tile of keys, the tiles of rows in turn.  Product i has
    // place i % places (also one that a tile of rows does not need: nothing is computed for it).
    bool ok = true;
#define AT_WAIT(bar, parity) (ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait((bar), (parity), abort_flag)))

    if (warp >= A::softmax_warps) {
    at_give<A::give_regs>();
    if (warp == A::copy_warp) {
        // ================================ copies ================================================
        const uint32_t issue = elect_one();
        // the pool's vector where box `lane` of a tile begins (-1: a page that is not there, -2: behind the last key)
        auto find = [&](int j) -> int {
            const int key = j * AT_KEYS + lane * TP.box_rows;
            if (lane >= TP.n_boxes || key >= S.len) return -2;
            const uint32_t pn = P.pages.page_rows.div((uint32_t)key);
            const int page = kv_page(P.pages, T.seq, pn);
            return page < 0 ? -1 : (int)(kv_vector(P.pages, page, (uint32_t)key - pn * P.pages.page_rows.d) + T.head * P.pages.page_rows.d);
        };
        uint32_t bytes_pending = 0;
        if (!A::quant) {
            int stage = 0; uint32_t phase = 0;
            int at = j0 < j1 ? find(j0) : -2, at_v = at;
            const int vectors = (int)(P.pages.n_pages * (uint32_t)P.pages.heads * P.pages.page_rows.d);
            auto load = [&](const CUtensorMap* map, uint32_t to, uint32_t bar, int where) {
                uint32_t boxes = 0;
                for (int b = 0; b < TP.n_boxes; ++b) {
                    const int v = __shfl_sync(0xFFFFFFFFu, where, b);
                    if (v == -2) break;
#pragma unroll
                    for (int s = 0; s < SUB; ++s)                                // (a box wholly outside the pool is filled with zeros)
                        at_tma_2d(to + (uint32_t)(s * AT_SUB_BYTES + b * TP.box_rows * 128), map, 64 * s, v < 0 ? vectors : v, bar, issue);
                    ++boxes;
                }
                mbar_arrive_expect_tx_elected(bar, boxes * (uint32_t)(TP.box_rows * 128 * SUB), issue);
                bytes_pending = bar;
            };
            // keys of a tile are wanted one tile before its values
            for (int j = j0; j < j1 + 1 && ok; ++j) {
                const int next = j + 1 < j1 ? find(j + 1) : -2;
                if (j < j1) {
                    const int st = (j - j0) % A::k_stages; const uint32_t ph = (uint32_t)((j - j0) / A::k_stages) & 1u;
                    if (!AT_WAIT(k_empty + 8 * st, ph ^ 1u)) break;
                    load(&TP.mapK, smem + A::k_at + (uint32_t)(st * A::tile_bytes), k_full + 8 * st, at);
                }
                if (j > j0) {
                    if (!AT_WAIT(v_empty + 8 * stage, phase ^ 1u)) break;
                    load(&TP.mapV, smem + A::v_at + (uint32_t)(stage * A::tile_bytes), v_full + 8 * stage, at_v);
                    if (++stage == A::v_stages) { stage = 0; phase ^= 1u; }
                }
                at_v = at; at = next;
            }
        } else {
            int at = j0 < j1 ? find(j0) : -2, at_v = at;
            auto load = [&](const void* pool, int stage, uint32_t phase, int where) {
                if (!AT_WAIT(raw_empty + 8 * stage, phase ^ 1u)) return;
                const uint32_t to = smem + A::raw_at + (uint32_t)(stage * A::raw_bytes), bar = raw_full + 8 * stage, bytes = (uint32_t)(TP.box_rows * TP.row_bytes);
                uint32_t boxes = 0;
                for (int b = 0; b < TP.n_boxes; ++b) {
                    const int v = __shfl_sync(0xFFFFFFFFu, where, b);
                    if (v < 0) continue;
                    at_bulk(to + (uint32_t)b * bytes, (const uint8_t*)pool + (long long)v * TP.row_bytes, bytes, bar, issue);
                    ++boxes;
                }
                mbar_arrive_expect_tx_elected(bar, boxes * bytes, issue);
                bytes_pending = bar;
            };
            constexpr int RK = A::quant ? A::rk_stages : 1, RV = A::quant ? A::rv_stages : 1;
            for (int j = j0; j < j1 + 1 && ok; ++j) {
                const int next = j + 1 < j1 ? find(j + 1) : -2;
                if (j < j1) {
                    load(P.k_pool, (j - j0) % RK, (uint32_t)((j - j0) / RK) & 1u, at);
                    const int st = (j - j0) % AT_SCALES; const uint32_t ph = (uint32_t)((j - j0) / AT_SCALES) & 1u;
                    if (!ok || !AT_WAIT(sc_empty + 8 * st, ph ^ 1u)) break;
                    const uint32_t to = smem + A::scale_at + (uint32_t)(st * 2 * AT_KEYS * 4), bytes = (uint32_t)TP.box_rows * 4u;
                    uint32_t boxes = 0;
                    bool zeros = false;
                    for (int b = 0; b < TP.n_boxes; ++b) {
                        const int v = __shfl_sync(0xFFFFFFFFu, at, b);
                        if (v == -2) break;
                        if (v == -1) {                                           // (a page that is not there: values of zero)
                            for (int i = lane; i < TP.box_rows; i += 32) {
                                asm volatile("st.shared.b32 [%0], %1;" :: "r"(to + (uint32_t)b * bytes + 4u * i), "r"(0u) : "memory");
                                asm volatile("st.shared.b32 [%0], %1;" :: "r"(to + AT_KEYS * 4u + (uint32_t)b * bytes + 4u * i), "r"(0u) : "memory");
                            }
                            zeros = true;
                            continue;
                        }
                        at_bulk(to + (uint32_t)b * bytes, P.k_scale + v, bytes, sc_full + 8 * st, issue);
                        at_bulk(to + AT_KEYS * 4u + (uint32_t)b * bytes, P.v_scale + v, bytes, sc_full + 8 * st, issue);
                        ++boxes;
                    }
                    if (zeros) __syncwarp();
                    mbar_arrive_expect_tx_elected(sc_full + 8 * st, 2 * boxes * bytes, issue);
                }
                if (j > j0) load(P.v_pool, RK + (j - 1 - j0) % RV, (uint32_t)((j - 1 - j0) / RV) & 1u, at_v);
                at_v = at; at = next;
            }
        }
        if (!ok && lane == 0) {
            atomicCAS(P.pages.status, 0, OC_ERR_TIMEOUT);
            *abort_flag = 1;
            // copies already issued still write this CTA's shared memory: a bounded chance to land
            if (bytes_pending) { const unsigned long long t0 = global_ns(); while (global_ns() - t0 < 20000000ull) {} }
        }
    } else if (warp == A::score_warp || warp == A::output_warp) {
        // ================================ MMAs ==================================================
        // A warp for each of the two products: waiting, computing operands and issuing take one nearly as long as the products take
        // the tensor cores.  With two places only, one warp does both: the scores of product i + 2 then follow the outputs of
        // product i in the tensor cores' queue without a barrier between them, and overwrite its probabilities in time.
        const uint32_t issue = elect_one();
        const int n_keys = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)(j1 - j0));                // (known to be the same in all lanes)
        constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(AT_KEYS >> 3) << 17) | ((uint32_t)(AT_ROWS >> 4) << 24);
        const int steps = (D + 15) / 16;
        const uint32_t n_out = (uint32_t)(D + 15) / 16u * 16u;
        const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((n_out >> 3) << 17) | ((uint32_t)(AT_ROWS >> 4) << 24);
        int ks = 0, vs = 0, ps = 0, po = 0;                                      // stages of keys and values; places of scores and outputs
        uint32_t kp = 0, vp = 0, pp = 0, sp = 1u;                                // their phases (the places begin empty)
        uint32_t begun[NT] = {};
        if (warp == A::score_warp) AT_WAIT(q_ready, 0u);
        auto scores = [&](int j, int t) {                                        // t: known when this is compiled
            if (j >= n_keys || !ok) return;
            if (t == 0) { if (!AT_WAIT(k_full + 8 * ks, kp)) return; tc_fence_after(); }
            if (!A::one_warp) { if (!AT_WAIT(p_done + 8 * ps, sp)) return; tc_fence_after(); }      // the probabilities that were there have been used
            if (on(j0 + j, t)) {
                const uint64_t q = make_smem_desc(smem + A::q_at + (uint32_t)(t * A::tile_bytes)), k = make_smem_desc(smem + A::k_at + (uint32_t)(ks * A::tile_bytes));
                at_mma_scores(tmem + (uint32_t)(ps * 128), q, k, IDESC_S, 0u, steps, issue);
                if (SUB == 2) at_mma_scores(tmem + (uint32_t)(ps * 128), q + (AT_SUB_BYTES >> 4), k + (AT_SUB_BYTES >> 4), IDESC_S, 1u, steps - 4, issue);
            }
            tc_commit<false>(s_full + 8 * ps, issue);
            if (++ps == A::places) { ps = 0; sp ^= 1u; }
            if (t == NT - 1) { tc_commit<false>(k_empty + 8 * ks, issue); if (++ks == A::k_stages) { ks = 0; kp ^= 1u; } }
        };
        auto outputs = [&](int j, int t) {
            if (!ok) return;
            if (t == 0 && !AT_WAIT(v_ready + 8 * vs, vp)) return;
            if (!AT_WAIT(p_ready + 8 * po, pp)) return;
            tc_fence_after();
            if (on(j0 + j, t)) {
                const uint64_t v = at_desc_v(smem + A::v_at + (uint32_t)(vs * A::tile_bytes));
                const uint32_t o = tmem + (uint32_t)(A::o_col + t * A::o_step), p = tmem + (uint32_t)(po * 128);
                at_mma_outputs(o, p, v, idesc_o, begun[t], issue);
                at_mma_outputs(o, p + 32u, v + 512u, idesc_o, 1u, issue);
                begun[t] = 1u;
            }
            tc_commit<false>(p_done + 8 * po, issue);
            if (++po == A::places) { po = 0; pp ^= 1u; }
            if (t == NT - 1) { tc_commit<false>(v_empty + 8 * vs, issue); if (++vs == A::v_stages) { vs = 0; vp ^= 1u; } }
        };
        if (A::one_warp) {
            if (warp == A::score_warp) {
#pragma unroll
                for (int t = 0; t < NT; ++t) scores(0, t);
                for (int j = 0; j < n_keys && ok; ++j)
#pragma unroll
                    for (int t = 0; t < NT; ++t) { outputs(j, t); scores(j + 1, t); }
            }
        } else if (warp == A::score_warp) {
            for (int j = 0; j < n_keys && ok; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t) scores(j, t);
        } else {
            for (int j = 0; j < n_keys && ok; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t) outputs(j, t);
        }
        if (!ok && lane == 0) { atomicCAS(P.pages.status, 0, OC_ERR_TIMEOUT); *abort_flag = 1; }
        // every MMA retires before tensor memory is released
        const uint32_t over = drain + (warp == A::output_warp ? 8u : 0u);
        tc_commit<false>(over, issue);
        const unsigned long long t0 = global_ns();
        while (!mbar_try_wait(over, 0) && global_ns() - t0 < WAIT_LIMIT_NS) {}
    } else {
        // ================================ helpers ===============================================
        const int h = warp - A::helper0;
        if (!A::quant) {
            for (int j = j0; j < j1; ++j) {
                const int st = (j - j0) % A::v_stages;
                if (!AT_WAIT(v_full + 8 * st, (uint32_t)((j - j0) / A::v_stages) & 1u)) break;
                const int key0 = j * AT_KEYS;
                const uint32_t base = smem + A::v_at + (uint32_t)(st * A::tile_bytes);
                uint32_t zero[4] = {};
#pragma unroll 8
                for (int i = h * 32 + lane; i < SUB * 1024; i += 32 * A::helpers) {              // pieces of 16 bytes
                    uint32_t w[4];
                    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(base + (uint32_t)(i * 16)) : "memory");
#pragma unroll
                    for (int e = 0; e < 4; ++e) zero[e] = attn_zero2(zero[e], w[e]);
                }
                if (__any_sync(0xFFFFFFFFu, attn_bad2(zero[0] | zero[1] | zero[2] | zero[3]))) {
                    int bad_first = 0x7FFFFFFF, bad_last = -1;
                    for (int i = h * 32 + lane; i < SUB * 1024; i += 32 * A::helpers) {
                        const uint32_t at = base + (uint32_t)(i * 16);
                        const int key = key0 + ((i >> 3) & 127);
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
                        bool change = false;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool a = (w[e] & 0x7F80u) == 0x7F80u, b = (w[e] & 0x7F800000u) == 0x7F800000u;
                            change |= a || b;
                            w[e] &= (a ? 0u : 0xFFFFu) | (b ? 0u : 0xFFFF0000u);
                        }
                        if (!change) continue;
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                        if (key < S.len) { bad_first = min(bad_first, key); bad_last = max(bad_last, key); }     // (behind the sequence lies anything)
                    }
                    if (bad_last >= 0) { attn_bad_key(P, s_bad, bad_first); attn_bad_key(P, s_bad, bad_last); }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(v_ready + 8 * st);
            }
        } else {
            const int units = D / 8, items = AT_KEYS * units;                    // of 8 elements, in the order in which they lie
            const bool value = h >= A::k_helpers;                                // this warp's share of the keys, or of the values
            const int ways = value ? A::v_helpers : A::k_helpers, share = value ? h - A::k_helpers : h;
            const int stages = value ? A::v_stages : A::k_stages, at0 = value ? A::v_at : A::k_at;
            // the elements that fill up a product's step of 16 are zeros for good
            if (units & 1)
                for (int i = share * 32 + lane; i < stages * AT_KEYS; i += 32 * ways) {
                    const uint32_t at = smem + (uint32_t)(at0 + (i >> 7) * A::tile_bytes + (units >> 3) * AT_SUB_BYTES + (i & 127) * 128 + (((units & 7) ^ (i & 7)) << 4));
                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" :: "r"(at), "r"(0u) : "memory");
                }
            auto widen = [&](uint32_t raw, uint32_t base) {
                constexpr int BATCH = 4;                                         // (loads on their way together)
                for (int i0 = share * 32 + lane; i0 < items; i0 += 32 * ways * BATCH) {
                    uint2 w[BATCH];
#pragma unroll
                    for (int b = 0; b < BATCH; ++b) {
                        const int i = i0 + b * 32 * ways;
                        w[b] = make_uint2(0u, 0u);
                        if (i >= items) break;
                        if (KT == OC_DTYPE_I8) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(w[b].x), "=r"(w[b].y) : "r"(raw + 8u * i) : "memory");
                        else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[b].x) : "r"(raw + 4u * i) : "memory");
                    }
#pragma unroll
                    for (int b = 0; b < BATCH; ++b) {
                        const int i = i0 + b * 32 * ways;
                        if (i >= items) break;
                        const uint32_t r = TP.units.div((uint32_t)i), u = (uint32_t)i - r * TP.units.d;
                        const uint4 v = KT == OC_DTYPE_I8 ? at_widen_i8(w[b]) : at_widen_i4(w[b].x);
                        const uint32_t at = base + (u >> 3) * AT_SUB_BYTES + r * 128u + (((u & 7u) ^ (r & 7u)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            };
            constexpr int RK = A::quant ? A::rk_stages : 1, RV = A::quant ? A::rv_stages : 1;
            const int raws = value ? RV : RK, raw0 = value ? RK : 0;
            for (int j = j0; j < j1 && ok; ++j) {
                const int i = j - j0, st = i % stages, rs = raw0 + i % raws;
                const uint32_t empty = (value ? v_empty : k_empty) + 8 * st, full = (value ? v_ready : k_full) + 8 * st;
                if (h == 0) {
                    const int sst = i % AT_SCALES;
                    if (!AT_WAIT(sc_full + 8 * sst, (uint32_t)(i / AT_SCALES) & 1u)) break;
                    // the softmax scale joins the keys' (one product less for each score); values' scales that are no numbers: as in bf16
                    float* of_k = (float*)(at_smem + A::scale_at) + 2 * sst * AT_KEYS + lane, *of_v = of_k + AT_KEYS, k4[4], zero = 0.0f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) { k4[k] = of_k[32 * k]; zero = fmaf(of_v[32 * k], 0.0f, zero); }
#pragma unroll
                    for (int k = 0; k < 4; ++k) of_k[32 * k] = k4[k] * P.scale_log2;
                    if (__any_sync(0xFFFFFFFFu, zero != 0.0f))
#pragma unroll 1
                        for (int k = 0; k < AT_KEYS; k += 32)
                            if (!isfinite(of_v[k])) { of_v[k] = 0.0f; if (j * AT_KEYS + k + lane < S.len) attn_bad_key(P, s_bad, j * AT_KEYS + k + lane); }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); // (written again by copies)
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sc_ready + 8 * sst);
                }
                if (!AT_WAIT(raw_full + 8 * rs, (uint32_t)(i / raws) & 1u) || !AT_WAIT(empty, ((uint32_t)(i / stages) & 1u) ^ 1u)) break;
                widen(smem + A::raw_at + (uint32_t)(rs * A::raw_bytes), smem + (uint32_t)(at0 + st * A::tile_bytes));
                if (lane == 0) { mbar_arrive(full); mbar_arrive(raw_empty + 8 * rs); }
            }
        }
        if (!ok && lane == 0) { atomicCAS(P.pages.status, 0, OC_ERR_TIMEOUT); *abort_flag = 1; }
    }
    } else {
        // ================================ softmax ===============================================
        at_take<A::take_regs>();
        // queries into shared memory (rows that are not there as zeros), 8 pieces of 16 bytes on their way at a time
        constexpr int UN = SUB * 8, BATCH = 8;
        for (int i0 = threadIdx.x; i0 < NT * AT_ROWS * UN; i0 += 32 * A::softmax_warps * BATCH) {
            uint4 v[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int i = i0 + b * 32 * A::softmax_warps, rr = i / UN, u = i % UN;
                const uint32_t r2 = first + (uint32_t)rr;
                v[b] = make_uint4(0, 0, 0, 0);
                if (r2 < rows && 8 * u < D) {
                    const uint32_t q2 = TP.group.div(r2);
                    const uint16_t* q = (const uint16_t*)P.q + attn_q_at(P, S, T.seq, (int)q2, (int)T.head * P.group + (int)(r2 - q2 * TP.group.d)) + 8 * u;
                    if (P.wide_q) v[b] = *(const uint4*)q;
                    else v[b] = make_uint4((uint32_t)q[0] | (uint32_t)q[1] << 16, (uint32_t)q[2] | (uint32_t)q[3] << 16,
                                           (uint32_t)q[4] | (uint32_t)q[5] << 16, (uint32_t)q[6] | (uint32_t)q[7] << 16);
                }
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int i = i0 + b * 32 * A::softmax_warps, rr = i / UN, u = i % UN;
                const uint32_t at = smem + A::q_at + (uint32_t)((rr >> 7) * A::tile_bytes + (u >> 3) * AT_SUB_BYTES + (rr & 127) * 128 + (((u & 7) ^ (rr & 7)) << 4));
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(v[b].x), "r"(v[b].y), "r"(v[b].z), "r"(v[b].w) : "memory");
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(q_ready);
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t o_at = t_lane + (uint32_t)(A::o_col + my_tile * A::o_step);
        int used = -1;                                                           // the last product of this tile of rows, until it is known to have retired
        const int my_a = my_tile == 0 ? ka[0] : ka[NT - 1], my_b = my_tile == 0 ? kb[0] : kb[NT - 1];
        const float c = A::quant ? 1.0f : P.scale_log2;                          // (in 8 and 4 bits it is in the keys' scales)
        float m = exists && lo < hi ? -INFINITY : 0.0f, l = 0.0f;                                           // what the row subtracts; its sum
        int n = 0;                                                               // tiles of keys done
        for (int j = j0; j < j1 && ok; ++j) {
            const int sst = (j - j0) % AT_SCALES;
            if (A::quant && (j < my_a || j >= my_b)) {
                if (!AT_WAIT(sc_ready + 8 * sst, (uint32_t)((j - j0) / AT_SCALES) & 1u)) break;
                if (lane == 0) mbar_arrive(sc_empty + 8 * sst);
            }
            const int product = NT * (j - j0) + my_tile, place = product % A::places;
            const uint32_t s_at = t_lane + (uint32_t)(place * 128);              // (and of the probabilities)
            if (!AT_WAIT(s_full + 8 * place, (uint32_t)(product / A::places) & 1u)) break;
            if (j < my_a || j >= my_b) {                                         // not needed
                // (The tile's last product retires before this warp lets any later one begin: the place's barrier goes on to phases of the
                // other tile's products, among them one of the same parity, so that a later look could miss the phase meant here.)
                if (used >= 0) {
                    if (!AT_WAIT(p_done + 8 * (used % A::places), (uint32_t)(used / A::places) & 1u)) break;
                    used = -1;
                }
                if (lane == 0) mbar_arrive(p_ready + 8 * place);
                continue;
            }
            tc_fence_after();
            if (A::quant && !AT_WAIT(sc_ready + 8 * sst, (uint32_t)((j - j0) / AT_SCALES) & 1u)) break;
            const int key0 = j * AT_KEYS;
            const bool cut = __any_sync(0xFFFFFFFFu, exists && lo < hi && (key0 < lo || key0 + AT_KEYS > hi));
            constexpr int CH = A::chunk;
            auto fetch = [&](int i, uint32_t* x) { tmem_ld32(s_at + 32u * i, x); };
            auto mask = [&](int i, uint32_t* x) {
                const int first_seen = lo - key0 - CH * i, end_seen = hi - key0 - CH * i;
#pragma unroll
                for (int e = 0; e < CH; ++e) if (e < first_seen || e >= end_seen) x[e] = 0xFF800000u;
            };
            // (masked scores have their keys' scales already: a scale of 0 would make NaN of -infinity)
            const float* ks = !A::quant || cut ? s_ones : (const float*)(at_smem + A::scale_at) + 2 * sst * AT_KEYS;
            const float* vs = (const float*)(at_smem + A::scale_at) + (2 * sst + 1) * AT_KEYS;
            auto scaled = [&](int i, uint32_t* x, const float* by) {             // keys CH i ..
#pragma unroll
                for (int e = 0; e < CH; e += 4) {
                    const float4 k = *(const float4*)(by + CH * i + e);
                    const f32x2 u = f2_mul(f2_bits(x[e], x[e + 1]), f2(k.x, k.y)), v = f2_mul(f2_bits(x[e + 2], x[e + 3]), f2(k.z, k.w));
                    x[e] = __float_as_uint(f2_lo(u)); x[e + 1] = __float_as_uint(f2_hi(u)); x[e + 2] = __float_as_uint(f2_lo(v)); x[e + 3] = __float_as_uint(f2_hi(v));
                }
            };
            auto fetched = [&](int i, uint32_t* x) { if (A::quant) scaled(i, x, ks); };
            if (cut) {                                                           // masked in their place: the code below is without
#pragma unroll 1
                for (int i = 0; i < 128 / CH; ++i) {
                    uint32_t x[CH];
                    fetch(i, x);
                    tmem_ld_wait();
                    if (A::quant) scaled(i, x, (const float*)(at_smem + A::scale_at) + 2 * sst * AT_KEYS);
                    mask(i, x);
#pragma unroll
                    for (int e = 0; e < CH; e += 16) at_tmem_st16(s_at + (uint32_t)(CH * i + e), x + e);
                }
                at_tmem_st_wait();
            }
            // The exponentials are taken with the maximum of the tiles before.  Only where that shows to be too small (the tile's sum
            // is above AT_SUM_MAX: some exponent is above 8), or nothing has been seen yet, the scores are fetched again for their
            // maximum, what has been summed up is rescaled, and the exponentials are taken anew: a tile or two of a sequence.
            uint32_t w[64];
            f32x2 sum[2];
            bool search = __any_sync(0xFFFFFFFFu, m == -INFINITY);
            for (;;) {
                if (search) {
                    float most[2] = {m, -INFINITY};
#pragma unroll 1
                    for (int i = 0; i < 128 / CH; ++i) {
                        uint32_t x[CH];
                        fetch(i, x);
                        tmem_ld_wait();
                        fetched(i, x);
#pragma unroll
                        for (int e = 0; e < CH; e += 4)
#pragma unroll
                            for (int f = 0; f < 2; ++f) most[f] = at_max3(most[f], __uint_as_float(x[e + 2 * f]), __uint_as_float(x[e + 2 * f + 1]));
                    }
                    // (a maximum of NaN is passed on to the whole row; that of +infinity makes every exponential of the row NaN)
                    const float top = at_max3(most[0], most[1], most[1]), to = top == INFINITY ? __int_as_float(0x7FFFFFFF) : top;
                    const float corr = to == -INFINITY ? 1.0f : at_exp2((m - to) * c);
                    if (n > 0) {
                        if (!AT_WAIT(p_done + 8 * (used % A::places), (uint32_t)(used / A::places) & 1u)) break;
                        tc_fence_after();
                        for (int d = 0; d < D; d += 16) {
                            uint32_t o[16];
                            at_tmem_ld16(o_at + (uint32_t)d, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(m == -INFINITY ? 0.0f : __uint_as_float(o[i]) * corr);
                            at_tmem_st16(o_at + (uint32_t)d, o);
                        }
                        at_tmem_st_wait();
                        tc_fence_before();
                    }
                    l *= corr;
                    m = to;
                }
                const float shift = m == -INFINITY ? 0.0f : -m * c;              // (nothing seen so far: every p is 0)
                const f32x2 c2 = f2(c), shift2 = f2(shift);
                sum[0] = sum[1] = 0;
                uint32_t s[2][CH];
                fetch(0, s[0]);
                bool fine = true;
#pragma unroll
                for (int i = 0; i < 128 / CH; ++i) {
                    uint32_t* x = s[i & 1];
                    tmem_ld_wait();
                    if (i < 128 / CH - 1) fetch(i + 1, s[(i + 1) & 1]);
                    if constexpr (A::quant) {                                    // the exponents, in the place of the scores
#pragma unroll
                        for (int e = 0; e < CH; e += 4) {
                            const float4 k = *(const float4*)(ks + CH * i + e);
                            const f32x2 u = f2_fma(f2_bits(x[e], x[e + 1]), f2(k.x, k.y), shift2), v = f2_fma(f2_bits(x[e + 2], x[e + 3]), f2(k.z, k.w), shift2);
                            x[e] = __float_as_uint(f2_lo(u)); x[e + 1] = __float_as_uint(f2_hi(u)); x[e + 2] = __float_as_uint(f2_lo(v)); x[e + 3] = __float_as_uint(f2_hi(v));
                        }
                    }
                    if (i == 128 / CH - 1) {
                        // The last scores are in registers.  If nothing asks for another round, the probabilities may take their place.
                        float top = __uint_as_float(x[0]);
#pragma unroll
                        for (int e = 0; e < CH; e += 2) top = at_max3(top, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                        const f32x2 so_far = f2_add(sum[0], sum[1]);
                        fine = search || __all_sync(0xFFFFFFFFu, f2_lo(so_far) + f2_hi(so_far) <= AT_SUM_MAX && (A::quant ? top : fmaf(top, c, shift)) <= AT_LAG);
                        if (!fine) break;
#pragma unroll
                        for (int k = 0; k < (128 - CH) / 2; k += CH / 2) at_tmem_st16(s_at + (uint32_t)k, w + k);
                    }
                    uint32_t* to = w + CH / 2 * i;
                    float4 v;
#pragma unroll
                    for (int e = 0; e < CH / 2; ++e) {
                        const f32x2 y = A::quant ? f2_bits(x[2 * e], x[2 * e + 1]) : f2_fma(f2_bits(x[2 * e], x[2 * e + 1]), c2, shift2);
                        f32x2 p = (A::poly >> (e & 7) & 1) ? at_exp2_poly(y) : f2(at_exp2(f2_lo(y)), at_exp2(f2_hi(y)));
                        sum[e & 1] = f2_add(sum[e & 1], p);
                        if (A::quant) {
                            if ((e & 1) == 0) v = *(const float4*)(vs + CH * i + 2 * e);
                            p = f2_mul(p, (e & 1) == 0 ? f2(v.x, v.y) : f2(v.z, v.w));
                        }
                        to[e] = pack_bf16x2(p);
                    }
                    if (i == 128 / CH - 1) at_tmem_st16(s_at + 48u, to);
                }
                if (fine) break;
                search = true;
            }
            if (!ok) break;
            l += (f2_lo(sum[0]) + f2_hi(sum[0])) + (f2_lo(sum[1]) + f2_hi(sum[1]));
            at_tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + 8 * place);
            used = product;
            if (A::quant && lane == 0) mbar_arrive(sc_empty + 8 * sst);
            ++n;
        }
        if (ok && used >= 0) AT_WAIT(p_done + 8 * (used % A::places), (uint32_t)(used / A::places) & 1u);
        if (!ok && lane == 0) { atomicCAS(P.pages.status, 0, OC_ERR_TIMEOUT); *abort_flag = 1; }
        tc_fence_after();
        // ---- results ----
        if (P.split == 1) {
            const bool some = lo < hi;
            const float inv = 1.0f / l;                                          // (all scores -infinity: 0 / 0)
            const int head = (int)T.head * P.group + qg;
            const long long at = exists ? attn_out_at(P, S, T.seq, qi, head) : 0;
            for (int d = 0; d < D; d += 32) {
                uint32_t o[32];
                if (n > 0) { tmem_ld32(o_at + (uint32_t)d, o); tmem_ld_wait(); }
                if (!exists || !ok) continue;
#pragma unroll
                for (int i = 0; i < 32; i += 8) {
                    if (d + i >= D) break;
                    float y[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = some ? __uint_as_float(o[i + e]) * inv : 0.0f;
                    const uint4 v = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
                    uint16_t* out = (uint16_t*)P.out + at + d + i;
                    if (P.wide_out) st_v4(out, v);
                    else {
                        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) { out[2 * e] = (uint16_t)x[e]; out[2 * e + 1] = (uint16_t)(x[e] >> 16); }
                    }
                }
            }
            // What is no number between the keys of the row: its lanes' columns side by side, one row after the other.
            const int bad_a = max(lo, s_bad[0]), bad_b = min(hi, s_bad[1]);
            __syncwarp();
            for (unsigned left = __ballot_sync(0xFFFFFFFFu, exists && ok && bad_a < bad_b); left; left &= left - 1u) {
                const int r = __ffs(left) - 1, a = __shfl_sync(0xFFFFFFFFu, bad_a, r), b = __shfl_sync(0xFFFFFFFFu, bad_b, r);
                const long long to = __shfl_sync(0xFFFFFFFFu, at, r) + 4 * lane;
                if (4 * lane >= D) continue;
                const float4 t = attn_not_finite<KT>(P, s_bad, T.seq, T.head, a, b, 4 * lane);
                const float x[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x[e] != 0.0f) {
                        uint16_t* o = (uint16_t*)P.out + to + e;
                        *o = (uint16_t)pack_bf16x2(__uint_as_float((uint32_t)*o << 16) + x[e], 0.0f);
                    }
            }
            if (P.lse && exists && ok) P.lse[(S.row0 + qi) * P.q_heads + head] = some ? m * (A::quant ? 0.69314718f : P.scale) + logf(l) : -INFINITY;
        } else {
            const int r = my_tile * AT_ROWS + my_row;
            float* part = (float*)at_smem + (long long)r * A::out_stride;
            s_stats[r][0] = m; s_stats[r][1] = l;
            // (both tiles' products have retired in this CTA: the rows overwrite queries, keys and values)
            asm volatile("bar.sync 1, %0;" :: "n"(32 * A::softmax_warps) : "memory");
            for (int d = 0; d < D; d += 32) {
                uint32_t o[32];
                if (n > 0) { tmem_ld32(o_at + (uint32_t)d, o); tmem_ld_wait(); }
#pragma unroll
                for (int i = 0; i < 32; i += 4)
                    if (d + i < D) *(float4*)(part + d + i) = n > 0 && m != -INFINITY ? make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]))
                                                                    : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
        }
    }
    if (P.split > 1) {
        cluster_sync();
        if (warp < A::softmax_warps && !*abort_flag) {
            int bad0, bad1;
            cluster_bad(s_bad, P.split, bad0, bad1);
            // Every split-th row: first the weights of its parts (a thread for each row), then the elements side by side.
            const int vecs = D / 4, mine = (NT * AT_ROWS) / P.split;
            const uint32_t stats = smem_u32(&s_stats[0][0]);
            if ((int)threadIdx.x < mine) {
                const int r = (int)threadIdx.x * P.split + (int)rank;
                const uint32_t rr = first + (uint32_t)r;
                int a = 0, b = 0;
                const int q2 = rr < rows ? (int)TP.group.div(rr) : 0;
                const bool there = rr < rows && attn_bounds(P, S, T.seq, q2, a, b);
                float top = -INFINITY, sum = 0.0f;
                for (int k = 0; k < P.split; ++k) { const float x = cluster_ld(cluster_map(stats, (uint32_t)k) + 8u * r); top = at_max3(top, x, x); }
                for (int k = 0; k < P.split; ++k) {
                    const uint32_t st = cluster_map(stats, (uint32_t)k) + 8u * r;
                    const float x = cluster_ld(st), f = x == -INFINITY ? 0.0f : at_exp2((x - top) * (A::quant ? 1.0f : P.scale_log2));
                    sum = fmaf(f, cluster_ld(st + 4), sum);
                    s_share[(int)threadIdx.x * P.split + k] = there && a < b ? f : 0.0f;
                }
                const float inv = 1.0f / sum;                                    // (all scores -infinity: 0 / 0)
                if (there && a < b) for (int k = 0; k < P.split; ++k) s_share[(int)threadIdx.x * P.split + k] *= inv;
                if (P.lse && there) P.lse[(S.row0 + q2) * P.q_heads + (int)T.head * P.group + (int)(rr - (uint32_t)q2 * TP.group.d)] = a < b ? top * (A::quant ? 0.69314718f : P.scale) + logf(sum) : -INFINITY;
                s_there[threadIdx.x] = there ? (a < b ? 2 : 1) : 0;
            }
            asm volatile("bar.sync 1, %0;" :: "n"(32 * A::softmax_warps) : "memory");
            for (int i = threadIdx.x; i < mine * vecs; i += 32 * A::softmax_warps) {
                const int rm = i / vecs, r = rm * P.split + (int)rank, d = 4 * (i % vecs);
                if (s_there[rm] == 0) continue;
                const uint32_t rr = first + (uint32_t)r;
                const int q2 = (int)TP.group.div(rr), head = (int)T.head * P.group + (int)(rr - (uint32_t)q2 * TP.group.d);
                float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (s_there[rm] == 2) {
                    const uint32_t at = smem + (uint32_t)(r * A::out_stride + d) * 4u;
                    for (int k = 0; k < P.split; k += 2) {                       // (a power of two of them; both on their way together)
                        const float4 o0 = cluster_ld4(cluster_map(at, (uint32_t)k)), o1 = cluster_ld4(cluster_map(at, (uint32_t)k + 1));
                        const float f0 = s_share[rm * P.split + k], f1 = s_share[rm * P.split + k + 1];
                        // (a part that saw nothing of the row has zeros)
                        y.x = fmaf(f0, o0.x, fmaf(f1, o1.x, y.x)); y.y = fmaf(f0, o0.y, fmaf(f1, o1.y, y.y));
                        y.z = fmaf(f0, o0.z, fmaf(f1, o1.z, y.z)); y.w = fmaf(f0, o0.w, fmaf(f1, o1.w, y.w));
                    }
                    if (bad0 < bad1) {
                        int a, b;
                        attn_bounds(P, S, T.seq, q2, a, b);
                        a = max(a, bad0); b = min(b, bad1);
                        if (a < b) attn_add4(y, attn_not_finite<KT>(P, s_bad, T.seq, T.head, a, b, d));
                    }
                }
                attn_store4<OC_DTYPE_BF16>(P, attn_out_at(P, S, T.seq, q2, head) + d, y);
            }
        }
        cluster_sync();                                                          // nobody reads a retired CTA's memory
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == A::score_warp) tmem_dealloc_cta1(tmem, 512);
#undef AT_WAIT
}

// ---- host side -------------------------------------------------------------------------------------
typedef CUresult (*AtEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static AtEncodeFn at_encode_fn() {
    static AtEncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess) fn = (AtEncodeFn)p;
        else cudaGetLastError();
    });
    return fn;
}
static bool at_encode(AtEncodeFn enc, CUtensorMap* map, const void* p, int64_t D, int64_t vectors, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)vectors}, strides[1] = {(cuuint64_t)D * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (void*)p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NT, int SUB, int KT>
static oc_status launch_tc_as(oc_ctx* ctx, AttnTcParams& TP, cudaStream_t s) {
    using A = At<NT, SUB, KT>;
    static_assert(A::smem <= 227 * 1024 - 4096, "shared memory");                // (beside the ranges and sums)
    static_assert(NT * AT_ROWS * A::out_stride * 4 <= A::rest_at, "rows that a cluster joins");
    auto* kernel = attention_tc_kernel<NT, SUB, KT>;
    static PerDeviceOnce once;                       // (the context's device is current here)
    if (!once.ensure(ctx->device, [&] {
            const bool ok = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, A::smem) == cudaSuccess &&
                            cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
            if (!ok) cudaGetLastError();
            return ok;
        })) return OC_ERR_CUDA;
    AttnParams& P = TP.a;
    const uint64_t rows = (uint64_t)P.rows_per_batch * (uint64_t)P.group;
    const uint64_t tiles = (rows + NT * AT_ROWS - 1) / (NT * AT_ROWS), problems = (uint64_t)P.n_seqs * (uint64_t)P.pages.heads;
    if (tiles * problems * ATT_SPLIT_MAX > 0x7FFFFFFFull) return OC_ERR_UNSUPPORTED;
    P.tiles = (uint32_t)tiles;
    const uint64_t key_tiles = (P.pages.seq_rows + AT_KEYS - 1) / AT_KEYS;
    int split = 1;
    while (split < ATT_SPLIT_MAX && tiles * problems * split * 2 <= (uint64_t)ctx->sm_count && (uint64_t)split * 2 <= key_tiles) split *= 2;
    P.split = split;
    LaunchScope scope(ctx, OC_K_ATTENTION, s);
    PdlLaunch l(dim3((unsigned)(tiles * problems * split)), dim3(A::threads), A::smem, s, (unsigned)split);
    cudaLaunchKernelEx(&l.cfg, kernel, (const AttnTcParams&)TP);
    return last_launch_status();
}
template <int SUB, int KT>
static oc_status launch_tc_rows(oc_ctx* ctx, AttnTcParams& TP, cudaStream_t s) {
    const uint64_t rows = (uint64_t)TP.a.rows_per_batch * (uint64_t)TP.a.group, problems = (uint64_t)TP.a.n_seqs * (uint64_t)TP.a.pages.heads;
    // one tile of rows in a CTA where pairs would leave SMs idle
    if (rows <= AT_ROWS || (rows + 2 * AT_ROWS - 1) / (2 * AT_ROWS) * problems < (uint64_t)ctx->sm_count) return launch_tc_as<1, SUB, KT>(ctx, TP, s);
    return launch_tc_as<2, SUB, KT>(ctx, TP, s);
}

oc_status launch_attention_tc(oc_ctx* ctx, const AttnParams& P, int kv_dtype, int64_t page_rows, cudaStream_t s) {
    AttnTcParams TP;
    memset(&TP, 0, sizeof(TP));
    TP.a = P;
    TP.group = FastDiv((uint32_t)P.group); TP.units = FastDiv((uint32_t)(P.pages.D / 8));
    TP.box_rows = (int)std::gcd<int64_t>(page_rows, AT_KEYS); TP.n_boxes = AT_KEYS / TP.box_rows;
    const int D = P.pages.D;
    TP.row_bytes = kv_dtype == OC_DTYPE_I4 ? D / 2 : D;
    if (kv_dtype == OC_DTYPE_BF16 && P.pages.n_tokens > 0) {
        AtEncodeFn enc = at_encode_fn();
        const int64_t vectors = (int64_t)P.pages.n_pages * P.pages.heads * page_rows;
        if (!enc || !at_encode(enc, &TP.mapK, P.k_pool, D, vectors, TP.box_rows) || !at_encode(enc, &TP.mapV, P.v_pool, D, vectors, TP.box_rows)) return OC_ERR_UNSUPPORTED;
    }
    if (D <= 64) {
        if (kv_dtype == OC_DTYPE_BF16) return launch_tc_rows<1, OC_DTYPE_BF16>(ctx, TP, s);
        if (kv_dtype == OC_DTYPE_I8) return launch_tc_rows<1, OC_DTYPE_I8>(ctx, TP, s);
        return launch_tc_rows<1, OC_DTYPE_I4>(ctx, TP, s);
    }
    if (kv_dtype == OC_DTYPE_BF16) return launch_tc_rows<2, OC_DTYPE_BF16>(ctx, TP, s);
    if (kv_dtype == OC_DTYPE_I8) return launch_tc_rows<2, OC_DTYPE_I8>(ctx, TP, s);
    return launch_tc_rows<2, OC_DTYPE_I4>(ctx, TP, s);
}

}  // namespace oc
