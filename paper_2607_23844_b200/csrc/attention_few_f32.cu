// Attention of few fp32 rows (a sequence's rows times the heads that share one of the cache are at most 4) over the paged
// cache: bound by reading the cache once, all arithmetic in fp32.
// A warp takes 32 keys at a time.  For the scores a lane is a key: it reads the key's row 16 bytes at a time (the lanes' rows are
// neighbours, so what one load leaves of a line the next ones find in L1) and multiplies with the queries in shared memory, no sum
// crosses lanes.  For the outputs a lane is a few columns, the keys' probabilities come round by shuffles, and values are read
// as they lie.  4 x 8192 keys of 16 heads of 64: 104 us (268 MB, 2.6 TB/s), in 8 bits 48; with tiles of 16 rows in shared memory, of
// which one is used, 300.  The warps of a CTA and the CTAs of a cluster split the keys and join at the end.
#include <string.h>

#include "attention_tc.cuh"

namespace oc {

static constexpr int AG_WARPS = 8, AG_STEP = 32;

template <int KT> __device__ __forceinline__ float ag_byte(uint32_t w, int i) {          // whole number i of a word: its offset form in a float's last bits
    if (KT == OC_DTYPE_I8) return __uint_as_float(__byte_perm(w ^ 0x80808080u, 0x4B000000u, 0x7440u + i)) - 8388736.0f;
    return __uint_as_float((((w ^ 0x88888888u) >> (4 * i)) & 15u) | 0x4B000000u) - 8388616.0f;
}

// ROWS: at least as many as there are; CPL: columns of a lane (32 CPL at least as many as there are)
template <int KT, int ROWS, int CPL>
__global__ void __launch_bounds__(AG_WARPS * 32)
attention_few_f32_kernel(const __grid_constant__ AttnParams P) {
    constexpr bool quant = KT != OC_DTYPE_F32;
    constexpr int E = KT == OC_DTYPE_F32 ? 4 : 8, DP = 32 * CPL;             // elements of a piece of a key's row; columns
    __shared__ __align__(16) float s_q[ROWS][DP];
    __shared__ float s_part[AG_WARPS][ROWS][DP];
    __shared__ float s_stat[AG_WARPS][ROWS][2], s_join[ROWS][2];
    __shared__ int s_lo[ROWS], s_hi[ROWS], s_bad[ATT_BAD];                         // (s_bad: keys with values that are no numbers)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = P.pages.D;
    pdl_enter();
    const uint32_t rank = P.split > 1 ? cluster_rank() : 0u;
    const uint32_t problem = blockIdx.x / (uint32_t)P.split;
    const uint32_t seq = problem / (uint32_t)P.pages.heads, head = problem - seq * (uint32_t)P.pages.heads;
    const AttnSeq S = attn_seq(P, seq);
    const int rows = S.n * P.group;
    if (rows <= 0) return;                                                   // (the whole cluster)
    if (threadIdx.x < ROWS) {
        int a = 0, b = 0;
        const bool there = (int)threadIdx.x < rows && attn_bounds(P, S, seq, (int)threadIdx.x / P.group, a, b);
        s_lo[threadIdx.x] = there ? a : -1; s_hi[threadIdx.x] = there ? max(a, b) : -1;
    }
    if (threadIdx.x == 0) attn_bad_none(s_bad);
    for (int i = threadIdx.x; i < ROWS * DP; i += AG_WARPS * 32) {
        const int r = i / DP, d = i % DP, row = r / P.group;
        s_q[r][d] = r < rows && d < D ? ((const float*)P.q)[attn_q_at(P, S, seq, row, (int)head * P.group + (r - row * P.group)) + d] : 0.0f;
    }
    __syncthreads();
    int low = 0, high = 0x7FFFFFFF, from = 0x7FFFFFFF, to = 0;               // keys [low, high) are seen by all rows, [from, to) by any
    float m[ROWS], l[ROWS], o[ROWS][CPL];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int a = s_lo[r], b = s_hi[r];
        if (a < b) { low = max(low, a); high = min(high, b); from = min(from, a); to = max(to, b); }
        m[r] = -INFINITY; l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < CPL; ++c) o[r][c] = 0.0f;
    }
    int k0 = from / AG_STEP, k1 = to > 0 ? (to + AG_STEP - 1) / AG_STEP : 0;
    if (k1 <= k0) k0 = k1 = 0;
    if (P.split > 1) {
        const int all = k1 - k0, a = (int)((long long)all * rank / P.split), b = (int)((long long)all * (rank + 1) / P.split);
        k1 = k0 + b; k0 += a;
    }
    auto find = [&](int k) -> int {                                          // this lane's key: the pool's vector; -1: no such page, nor key
        const uint32_t key = (uint32_t)k * AG_STEP + lane;
        if (k >= k1 || (int)key >= S.len) return -1;
        const uint32_t pn = P.pages.page_rows.div(key);
        const int page = kv_page(P.pages, seq, pn);
        return page < 0 ? -1 : (int)(kv_vector(P.pages, page, key - pn * P.pages.page_rows.d) + head * P.pages.page_rows.d);
    };
    int vec = find(k0 + warp);
    for (int k = k0 + warp; k < k1; k += AG_WARPS) {
        const int next = find(k + AG_WARPS), key = k * AG_STEP + lane;
        float s[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) s[r] = 0.0f;
        const float ks = quant && vec >= 0 ? __ldg(P.k_scale + vec) : 0.0f;
        float vs = quant && vec >= 0 ? __ldg(P.v_scale + vec) : 0.0f;
        if (quant && !isfinite(vs)) { vs = 0.0f; attn_bad_key(P, s_bad, key); } // (0 * NaN would reach rows that do not see it)
        // (a lane without a key works on zeros)
#pragma unroll 4
        for (int d = 0; d < D; d += E) {
            float x[E];
            if (KT == OC_DTYPE_F32) {
                const float4 v = vec >= 0 ? __ldg((const float4*)((const float*)P.k_pool + (long long)vec * D + d)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
            } else if (KT == OC_DTYPE_I8) {
                const uint2 w = vec >= 0 ? __ldg((const uint2*)((const uint8_t*)P.k_pool + (long long)vec * D + d)) : make_uint2(0u, 0u);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = ag_byte<KT>(e < 4 ? w.x : w.y, e & 3);
            } else {
                const uint32_t w = vec >= 0 ? __ldg((const uint32_t*)((const uint8_t*)P.k_pool + (((long long)vec * D + d) >> 1))) : 0u;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = ag_byte<KT>(w, e);
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const float4 q = *(const float4*)&s_q[r][d + e];
                    s[r] = fmaf(q.x, x[e], fmaf(q.y, x[e + 1], fmaf(q.z, x[e + 2], fmaf(q.w, x[e + 3], s[r]))));
                }
        }
        const bool cut = k * AG_STEP < low || (k + 1) * AG_STEP > high;
        float p[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float x = quant ? s[r] * ks : s[r];
            if (cut && (key < s_lo[r] || key >= s_hi[r])) x = -INFINITY;
            float top = x;
#pragma unroll
            for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            top = fmaxf(top, m[r]);
            const float base = top == -INFINITY ? 0.0f : top;                // (nothing seen so far: every p is 0)
            if (top > m[r]) {                                                // (the same in all lanes)
                const float corr = m[r] == -INFINITY ? 0.0f : exp2f((m[r] - base) * P.scale_log2);
                l[r] *= corr;
#pragma unroll
                for (int c = 0; c < CPL; ++c) o[r][c] *= corr;
                m[r] = top;
            }
            const float e = exp2f((x - base) * P.scale_log2);
            l[r] += e;
            p[r] = quant ? e * vs : e;
        }
        constexpr int G = 4;                                                 // keys on their way together
        for (int j0 = 0; j0 < AG_STEP; j0 += G) {
            float x[G][CPL];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int v = __shfl_sync(0xFFFFFFFFu, vec, j0 + g);
#pragma unroll
                for (int c = 0; c < CPL; ++c) x[g][c] = 0.0f;
                if (v >= 0 && lane * CPL < D) {                              // (columns CPL lane ..: D is a multiple of 8)
                    const long long at = (long long)v * D + lane * CPL;
                    if (KT == OC_DTYPE_F32) {
                        if constexpr (CPL == 4) { const float4 y = __ldg((const float4*)((const float*)P.v_pool + at)); x[g][0] = y.x; x[g][1] = y.y; x[g][2] = y.z; x[g][3] = y.w; }
                        else { const float2 y = __ldg((const float2*)((const float*)P.v_pool + at)); x[g][0] = y.x; x[g][1] = y.y; }
                    } else if (KT == OC_DTYPE_I8) {
                        uint32_t w;
                        if constexpr (CPL == 4) w = __ldg((const uint32_t*)((const uint8_t*)P.v_pool + at));
                        else w = __ldg((const uint16_t*)((const uint8_t*)P.v_pool + at));
#pragma unroll
                        for (int c = 0; c < CPL; ++c) x[g][c] = ag_byte<KT>(w, c);
                    } else {
                        uint32_t w;
                        if constexpr (CPL == 4) w = __ldg((const uint16_t*)((const uint8_t*)P.v_pool + (at >> 1)));
                        else w = __ldg((const uint8_t*)P.v_pool + (at >> 1));
#pragma unroll
                        for (int c = 0; c < CPL; ++c) x[g][c] = ag_byte<KT>(w, c);
                    }
                }
            }
            if (!quant) {                                                    // (0 times what is no number is NaN, and stays it)
                float zero[2] = {0.0f, 0.0f};
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int c = 0; c < CPL; ++c) zero[g & 1] = fmaf(x[g][c], 0.0f, zero[g & 1]);
                if (zero[0] + zero[1] != 0.0f) {
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int c = 0; c < CPL; ++c)
                            if (!isfinite(x[g][c])) { x[g][c] = 0.0f; attn_bad_key(P, s_bad, k * AG_STEP + j0 + g); }
                }
            }
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float w = __shfl_sync(0xFFFFFFFFu, p[r], j0 + g);
#pragma unroll
                    for (int c = 0; c < CPL; ++c) o[r][c] = fmaf(w, x[g][c], o[r][c]);
                }
        }
        vec = next;
    }
    // ---- the warps' results side by side, then those of the cluster's CTAs ----
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], d);
        if (lane == 0) { s_stat[warp][r][0] = m[r]; s_stat[warp][r][1] = l[r]; }
#pragma unroll
        for (int c = 0; c < CPL; ++c) s_part[warp][r][lane * CPL + c] = o[r][c];
    }
    __syncthreads();
    const int used = min(rows, ROWS);
    int bad0 = 0, bad1 = 0;
    auto finish = [&](int r, int d, float y, float top, float sum) {
        const int i = r / P.group, hq = (int)head * P.group + (r - i * P.group), a = s_lo[r], b = s_hi[r];
        if (a < 0) return;
        y = a < b ? y / sum : 0.0f;                                          // (all scores -infinity: 0 / 0)
        const int bad_a = max(a, bad0), bad_b = min(b, bad1);
        if (bad_a < bad_b) {
            const float4 t = attn_not_finite<KT>(P, s_bad, seq, head, bad_a, bad_b, d & ~3);
            y += (d & 3) == 0 ? t.x : (d & 3) == 1 ? t.y : (d & 3) == 2 ? t.z : t.w;
        }
        ((float*)P.out)[attn_out_at(P, S, seq, i, hq) + d] = y;
        if (P.lse && d == 0) P.lse[(S.row0 + i) * P.q_heads + hq] = a < b ? top * P.scale + logf(sum) : -INFINITY;
    };
    if (P.split == 1) { bad0 = s_bad[0]; bad1 = s_bad[1]; }
    for (int it = threadIdx.x; it < used * D; it += AG_WARPS * 32) {
        const int r = it / D, d = it - r * D;
        float top = -INFINITY, sum = 0.0f, y = 0.0f;
        for (int w = 0; w < AG_WARPS; ++w) top = fmaxf(top, s_stat[w][r][0]);
        for (int w = 0; w < AG_WARPS; ++w) {
            const float mw = s_stat[w][r][0], f = mw == -INFINITY ? 0.0f : exp2f((mw - top) * P.scale_log2);
            sum = fmaf(f, s_stat[w][r][1], sum);
            if (mw != -INFINITY) y = fmaf(f, s_part[w][r][d], y);
        }
        if (P.split == 1) { finish(r, d, y, top, sum); continue; }
        s_part[0][r][d] = y;                                                 // (read by this thread alone)
        if (d == 0) { s_join[r][0] = top; s_join[r][1] = sum; }
    }
    if (P.split == 1) return;
    cluster_sync();
    cluster_bad(s_bad, P.split, bad0, bad1);
    const uint32_t part_at = smem_u32(&s_part[0][0][0]), join_at = smem_u32(&s_join[0][0]);
    for (int it = (int)rank * AG_WARPS * 32 + threadIdx.x; it < used * D; it += P.split * AG_WARPS * 32) {
        const int r = it / D, d = it - r * D;
        float top = -INFINITY, sum = 0.0f, y = 0.0f;
        for (int w = 0; w < P.split; ++w) top = fmaxf(top, cluster_ld(cluster_map(join_at, (uint32_t)w) + 8u * r));
        for (int w = 0; w < P.split; ++w) {
            const uint32_t st = cluster_map(join_at, (uint32_t)w) + 8u * r;
            // (a part whose scores are all NaN has no maximum either, but its sum is NaN: it counts)
            const float mw = cluster_ld(st), f = mw == -INFINITY ? 0.0f : exp2f((mw - top) * P.scale_log2);
            sum = fmaf(f, cluster_ld(st + 4u), sum);
            if (mw != -INFINITY) y = fmaf(f, cluster_ld(cluster_map(part_at, (uint32_t)w) + (uint32_t)(r * DP + d) * 4u), y);
        }
        finish(r, d, y, top, sum);
    }
    cluster_sync();                                                          // nobody reads a retired CTA's memory
}

// ---- host side -------------------------------------------------------------------------------------
template <int KT, int ROWS, int CPL>
static oc_status launch_few_f32_as(oc_ctx* ctx, AttnParams& P, cudaStream_t s) {
    auto* kernel = attention_few_f32_kernel<KT, ROWS, CPL>;
    static PerDeviceOnce once;                       // (the context's device is current here)
    if (!once.ensure(ctx->device, [&] {
            const bool ok = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
            if (!ok) cudaGetLastError();
            return ok;
        })) return OC_ERR_CUDA;
    const uint64_t problems = (uint64_t)P.n_seqs * (uint64_t)P.pages.heads;
    if (problems * ATT_SPLIT_MAX > 0x7FFFFFFFull) return OC_ERR_UNSUPPORTED;
    // CTAs enough for the device several times over, each with a step for every warp at least
    int split = 1;
    while (split < ATT_SPLIT_MAX && problems * split < 4ull * ctx->sm_count && (uint64_t)P.pages.seq_rows >= (uint64_t)split * 2 * AG_WARPS * AG_STEP) split *= 2;
    P.split = split;
    LaunchScope scope(ctx, OC_K_ATTENTION, s);
    PdlLaunch l(dim3((unsigned)(problems * split)), dim3(AG_WARPS * 32), 0, s, (unsigned)split);
    cudaLaunchKernelEx(&l.cfg, kernel, (const AttnParams&)P);
    return last_launch_status();
}
template <int KT>
static oc_status launch_few_f32(oc_ctx* ctx, AttnParams& P, cudaStream_t s) {
    const bool one = (uint64_t)P.rows_per_batch * (uint64_t)P.group <= 1;
    if (P.pages.D <= 64) return one ? launch_few_f32_as<KT, 1, 2>(ctx, P, s) : launch_few_f32_as<KT, 4, 2>(ctx, P, s);
    return one ? launch_few_f32_as<KT, 1, 4>(ctx, P, s) : launch_few_f32_as<KT, 4, 4>(ctx, P, s);
}

bool attention_few_rows_f32(const AttnParams& P) { return (uint64_t)P.rows_per_batch * (uint64_t)P.group <= 4; }

oc_status launch_attention_few_f32(oc_ctx* ctx, AttnParams& P, int kv_dtype, cudaStream_t s) {
    if (kv_dtype == OC_DTYPE_F32) return launch_few_f32<OC_DTYPE_F32>(ctx, P, s);
    return kv_dtype == OC_DTYPE_I8 ? launch_few_f32<OC_DTYPE_I8>(ctx, P, s) : launch_few_f32<OC_DTYPE_I4>(ctx, P, s);
}

}  // namespace oc
