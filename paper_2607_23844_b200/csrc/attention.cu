// Attention over the paged cache for fp32 queries, on the fp32 pipelines, and the choice of kernel.
//     out[r] = sum_j p_j V[j] / sum_j p_j,   p_j = exp(scale * q[r] . K[j] - m),   m the row's running maximum
// One CTA takes a tile of TR rows (the heads that share a head of the cache are rows of their own) and walks over the keys 64 at
// a time; the maximum, the sum and the output of a row are carried along and rescaled when the maximum grows.
// Thread (ty, tx) of 16 x 16 holds the scores of TR / 16 rows with 4 keys, and of the output TR / 16 rows with 4 or 8
// elements.  Where there are few tiles, the CTAs of a cluster split the keys and join their results through
// distributed shared memory.
// Bound by shared memory's reads beside the FMAs: 2 x 1024 x 1024, 16 heads of 64 or 128: 338 and 711 us, 25 and 24 TFLOP/s.  Tiles are
// fetched into registers a step ahead.
#include <string.h>

#include <algorithm>

#include "attention_tc.cuh"

namespace oc {

static constexpr int AS_KEYS = 64, AS_THREADS = 256;

template <int TR, int DP> struct AsSmem {
    static constexpr int QS = DP + 4, KS = DP + 4, PS = AS_KEYS + 4;         // floats between rows (4: rows fall on other banks)
    static constexpr int q = 0, kv = TR * QS, p = kv + AS_KEYS * KS, floats = p + TR * PS;
    static constexpr int bytes = floats * 4;
};

// 8 elements of the cache at unit u of vector v, as floats
template <int KT> __device__ __forceinline__ void as_load(const void* pool, const float* scales, uint32_t v, int D, int u, f32x2* f) {
    const long long at = (long long)v * D + 8 * u;
    if (KT == OC_DTYPE_F32) {
        RowVec<OC_DTYPE_F32>::unpack(ld_nc_v4((const float*)pool + at), f);
        RowVec<OC_DTYPE_F32>::unpack(ld_nc_v4((const float*)pool + at + 4), f + 2);
    } else {
        const float s = __ldg(scales + v);
        uint2 w;
        if (KT == OC_DTYPE_I8) w = __ldg((const uint2*)((const uint8_t*)pool + at));
        else w.x = __ldg((const uint32_t*)((const uint8_t*)pool + (at >> 1)));
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = s * (float)(KT == OC_DTYPE_I8 ? (int)((i < 4 ? w.x : w.y) << (24 - 8 * (i & 3))) >> 24 : (int)(w.x << (28 - 4 * i)) >> 28);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = f2(x[2 * i], x[2 * i + 1]);
    }
}

template <int TR, int DP, int KT>
__global__ void __launch_bounds__(AS_THREADS)
attention_simt_kernel(const __grid_constant__ AttnParams P) {
    using M = AsSmem<TR, DP>;
    constexpr int R = TR / 16, C = DP / 64;                                  // rows of a thread; vectors of 4 outputs
    extern __shared__ __align__(16) float as_smem[];
    __shared__ int range[2];                                                 // first and last key that the tile sees
    __shared__ int bounds[TR][2];                                            // of each row; lo = -1: the row is left as it is
    __shared__ float stats[TR][2];
    __shared__ int bad[ATT_BAD];                                                   // keys with values that are no numbers
    float *sq = as_smem + M::q, *skv = as_smem + M::kv, *sp = as_smem + M::p;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, D = P.pages.D;
    pdl_enter();
    const uint32_t rank = P.split > 1 ? cluster_rank() : 0u;
    const AttnTile T = attn_tile(P, blockIdx.x / (uint32_t)P.split);
    const AttnSeq S = attn_seq(P, T.seq);
    const long long first = (long long)T.tile * TR, rows = (long long)S.n * P.group;
    if (first >= rows) return;                                               // (the whole cluster)
    if (tid == 0) { range[0] = 0x7FFFFFFF; range[1] = 0; attn_bad_none(bad); }
    __syncthreads();
    if (tid < TR) {
        int lo = -1, hi = -1;
        if (first + tid < rows && attn_bounds(P, S, T.seq, (int)((first + tid) / P.group), lo, hi)) {
            if (lo < hi) { atomicMin(&range[0], lo); atomicMax(&range[1], hi); }
        } else {
            lo = hi = -1;
        }
        bounds[tid][0] = lo; bounds[tid][1] = hi;
    }
#pragma unroll
    for (int it = 0; it < (TR * (DP / 8) + AS_THREADS - 1) / AS_THREADS; ++it) {
        const int i = tid + it * AS_THREADS, r = i / (DP / 8), u = i % (DP / 8);
        if (r >= TR) break;
        f32x2 f[4] = {};
        if (first + r < rows && 8 * u < D) {
            const int row = (int)((first + r) / P.group), g = (int)((first + r) % P.group);
            const float* q = (const float*)P.q + attn_q_at(P, S, T.seq, row, (int)T.head * P.group + g) + 8 * u;
            if (P.wide_q) { RowVec<OC_DTYPE_F32>::unpack(*(const uint4*)q, f); RowVec<OC_DTYPE_F32>::unpack(*(const uint4*)(q + 4), f + 2); }
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = f2(q[2 * e], q[2 * e + 1]);
        }
        store_row_smem<8>(sq + r * M::QS + 8 * u, f);
    }
    __syncthreads();
    // this CTA's share of the tiles of keys
    int k0 = range[0] / AS_KEYS, k1 = range[1] > 0 ? (range[1] + AS_KEYS - 1) / AS_KEYS : 0;
    if (k1 <= k0) k0 = k1 = 0;
    if (P.split > 1) {
        const int n = k1 - k0, a = (int)((long long)n * rank / P.split), b = (int)((long long)n * (rank + 1) / P.split);
        k1 = k0 + b; k0 += a;
    }
    float m[R], l[R], o[R][C][4];
    int lo[R], hi[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = -INFINITY; l[r] = 0.0f;
        lo[r] = bounds[ty * R + r][0]; hi[r] = bounds[ty * R + r][1];
#pragma unroll
        for (int c = 0; c < C; ++c) o[r][c][0] = o[r][c][1] = o[r][c][2] = o[r][c][3] = 0.0f;
    }
    // A tile of keys or values on its way in registers: fetched while the one before is worked on.
    constexpr int ITEMS = AS_KEYS * (DP / 8) / AS_THREADS;
    f32x2 ahead[ITEMS][4];
    auto fetch = [&](const void* pool, const float* scales, int key0) {
        int vec[ITEMS];
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) {
            const int i = tid + it * AS_THREADS, j = i / (DP / 8), u = i % (DP / 8), key = key0 + j;
            vec[it] = -1;
            if (key < S.len && 8 * u < D) {
                const uint32_t pn = P.pages.page_rows.div((uint32_t)key);
                const int page = kv_page(P.pages, T.seq, pn);
                if (page >= 0) vec[it] = (int)(kv_vector(P.pages, page, (uint32_t)key - pn * P.pages.page_rows.d) + T.head * P.pages.page_rows.d);
            }
        }
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) {
            ahead[it][0] = ahead[it][1] = ahead[it][2] = ahead[it][3] = 0;
            if (vec[it] >= 0) as_load<KT>(pool, scales, (uint32_t)vec[it], D, (tid + it * AS_THREADS) % (DP / 8), ahead[it]);
        }
    };
    auto put = [&](bool value, int key0) {
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) {
            const int i = tid + it * AS_THREADS, j = i / (DP / 8), u = i % (DP / 8);
            f32x2* f = ahead[it];
            if (value && max_bits<8>(f, 0u) >= 0x7F800000u) {
                attn_bad_key(P, bad, key0 + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = f2_lo(f[e]), b = f2_hi(f[e]);
                    f[e] = f2(isfinite(a) ? a : 0.0f, isfinite(b) ? b : 0.0f);
                }
            }
            store_row_smem<8>(skv + j * M::KS + 8 * u, f);
        }
    };
    if (k0 < k1) fetch(P.k_pool, P.k_scale, k0 * AS_KEYS);
    for (int kt = k0; kt < k1; ++kt) {
        const int key0 = kt * AS_KEYS;
        __syncthreads();                                                     // (the last tile's values have been read)
        put(false, key0);
        fetch(P.v_pool, P.v_scale, key0);
        __syncthreads();
        float s[R][4] = {};
        for (int d = 0; d < D; d += 4) {
            float4 a[R], b[4];
#pragma unroll
            for (int r = 0; r < R; ++r) a[r] = *(const float4*)(sq + (ty * R + r) * M::QS + d);
#pragma unroll
            for (int c = 0; c < 4; ++c) b[c] = *(const float4*)(skv + (tx + 16 * c) * M::KS + d);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    s[r][c] = fmaf(a[r].x, b[c].x, fmaf(a[r].y, b[c].y, fmaf(a[r].z, b[c].z, fmaf(a[r].w, b[c].w, s[r][c]))));
        }
        __syncthreads();                                                     // (the keys have been read)
        put(true, key0);
        if (kt + 1 < k1) fetch(P.k_pool, P.k_scale, key0 + AS_KEYS);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float most = m[r];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int key = key0 + tx + 16 * c;
                if (key < lo[r] || key >= hi[r]) s[r][c] = -INFINITY;
                most = fmaxf(most, s[r][c]);
            }
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            const float base = most == -INFINITY ? 0.0f : most;              // (nothing seen so far: every p is 0)
            const float corr = m[r] == -INFINITY ? 0.0f : exp2f((m[r] - base) * P.scale_log2);
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float p = exp2f((s[r][c] - base) * P.scale_log2);
                sum += p;
                sp[(ty * R + r) * M::PS + tx + 16 * c] = p;
            }
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            l[r] = l[r] * corr + sum;
            m[r] = most;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][c][e] *= corr;
        }
        __syncthreads();
        for (int j = 0; j < AS_KEYS; j += 4) {
            float4 p[R];
#pragma unroll
            for (int r = 0; r < R; ++r) p[r] = *(const float4*)(sp + (ty * R + r) * M::PS + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const float4 v = *(const float4*)(skv + (j + e) * M::KS + 64 * c + 4 * tx);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float w = e == 0 ? p[r].x : e == 1 ? p[r].y : e == 2 ? p[r].z : p[r].w;
                        o[r][c][0] = fmaf(w, v.x, o[r][c][0]); o[r][c][1] = fmaf(w, v.y, o[r][c][1]);
                        o[r][c][2] = fmaf(w, v.z, o[r][c][2]); o[r][c][3] = fmaf(w, v.w, o[r][c][3]);
                    }
                }
            }
        }
    }
    int bad0 = 0, bad1 = 0;
    auto finish = [&](int r, int c, const float* x, float sum, float most) {  // r: row of the tile; columns 64 c + 4 tx ..
        const int row = (int)((first + r) / P.group), head = (int)T.head * P.group + (int)((first + r) % P.group);
        const int a = bounds[r][0], b = bounds[r][1];
        const float inv = a < b ? 1.0f / sum : 0.0f;                         // (all scores -infinity: 0 / 0)
        float4 y = a < b ? make_float4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const int d = 64 * c + 4 * tx;
        if (d < D) {
            const int bad_a = max(a, bad0), bad_b = min(b, bad1);
            if (bad_a < bad_b) attn_add4(y, attn_not_finite<KT>(P, bad, T.seq, T.head, bad_a, bad_b, d));
            attn_store4<OC_DTYPE_F32>(P, attn_out_at(P, S, T.seq, row, head) + d, y);
        }
        if (P.lse && d == 0) P.lse[(S.row0 + row) * P.q_heads + head] = a < b ? most * P.scale + logf(sum) : -INFINITY;
    };
    if (P.split == 1) {
        __syncthreads();                                                     // (`bad` is final)
        bad0 = bad[0]; bad1 = bad[1];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (lo[r] >= 0)
#pragma unroll
                for (int c = 0; c < C; ++c) finish(ty * R + r, c, o[r][c], l[r], m[r]);
        return;
    }
    // The cluster's CTAs put their sums side by side, and each joins every split-th row.
    __syncthreads();
    float* part = as_smem;                                                   // [TR][DP]
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (tx == 0) { stats[ty * R + r][0] = m[r]; stats[ty * R + r][1] = l[r]; }
#pragma unroll
        for (int c = 0; c < C; ++c) *(float4*)(part + (ty * R + r) * DP + 64 * c + 4 * tx) = make_float4(o[r][c][0], o[r][c][1], o[r][c][2], o[r][c][3]);
    }
    cluster_sync();
    cluster_bad(bad, P.split, bad0, bad1);                                   // (they may be another CTA's)
    const uint32_t part_at = smem_u32(part), stats_at = smem_u32(&stats[0][0]);
    for (int r = ty * P.split + (int)rank; r < TR; r += 16 * P.split) {
        if (bounds[r][0] < 0) continue;
        float most = -INFINITY, sum = 0.0f;
        for (int k = 0; k < P.split; ++k) most = fmaxf(most, cluster_ld(cluster_map(stats_at, (uint32_t)k) + r * 8));
        const float base = most == -INFINITY ? 0.0f : most;
        float x[C][4] = {};
        for (int k = 0; k < P.split; ++k) {
            const uint32_t st = cluster_map(stats_at, (uint32_t)k) + r * 8;
            const float w = exp2f((cluster_ld(st) - base) * P.scale_log2);
            sum = fmaf(w, cluster_ld(st + 4), sum);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const float4 v = cluster_ld4(cluster_map(part_at, (uint32_t)k) + (uint32_t)(r * DP + 64 * c + 4 * tx) * 4);
                x[c][0] = fmaf(w, v.x, x[c][0]); x[c][1] = fmaf(w, v.y, x[c][1]); x[c][2] = fmaf(w, v.z, x[c][2]); x[c][3] = fmaf(w, v.w, x[c][3]);
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) finish(r, c, x[c], sum, most);
    }
    cluster_sync();                                                          // nobody reads a retired CTA's memory
}

// ---- host side -------------------------------------------------------------------------------------
template <int TR, int DP, int KT>
static oc_status launch_simt_as(oc_ctx* ctx, AttnParams& P, cudaStream_t s) {
    using M = AsSmem<TR, DP>;
    auto* kernel = attention_simt_kernel<TR, DP, KT>;
    static PerDeviceOnce once;                       // (the context's device is current here)
    if (!once.ensure(ctx->device, [&] {
            const bool ok = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, M::bytes) == cudaSuccess &&
                            cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
            if (!ok) cudaGetLastError();
            return ok;
        })) return OC_ERR_CUDA;
    const uint64_t rows = (uint64_t)P.rows_per_batch * (uint64_t)P.group;
    const uint64_t tiles = (rows + TR - 1) / TR, problems = (uint64_t)P.n_seqs * (uint64_t)P.pages.heads;
    if (tiles * problems * ATT_SPLIT_MAX > 0x7FFFFFFFull) return OC_ERR_UNSUPPORTED;
    P.tiles = (uint32_t)tiles;
    const uint64_t key_tiles = (P.pages.seq_rows + AS_KEYS - 1) / AS_KEYS;
    int split = 1;
    while (split < ATT_SPLIT_MAX && tiles * problems * split * 2 <= 2ull * ctx->sm_count && (uint64_t)split * 2 <= key_tiles) split *= 2;
    P.split = split;
    LaunchScope scope(ctx, OC_K_ATTENTION, s);
    PdlLaunch l(dim3((unsigned)(tiles * problems * split)), dim3(AS_THREADS), M::bytes, s, (unsigned)split);
    cudaLaunchKernelEx(&l.cfg, kernel, (const AttnParams&)P);
    return last_launch_status();
}
template <int KT>
static oc_status launch_simt(oc_ctx* ctx, AttnParams& P, cudaStream_t s) {
    // tiles of 16 rows where there are no more of them, or where those of 64 would leave most SMs idle
    const uint64_t rows = (uint64_t)P.rows_per_batch * (uint64_t)P.group, key_tiles = (P.pages.seq_rows + AS_KEYS - 1) / AS_KEYS;
    const bool few = rows <= 16 || (rows + 63) / 64 * P.n_seqs * P.pages.heads * std::min<uint64_t>(key_tiles, ATT_SPLIT_MAX) < (uint64_t)ctx->sm_count / 2;
    if (P.pages.D <= 64) return few ? launch_simt_as<16, 64, KT>(ctx, P, s) : launch_simt_as<64, 64, KT>(ctx, P, s);
    return few ? launch_simt_as<16, 128, KT>(ctx, P, s) : launch_simt_as<64, 128, KT>(ctx, P, s);
}

oc_status launch_attention(oc_ctx* ctx, const oc_kv_desc& cache, const oc_attention_desc& d, const int32_t* page_table, const int32_t* kv_len,
                           const int32_t* q_start, const int32_t* idx, const void* q, const void* k_pool, const float* k_scale,
                           const void* v_pool, const float* v_scale, void* out, float* lse, cudaStream_t s) {
    AttnParams P;
    memset(&P, 0, sizeof(P));
    P.pages = kv_pages(cache, page_table, ctx->d_status);
    P.kv_len = kv_len; P.q_start = q_start; P.idx = idx; P.q = q; P.k_pool = k_pool; P.v_pool = v_pool; P.k_scale = k_scale; P.v_scale = v_scale;
    P.out = out; P.lse = lse;
    P.q_batch = d.q.batch_stride; P.q_row = d.q.row_stride; P.q_head = d.q.head_stride;
    P.o_batch = d.out.batch_stride; P.o_row = d.out.row_stride; P.o_head = d.out.head_stride;
    P.n_rows = (uint32_t)d.n_rows; P.rows_per_batch = (uint32_t)std::min(d.rows_per_batch, d.n_rows); P.n_seqs = (uint32_t)cache.n_seqs;
    P.q_heads = d.q_heads; P.group = d.q_heads / cache.heads;
    // (a unit, or a number of units, beyond every position means the same as the largest position)
    P.unit = std::min<int64_t>(d.unit, 0x7FFFFFFF); P.back = std::min<int64_t>(d.back, 0x7FFFFFFF); P.ahead = std::min<int64_t>(d.ahead, 0x7FFFFFFF);
    P.scale = d.scale; P.scale_log2 = d.scale * 1.44269504f;
    P.long_first = q_start || d.unit > 0;
    P.part_shift = 7;
    while ((P.pages.seq_rows - 1) >> P.part_shift >= 128) ++P.part_shift;
    const uint64_t eb = d.dtype == OC_DTYPE_F32 ? 4 : 2;
    P.wide_q = ((uintptr_t)q | ((q_start ? 0u : (uint64_t)P.q_batch) | (uint64_t)P.q_row | (uint64_t)P.q_head) * eb) % 16 == 0;
    P.wide_out = ((uintptr_t)out | ((q_start ? 0u : (uint64_t)P.o_batch) | (uint64_t)P.o_row | (uint64_t)P.o_head) * eb) % 16 == 0;
    if (d.dtype == OC_DTYPE_F32) {
        if (attention_few_rows_f32(P)) return launch_attention_few_f32(ctx, P, cache.dtype, s);
        if (cache.dtype == OC_DTYPE_F32) return launch_simt<OC_DTYPE_F32>(ctx, P, s);
        if (cache.dtype == OC_DTYPE_I8) return launch_simt<OC_DTYPE_I8>(ctx, P, s);
        return launch_simt<OC_DTYPE_I4>(ctx, P, s);
    }
    if (attention_few_rows(P)) return launch_attention_few(ctx, P, cache.dtype, s);
    return launch_attention_tc(ctx, P, cache.dtype, cache.page_rows, s);
}

}  // namespace oc
