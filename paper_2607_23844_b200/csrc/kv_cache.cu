// Rows of keys and values into the pages of a cache, and back:
//     floating point  a copy
//     whole numbers   scale = max|x| / L,  q = rint(x * L / max|x|),  value = q * scale       (L = 127 in 8 bits, 7 in 4)
// Both directions are bound by the bytes that they move.  A thread owns one unit of 8 elements of one token and walks over
// the heads, HEADS of them at a time so that as many 16-byte loads are in flight; lph lanes make up a head, and the
// tokens of 32 / lph neighbouring rows share a warp: kept lists ascend, so their vectors of a head are mostly
// neighbours in a page too.
// Measured on 230400 tokens with 5 heads of 64 (keys and values), put | get: bf16 590 MB 92 | 96 us (6.4 TB/s), fp32 1180 MB 176 | 179 (6.7);
// bf16 to 8 bits 451 MB 173 | 87, to 4 bits 166 | 84; fp32 to 8 bits 174 | 140.  Putting whole numbers is bound by their 247
// instructions for 8 elements (the largest magnitude, the quotients, their exact rounding).
#include <string.h>

#include "kv_cache.cuh"

namespace oc {

static constexpr int KV_WARPS = 4, KV_HEADS = 4;

struct KvMoveParams {
    KvPages pages;
    const int32_t* idx;
    void* dense[2]; void* pool[2]; float* scale[2];      // k, v
    long long batch_stride[2], row_stride[2], head_stride[2];
    FastDiv rows_per_batch;
    uint32_t n_rows;
    int lph, rpw, head_blocks, block_heads;              // lanes of a head; rows of a warp; blocks of up to KV_HEADS heads
    bool wide[2];                                        // dense rows may be read and written 16 bytes at a time
};

// 8 elements of a dense row
template <int DT> __device__ __forceinline__ void kv_load(const void* p, bool wide, f32x2* f, uint4* raw) {
    if constexpr (DT == OC_DTYPE_BF16) {
        if (wide) raw[0] = ld_v4(p);
        else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)((const uint16_t*)p)[2 * i] | (uint32_t)((const uint16_t*)p)[2 * i + 1] << 16;
            raw[0] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
        if (wide) { raw[0] = ld_v4(p); raw[1] = ld_v4((const uint8_t*)p + 16); }
        else {
            const uint32_t* w = (const uint32_t*)p;
            raw[0] = make_uint4(w[0], w[1], w[2], w[3]); raw[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
        if (f) RowVec<DT>::unpack(raw[1], f + 2);
    }
    if (f) RowVec<DT>::unpack(raw[0], f);
}
template <int DT> __device__ __forceinline__ void kv_store(void* p, bool wide, const uint4* raw) {
    if (wide) {
        st_v4(p, raw[0]);
        if (DT == OC_DTYPE_F32) st_v4((uint8_t*)p + 16, raw[1]);
        return;
    }
#pragma unroll
    for (int j = 0; j < (DT == OC_DTYPE_F32 ? 2 : 1); ++j) {
        const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (DT == OC_DTYPE_F32) ((uint32_t*)p)[4 * j + i] = w[i];
            else { ((uint16_t*)p)[2 * i] = (uint16_t)w[i]; ((uint16_t*)p)[2 * i + 1] = (uint16_t)(w[i] >> 16); }
        }
    }
}

// DT: type of the rows; KT: of the cache
template <bool PUT, int DT, int KT>
__global__ void __launch_bounds__(KV_WARPS * 32)
kv_move_kernel(const __grid_constant__ KvMoveParams P) {
    constexpr int EB = DT == OC_DTYPE_F32 ? 4 : 2;
    constexpr bool Q = KT == OC_DTYPE_I8 || KT == OC_DTYPE_I4;
    constexpr int L = KT == OC_DTYPE_I4 ? 7 : 127;
    constexpr int UB = KT == OC_DTYPE_F32 ? 32 : KT == OC_DTYPE_BF16 ? 16 : KT == OC_DTYPE_I8 ? 8 : 4;       // bytes of a unit
    const int lane = threadIdx.x & 31, sub = lane / P.lph, u = lane - sub * P.lph;
    const int m = blockIdx.y >= (unsigned)P.head_blocks, h0 = ((int)blockIdx.y - m * P.head_blocks) * P.block_heads;
    const int heads = min(P.block_heads, P.pages.heads - h0);
    pdl_enter();
    const uint32_t r = (blockIdx.x * KV_WARPS + (threadIdx.x >> 5)) * (uint32_t)P.rpw + sub;
    bool in = sub < P.rpw && r < P.n_rows;                                    // (rows past the end run along for the shuffles)
    uint32_t t = r;
    if (P.idx && in) {
        const int i = __ldg(P.idx + r);
        in = i >= 0;                                                         // the unused tail of a kept list
        t = (uint32_t)i;
        if (in && t >= P.pages.n_tokens) { atomicCAS(P.pages.status, 0, OC_ERR_INVALID_ARG); in = false; }
    }
    int page = -1;
    uint32_t vec = 0;
    if (in) {
        const uint32_t seq = t / P.pages.seq_rows, p = t - seq * P.pages.seq_rows, pn = P.pages.page_rows.div(p);
        page = kv_page(P.pages, seq, pn);
        vec = page < 0 ? 0u : kv_vector(P.pages, page, p - pn * P.pages.page_rows.d);
        if (PUT && page < 0) in = false;
    }
    const uint32_t b = in ? P.rows_per_batch.div(r) : 0u;
    uint8_t* dense = (uint8_t*)P.dense[m] + ((long long)b * P.batch_stride[m] + (long long)(in ? r - b * P.rows_per_batch.d : 0u) * P.row_stride[m] + 8 * u) * EB;
    const long long head_bytes = P.head_stride[m] * EB;
    const bool wide = P.wide[m];
    uint8_t* pool = (uint8_t*)P.pool[m];
    float* scales = P.scale[m];
    if (PUT) {
        int from[5];                                                         // lanes of the same head 1, 2, 4 .. further
#pragma unroll
        for (int i = 0; i < 5; ++i) { const int o = u + (1 << i); from[i] = sub * P.lph + (o >= P.lph ? o - P.lph : o); }
        f32x2 f[KV_HEADS][4];
        uint4 raw[KV_HEADS][2];
#pragma unroll
        for (int k = 0; k < KV_HEADS; ++k) {
            raw[k][0] = raw[k][1] = make_uint4(0, 0, 0, 0);
            if (Q) { f[k][0] = f[k][1] = f[k][2] = f[k][3] = 0; }
            if (in && k < heads) kv_load<DT>(dense + (h0 + k) * head_bytes, wide, Q ? f[k] : nullptr, raw[k]);
        }
#pragma unroll
        for (int k = 0; k < KV_HEADS; ++k) {
            if (k >= heads) break;
            const uint32_t v = vec + (uint32_t)(h0 + k) * P.pages.page_rows.d;
            uint8_t* to = pool + ((long long)v * (P.pages.D >> 3) + u) * UB;
            if (!Q) {
                if (in) { st_v4(to, raw[k][0]); if (KT == OC_DTYPE_F32) st_v4(to + 16, raw[k][1]); }
                continue;
            }
            uint32_t most = max_bits<8>(f[k], 0u);
            // (the largest of a head's lanes, however many: going around them twice as far each time)
#pragma unroll
            for (int i = 0; i < 5; ++i)
                if ((1 << i) < P.lph) most = max(most, __shfl_sync(0xFFFFFFFFu, most, from[i]));
            const KvQuant q = kv_quant<L>(most);
            if (!in) continue;
            uint32_t n[8];
            kv_levels<L, DT>(f[k], q, n);
            if (KT == OC_DTYPE_I8) {
                uint32_t w[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) w[i] = __byte_perm(__byte_perm(n[4 * i], n[4 * i + 1], 0x0040u), __byte_perm(n[4 * i + 2], n[4 * i + 3], 0x0040u), 0x5410u);
                *(uint2*)to = make_uint2(w[0], w[1]);
            } else {
                uint32_t w = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) w |= (n[i] & 15u) << (4 * i);
                *(uint32_t*)to = w;
            }
            if (u == 0) scales[v] = q.scale;
        }
    } else {
        uint4 raw[KV_HEADS][2];
        float sc[KV_HEADS];
#pragma unroll
        for (int k = 0; k < KV_HEADS; ++k) {
            raw[k][0] = raw[k][1] = make_uint4(0, 0, 0, 0);
            sc[k] = 0.0f;
            if (!in || page < 0 || k >= heads) continue;
            const uint32_t v = vec + (uint32_t)(h0 + k) * P.pages.page_rows.d;
            const uint8_t* from = pool + ((long long)v * (P.pages.D >> 3) + u) * UB;
            if (KT == OC_DTYPE_F32) { raw[k][0] = ld_v4(from); raw[k][1] = ld_v4(from + 16); }
            else if (KT == OC_DTYPE_BF16) raw[k][0] = ld_v4(from);
            else if (KT == OC_DTYPE_I8) { const uint2 w = *(const uint2*)from; raw[k][0].x = w.x; raw[k][0].y = w.y; }
            else raw[k][0].x = *(const uint32_t*)from;
            if (Q) sc[k] = scales[v];
        }
        if (!in) return;
#pragma unroll
        for (int k = 0; k < KV_HEADS; ++k) {
            if (k >= heads) break;
            if (Q) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int n = KT == OC_DTYPE_I8 ? (int)((i < 4 ? raw[k][0].x : raw[k][0].y) << (24 - 8 * (i & 3))) >> 24
                                                    : (int)(raw[k][0].x << (28 - 4 * i)) >> 28;
                    x[i] = (float)n * sc[k];
                }
                if (DT == OC_DTYPE_BF16) {
                    raw[k][0] = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
                } else {
                    raw[k][0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
                    raw[k][1] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
                }
            }
            kv_store<DT>(dense + (h0 + k) * head_bytes, wide, raw[k]);
        }
    }
}

template <bool PUT>
static void launch_kv_as(const KvMoveParams& P, int dt, int kt, dim3 grid, cudaStream_t s) {
    constexpr int T = KV_WARPS * 32;
    if (dt == OC_DTYPE_F32) {
        if (kt == OC_DTYPE_F32) OC_LAUNCH((kv_move_kernel<PUT, OC_DTYPE_F32, OC_DTYPE_F32>), grid, T, 0, s, P);
        else if (kt == OC_DTYPE_I8) OC_LAUNCH((kv_move_kernel<PUT, OC_DTYPE_F32, OC_DTYPE_I8>), grid, T, 0, s, P);
        else OC_LAUNCH((kv_move_kernel<PUT, OC_DTYPE_F32, OC_DTYPE_I4>), grid, T, 0, s, P);
    } else {
        if (kt == OC_DTYPE_BF16) OC_LAUNCH((kv_move_kernel<PUT, OC_DTYPE_BF16, OC_DTYPE_BF16>), grid, T, 0, s, P);
        else if (kt == OC_DTYPE_I8) OC_LAUNCH((kv_move_kernel<PUT, OC_DTYPE_BF16, OC_DTYPE_I8>), grid, T, 0, s, P);
        else OC_LAUNCH((kv_move_kernel<PUT, OC_DTYPE_BF16, OC_DTYPE_I4>), grid, T, 0, s, P);
    }
}

oc_status launch_kv_move(oc_ctx* ctx, bool put, const oc_kv_desc& cache, const oc_kv_rows& rows, const int32_t* page_table, const int32_t* idx,
                         const void* k, const void* k_pool, const float* k_scale, const void* v, const void* v_pool,
                         const float* v_scale, cudaStream_t s) {
    KvMoveParams P;
    P.pages = kv_pages(cache, page_table, ctx->d_status);
    P.idx = idx; P.n_rows = (uint32_t)rows.n_rows;
    P.rows_per_batch = FastDiv((uint32_t)(rows.rows_per_batch < rows.n_rows ? rows.rows_per_batch : rows.n_rows));
    const void* dense[2] = {k, v}; const void* pool[2] = {k_pool, v_pool}; const float* scale[2] = {k_scale, v_scale};
    const oc_rope_view* views[2] = {&rows.k, &rows.v};
    const uint64_t eb = rows.dtype == OC_DTYPE_F32 ? 4 : 2;
    for (int i = 0; i < 2; ++i) {
        P.dense[i] = (void*)dense[i]; P.pool[i] = (void*)pool[i]; P.scale[i] = (float*)scale[i];
        P.batch_stride[i] = views[i]->batch_stride; P.row_stride[i] = views[i]->row_stride; P.head_stride[i] = views[i]->head_stride;
        P.wide[i] = ((uintptr_t)dense[i] | ((uint64_t)views[i]->batch_stride | (uint64_t)views[i]->row_stride | (uint64_t)views[i]->head_stride) * eb) % 16 == 0;
    }
    P.lph = cache.head_dim / 8; P.rpw = 32 / P.lph;
    P.head_blocks = (cache.heads + KV_HEADS - 1) / KV_HEADS; P.block_heads = (cache.heads + P.head_blocks - 1) / P.head_blocks;
    const uint32_t per_cta = (uint32_t)(KV_WARPS * P.rpw);
    const dim3 grid((P.n_rows + per_cta - 1) / per_cta, (unsigned)(P.head_blocks * (v ? 2 : 1)));
    LaunchScope scope(ctx, put ? OC_K_KV_PUT : OC_K_KV_GET, s);
    if (put) launch_kv_as<true>(P, rows.dtype, cache.dtype, grid, s);
    else launch_kv_as<false>(P, rows.dtype, cache.dtype, grid, s);
    return last_launch_status();
}

}  // namespace oc
