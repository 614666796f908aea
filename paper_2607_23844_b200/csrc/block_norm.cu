// The row work between two blocks of a transformer whose tokens are partly cached, in one pass, and the 8-bit
// form of rows:
//     v = z[s] (s = slot of the row's unit) or the cached row,   r = a x + gate * post(v),
//     out = r,   cache = v,   h[s] = pre(r) (1 + scale) + shift    (h in fp32, bf16, or 8 bits with a scale per row)
// Statistics are taken from the registers that hold the row, in fp32 and in two passes (mean, then squared
// distances), so a large common offset costs no precision and nothing is read twice.  r stays in fp32 between
// the residual sum and the second norm: `out` is its rounding, h is not computed from that rounding.
#include "rows.cuh"

namespace oc {

struct BlockNormParams {
    const void* x; const void* z; const void* cache; void* cache_out; void* out; void* h; float* h_scale;
    const int32_t* slot_of;
    const void *post_w, *post_b, *gate, *pre_w, *pre_b, *scale, *shift;
    long long mod_stride;
    uint32_t n_rows, rows_per_group, unit_rows, dense_rows;
    int C, nvec, post_norm, pre_norm, h_dtype;
    float post_eps, pre_eps, res_scale, inv_c;
    int* status;
};

// (v - mean) * rstd in place; mean is 0 for an RMS norm.  Lanes past the row's end hold zeros and stay so.
template <int TPR, int VPT, int E>
__device__ __forceinline__ void normalise(float (&f)[VPT][E], int how, float eps, float inv_c, int nvec, int t,
                                          RowScratch* scratch, int& parity) {
    if (how == OC_NORM_NONE) return;
    float mean = 0.0f;
    if (how == OC_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) s += f[j][e];
        mean = row_sum<TPR>(s, scratch, parity) * inv_c;
    }
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
        if (j * TPR + t < nvec) {
#pragma unroll
            for (int e = 0; e < E; ++e) { f[j][e] -= mean; q = fmaf(f[j][e], f[j][e], q); }
        }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(q, scratch, parity) * inv_c + eps);   // (rsqrtf is off by up to 2 ulp, for the whole row)
#pragma unroll
    for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) f[j][e] *= rstd;
}

template <int DT, int PT, int TPR, int VPT>
__global__ void __launch_bounds__(TPR > 32 ? TPR : ROW_THREADS)
block_norm_kernel(const __grid_constant__ BlockNormParams P) {
    constexpr int E = RowVec<DT>::E;
    constexpr int THREADS = TPR > 32 ? TPR : ROW_THREADS, ROWS = THREADS / TPR;
    __shared__ RowScratch scratch_mem;
    RowScratch* scratch = TPR > 32 ? &scratch_mem : nullptr;
    int parity = 0;
    const int t = threadIdx.x % TPR;
    const uint32_t row = blockIdx.x * ROWS + threadIdx.x / TPR;
    pdl_enter();
    // (rows past the end run along with their warp or CTA -- the reductions need every lane -- and move nothing)
    const bool in = row < P.n_rows;
    const uint32_t unit = P.unit_rows == 1 ? row : row / P.unit_rows;
    uint32_t dense = row;
    bool computed = in;
    if (P.slot_of && in) {
        const int s = __ldg(P.slot_of + unit);
        computed = s >= 0;
        dense = (uint32_t)s * P.unit_rows + (row - unit * P.unit_rows);
        if (computed && ((uint32_t)s >= P.dense_rows / P.unit_rows)) {       // not a row of the dense buffers
            if (t == 0) atomicCAS(P.status, 0, OC_ERR_INVALID_ARG);
            computed = false;
        }
    }
    const bool want_r = in && (P.out || (P.h && computed));
    const bool want_v = in && P.z && (want_r || P.cache_out);

    const long long row_at = (long long)row * P.C, dense_at = (long long)dense * P.C;
    constexpr int EB = 16 / E;                                               // bytes of an element
    uint4 xv[VPT], vv[VPT];
    const uint8_t* xp = (const uint8_t*)P.x + row_at * EB;
    const uint8_t* vp = computed ? (const uint8_t*)P.z + dense_at * EB : (const uint8_t*)P.cache + row_at * EB;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        xv[j] = vv[j] = make_uint4(0, 0, 0, 0);
        if (j * TPR + t < P.nvec) {
            if (want_r) xv[j] = ld_v4(xp + (j * TPR + t) * 16);
            if (want_v) vv[j] = ld_v4(vp + (j * TPR + t) * 16);
        }
    }
    if (P.cache_out && in && (computed || P.cache_out != P.cache)) {
        uint8_t* cp = (uint8_t*)P.cache_out + row_at * EB;
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (j * TPR + t < P.nvec) st_v4(cp + (j * TPR + t) * 16, vv[j]);
    }
    const long long group_at = P.mod_stride == 0 || !in ? 0 : (long long)(row / P.rows_per_group) * P.mod_stride;

    float r[VPT][E];
    if (P.z) {
#pragma unroll
        for (int j = 0; j < VPT; ++j) RowVec<DT>::unpack(vv[j], r[j]);
        normalise<TPR, VPT, E>(r, P.post_norm, P.post_eps, P.inv_c, P.nvec, t, scratch, parity);
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (j * TPR + t < P.nvec) {
                const long long at = (long long)(j * TPR + t) * E;
                float p[E], x[E];
                if (P.post_w) {
                    load_param<PT, E>(P.post_w, at, p);
#pragma unroll
                    for (int e = 0; e < E; ++e) r[j][e] *= p[e];
                }
                if (P.post_b) {
                    load_param<PT, E>(P.post_b, at, p);
#pragma unroll
                    for (int e = 0; e < E; ++e) r[j][e] += p[e];
                }
                if (P.gate) {
                    load_param<PT, E>(P.gate, group_at + at, p);
#pragma unroll
                    for (int e = 0; e < E; ++e) r[j][e] *= p[e];
                }
                RowVec<DT>::unpack(xv[j], x);
#pragma unroll
                for (int e = 0; e < E; ++e) r[j][e] = fmaf(P.res_scale, x[e], r[j][e]);
            }
    } else {
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            RowVec<DT>::unpack(xv[j], r[j]);
#pragma unroll
            for (int e = 0; e < E; ++e) r[j][e] *= P.res_scale;
        }
    }
    if (P.out && in) {
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (j * TPR + t < P.nvec) store_row<DT, E>(P.out, row_at + (long long)(j * TPR + t) * E, r[j]);
    }
    if (!P.h) return;
    // a warp (or CTA) none of whose rows goes on is done
    if (TPR > 32 ? !computed : __all_sync(0xFFFFFFFFu, !computed)) return;
    normalise<TPR, VPT, E>(r, P.pre_norm, P.pre_eps, P.inv_c, P.nvec, t, scratch, parity);
#pragma unroll
    for (int j = 0; j < VPT; ++j)
        if (j * TPR + t < P.nvec) {
            const long long at = (long long)(j * TPR + t) * E;
            float p[E];
            if (P.pre_w) {
                load_param<PT, E>(P.pre_w, at, p);
#pragma unroll
                for (int e = 0; e < E; ++e) r[j][e] *= p[e];
            }
            if (P.pre_b) {
                load_param<PT, E>(P.pre_b, at, p);
#pragma unroll
                for (int e = 0; e < E; ++e) r[j][e] += p[e];
            }
            if (P.scale) {
                load_param<PT, E>(P.scale, group_at + at, p);
#pragma unroll
                for (int e = 0; e < E; ++e) r[j][e] = fmaf(r[j][e], p[e], r[j][e]);
            }
            if (P.shift) {
                load_param<PT, E>(P.shift, group_at + at, p);
#pragma unroll
                for (int e = 0; e < E; ++e) r[j][e] += p[e];
            }
        }
    if (P.h_dtype == OC_DTYPE_I8) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < VPT; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) { const uint32_t b = __float_as_uint(r[j][e]) & 0x7FFFFFFFu; m = b > m ? b : m; }
        const RowQuant q = row_quant(row_max_bits<TPR>(m, scratch, parity));
        if (!computed) return;
        if (t == 0) P.h_scale[dense] = q.scale;
#pragma unroll
        for (int j = 0; j < VPT; ++j)
            if (j * TPR + t < P.nvec) store_row_s8<E>(P.h, dense_at + (long long)(j * TPR + t) * E, r[j], q.inv);
        return;
    }
    if (!computed) return;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
        if (j * TPR + t < P.nvec) {
            const long long at = dense_at + (long long)(j * TPR + t) * E;
            if (P.h_dtype == OC_DTYPE_BF16) store_row<OC_DTYPE_BF16, E>(P.h, at, r[j]);
            else store_row<OC_DTYPE_F32, E>(P.h, at, r[j]);
        }
}

struct QuantParams {
    const void* x; const int32_t* idx; int8_t* q; float* scale;
    long long x_stride;
    uint32_t n_rows, x_rows;
    int C, nvec;
    int* status;
};

template <int DT, int TPR, int VPT>
__global__ void __launch_bounds__(TPR > 32 ? TPR : ROW_THREADS)
quantize_rows_kernel(const __grid_constant__ QuantParams P) {
    constexpr int E = RowVec<DT>::E;
    constexpr int THREADS = TPR > 32 ? TPR : ROW_THREADS, ROWS = THREADS / TPR;
    __shared__ RowScratch scratch_mem;
    RowScratch* scratch = TPR > 32 ? &scratch_mem : nullptr;
    int parity = 0;
    const int t = threadIdx.x % TPR;
    const uint32_t row = blockIdx.x * ROWS + threadIdx.x / TPR;
    pdl_enter();
    bool in = row < P.n_rows;
    uint32_t src = row;
    if (P.idx && in) {
        const int i = __ldg(P.idx + row);
        in = i >= 0;                                                         // the unused tail of a kept list
        src = (uint32_t)i;
        if (in && src >= P.x_rows) {
            if (t == 0) atomicCAS(P.status, 0, OC_ERR_INVALID_ARG);
            in = false;
        }
    }
    const uint8_t* xp = (const uint8_t*)P.x + (long long)src * P.x_stride * (16 / E);
    float r[VPT][E];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (in && j * TPR + t < P.nvec) v = ld_v4(xp + (j * TPR + t) * 16);
        RowVec<DT>::unpack(v, r[j]);
#pragma unroll
        for (int e = 0; e < E; ++e) { const uint32_t b = __float_as_uint(r[j][e]) & 0x7FFFFFFFu; m = b > m ? b : m; }
    }
    const RowQuant q = row_quant(row_max_bits<TPR>(m, scratch, parity));
    if (!in) return;
    if (t == 0) P.scale[row] = q.scale;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
        if (j * TPR + t < P.nvec) store_row_s8<E>(P.q, (long long)row * P.C + (long long)(j * TPR + t) * E, r[j], q.inv);
}

template <int DT, int PT>
static bool launch_block_norm_as(const BlockNormParams& P, cudaStream_t s) {
    return row_split(P.nvec, [&](auto split) {
        constexpr int TPR = decltype(split)::tpr, VPT = decltype(split)::vpt;
        constexpr int THREADS = TPR > 32 ? TPR : ROW_THREADS, ROWS = THREADS / TPR;
        OC_LAUNCH((block_norm_kernel<DT, PT, TPR, VPT>), (P.n_rows + ROWS - 1) / ROWS, THREADS, 0, s, P);
    });
}

oc_status launch_block_norm(oc_ctx* ctx, const oc_block_norm_desc& d, const void* x, const void* z, const int32_t* slot_of,
                            const void* cache, void* cache_out, void* out, const void* post_w, const void* post_b,
                            const void* gate, const void* pre_w, const void* pre_b, const void* scale, const void* shift,
                            void* h, float* h_scale, cudaStream_t s) {
    const int e = d.dtype == OC_DTYPE_BF16 ? 8 : 4;
    BlockNormParams P;
    P.x = x; P.z = z; P.cache = cache; P.cache_out = cache_out; P.out = out; P.h = h; P.h_scale = h_scale; P.slot_of = slot_of;
    P.post_w = post_w; P.post_b = post_b; P.gate = gate; P.pre_w = pre_w; P.pre_b = pre_b; P.scale = scale; P.shift = shift;
    P.mod_stride = d.mod_stride;
    P.n_rows = (uint32_t)d.n_rows; P.rows_per_group = (uint32_t)d.rows_per_group; P.unit_rows = (uint32_t)d.unit_rows;
    P.dense_rows = (uint32_t)d.dense_rows;
    P.C = (int)d.C; P.nvec = (int)(d.C / e); P.post_norm = d.post_norm; P.pre_norm = d.pre_norm; P.h_dtype = d.h_dtype;
    P.post_eps = d.post_eps; P.pre_eps = d.pre_eps; P.res_scale = d.res_scale; P.inv_c = 1.0f / (float)d.C;
    P.status = ctx->d_status;
    if (P.nvec > 3072) return OC_ERR_UNSUPPORTED;
    LaunchScope scope(ctx, OC_K_BLOCK_NORM, s);
    const bool pf = d.param_dtype == OC_DTYPE_F32;
    if (d.dtype == OC_DTYPE_BF16) {
        if (pf) launch_block_norm_as<OC_DTYPE_BF16, OC_DTYPE_F32>(P, s);
        else launch_block_norm_as<OC_DTYPE_BF16, OC_DTYPE_BF16>(P, s);
    } else {
        if (pf) launch_block_norm_as<OC_DTYPE_F32, OC_DTYPE_F32>(P, s);
        else launch_block_norm_as<OC_DTYPE_F32, OC_DTYPE_BF16>(P, s);
    }
    return last_launch_status();
}

oc_status launch_quantize_rows(oc_ctx* ctx, const void* x, int dtype, int64_t x_rows, int64_t x_stride, const int32_t* idx,
                               int64_t n_rows, int64_t K, int8_t* q, float* scale, cudaStream_t s) {
    QuantParams P;
    P.x = x; P.idx = idx; P.q = q; P.scale = scale; P.x_stride = x_stride;
    P.n_rows = (uint32_t)n_rows; P.x_rows = (uint32_t)x_rows; P.C = (int)K;
    P.nvec = (int)(K / (dtype == OC_DTYPE_BF16 ? 8 : 4));
    P.status = ctx->d_status;
    if (P.nvec > 3072) return OC_ERR_UNSUPPORTED;
    LaunchScope scope(ctx, OC_K_QUANT, s);
    row_split(P.nvec, [&](auto split) {
        constexpr int TPR = decltype(split)::tpr, VPT = decltype(split)::vpt;
        constexpr int THREADS = TPR > 32 ? TPR : ROW_THREADS, ROWS = THREADS / TPR;
        const dim3 grid((P.n_rows + ROWS - 1) / ROWS);
        if (dtype == OC_DTYPE_BF16) OC_LAUNCH((quantize_rows_kernel<OC_DTYPE_BF16, TPR, VPT>), grid, THREADS, 0, s, P);
        else OC_LAUNCH((quantize_rows_kernel<OC_DTYPE_F32, TPR, VPT>), grid, THREADS, 0, s, P);
    });
    return last_launch_status();
}

}  // namespace oc
