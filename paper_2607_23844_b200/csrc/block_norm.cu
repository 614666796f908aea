// The row work between two blocks of a transformer whose tokens are partly cached, in one pass, and the 8-bit
// form of rows:
//     v = z[s] (s = slot of the row's unit) or the cached row,   r = a x + gate * post(v),
//     out = r,   cache = v,   h[s] = pre(r) (1 + scale) + shift    (h in fp32, bf16, or 8 bits with a scale per row)
// Statistics are taken from the registers that hold the row, in fp32 and in two passes (mean, then squared
// distances), so a large common offset costs no precision and nothing is read twice.  r stays in fp32 between
// the residual sum and the second norm: `out` is its rounding, h is not computed from that rounding.
//
// Bound by DRAM where rows are many: 230400 rows of 320 bf16 under Frame Cache, 667 MB, take 115 us (5.8 TB/s).  8192
// rows of 1536 (107 MB) take 23.9 us: about five rounds of row sets an SM, whose parameters cost 4 us (20.2 without).
#include <algorithm>
#include <atomic>

#include "rows.cuh"

namespace oc {

struct BlockNormParams {
    const void* x; const void* z; const void* cache; void* cache_out; void* out; void* h; float* h_scale;
    const int32_t* slot_of;
    const void *post_w, *post_b, *gate, *pre_w, *pre_b, *scale, *shift;
    long long mod_stride;
    uint32_t n_rows, dense_units;
    FastDiv unit_rows, rows_per_group;
    int C, nvec, post_norm, pre_norm, h_dtype;
    uint32_t sets, queue;                    // sets of rows; how many a CTA works through, one after the other
    int folds;                               // which folded parameters there are (Fold bits); 16: they are kept in shared memory
    float post_eps, pre_eps, res_scale, inv_c;
    int* status;
};

// (v - mean) / sqrt(mean square + eps) in place; mean is 0 for an RMS norm.  Vectors past the row's end hold zeros
// and stay so.
template <class S, int E>
__device__ __forceinline__ void normalise(f32x2 (&f)[S::vpt][E / 2], int how, float eps, float inv_c, int nvec, int t,
                                          RowScratch* scratch, int& parity) {
    if (how == OC_NORM_NONE) return;
    f32x2 q = 0;
    if (how == OC_NORM_LAYER) {
        f32x2 s = 0;
#pragma unroll
        for (int j = 0; j < S::vpt; ++j)
#pragma unroll
            for (int e = 0; e < E / 2; ++e) s = f2_add(s, f[j][e]);
        const float mean = row_sum<S::tpr>(f2_lo(s) + f2_hi(s), scratch, parity) * inv_c;
#pragma unroll
        for (int j = 0; j < S::vpt; ++j) {
            const f32x2 m = f2(S::has(j, t, nvec) ? -mean : 0.0f);
#pragma unroll
            for (int e = 0; e < E / 2; ++e) { f[j][e] = f2_add(f[j][e], m); q = f2_fma(f[j][e], f[j][e], q); }
        }
    } else {
#pragma unroll
        for (int j = 0; j < S::vpt; ++j)
#pragma unroll
            for (int e = 0; e < E / 2; ++e) q = f2_fma(f[j][e], f[j][e], q);
    }
    // (rsqrtf would be off by up to 2 ulp, for the whole row)
    const f32x2 rstd = f2(1.0f / sqrtf(row_sum<S::tpr>(f2_lo(q) + f2_hi(q), scratch, parity) * inv_c + eps));
#pragma unroll
    for (int j = 0; j < S::vpt; ++j)
#pragma unroll
        for (int e = 0; e < E / 2; ++e) f[j][e] = f2_mul(f[j][e], rstd);
}

// The up to seven parameter vectors of a group act as four: t = post * A + B, h = pre * C + D with
//     A = post_w gate, B = post_b gate, C = pre_w (1 + scale), D = pre_b (1 + scale) + shift.
enum Fold { FOLD_A = 1, FOLD_B = 2, FOLD_C = 4, FOLD_D = 8, FOLD_KEPT = 16 };
template <int PT, int E>
__device__ __forceinline__ void fold(const BlockNormParams& P, int which, long long group_at, int at, f32x2* f) {
    const void* w = which == FOLD_A ? P.post_w : which == FOLD_B ? P.post_b : which == FOLD_C ? P.pre_w : P.pre_b;
    const void* m = which <= FOLD_B ? P.gate : P.scale;
    f32x2 p[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) f[e] = f2(which == FOLD_D ? 0.0f : 1.0f);
    if (w) load_param<PT, E>(w, at, f);
    if (m && (which != FOLD_D || w)) {
        load_param<PT, E>(m, group_at + at, p);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) f[e] = which <= FOLD_B ? f2_mul(f[e], p[e]) : f2_fma(f[e], p[e], f[e]);
    }
    if (which == FOLD_D && P.shift) {
        load_param<PT, E>(P.shift, group_at + at, p);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) f[e] = f2_add(f[e], p[e]);
    }
}
// E elements of a kept vector
template <int E> __device__ __forceinline__ void kept(const float* v, int at, f32x2* f) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) RowVec<OC_DTYPE_F32>::unpack(*(const uint4*)(v + at + 4 * i), f + 2 * i);
}
// r = r * a + b over a row, a and b (either may be absent) from shared memory or folded on the spot
template <int PT, class S, int E>
__device__ __forceinline__ void affine(f32x2 (&r)[S::vpt][E / 2], const BlockNormParams& P, int which_a, int which_b, const float* a,
                                       const float* b, bool in_smem, long long group_at, int t) {
    const bool has_a = P.folds & which_a, has_b = P.folds & which_b;
#pragma unroll
    for (int j = 0; j < S::vpt; ++j)
        if (S::has(j, t, P.nvec)) {
            const int at = (j * S::tpr + t) * E;
            f32x2 p[E / 2];
            if (has_a) {
                if (in_smem) kept<E>(a, at, p); else fold<PT, E>(P, which_a, group_at, at, p);
#pragma unroll
                for (int e = 0; e < E / 2; ++e) r[j][e] = f2_mul(r[j][e], p[e]);
            }
            if (has_b) {
                if (in_smem) kept<E>(b, at, p); else fold<PT, E>(P, which_b, group_at, at, p);
#pragma unroll
                for (int e = 0; e < E / 2; ++e) r[j][e] = f2_add(r[j][e], p[e]);
            }
        }
}

// What a row's threads know about it before its data is there.
struct RowPlan {
    uint32_t row, dense;
    bool in, computed, want_r, want_v;
};

// A CTA works through consecutive sets of rows.  A row's x and v travel through shared memory (16-byte
// asynchronous copies, each thread's own vectors into its own words, so that nobody waits for anybody): the next
// row's are asked for as soon as this one's are used up, half way through its work.  The folded parameters of the
// group at hand lie in shared memory too -- every row reads all of them: 8192 rows of 1536 take 23.0 us, and 29.5 where
// each row reads and folds them itself; 230400 of 320 take 119 and 162.  A set of rows that belongs to several groups
// folds its own.
template <int DT, int PT, bool Z, class S>       // Z: there is a block's output
__global__ void __launch_bounds__(RowCta<S::tpr>::threads)
block_norm_kernel(const __grid_constant__ BlockNormParams P) {
    constexpr int E = RowVec<DT>::E, EB = 16 / E, TPR = S::tpr, VPT = S::vpt;   // (EB: bytes of an element)
    constexpr int THREADS = RowCta<TPR>::threads, ROWS = RowCta<TPR>::rows;
    extern __shared__ __align__(16) uint4 smem4[];                           // [x, v if Z][VPT][THREADS], then the folded vectors
    __shared__ RowScratch scratch_mem[ROWS];
    RowScratch* scratch = TPR > 32 ? scratch_mem + threadIdx.x / TPR : nullptr;
    int parity = 0;
    const int t = threadIdx.x % TPR;
    const uint4* held = smem4 + threadIdx.x;
    const uint32_t copy_to = smem_u32(held);
    float* tab[4];
    {
        float* at = (float*)(smem4 + (Z ? 2 : 1) * VPT * THREADS);
#pragma unroll
        for (int i = 0; i < 4; ++i) { tab[i] = at; if (P.folds & (1 << i)) at += P.C; }
    }
    pdl_enter();

    auto slot_at = [&](uint32_t row) -> int { return P.slot_of && row < P.n_rows ? __ldg(P.slot_of + P.unit_rows.div(row)) : 0; };
    auto plan = [&](uint32_t row, int slot) {
        RowPlan r;
        r.row = row; r.in = row < P.n_rows; r.dense = row; r.computed = r.in;
        if (P.slot_of && r.in) {
            r.computed = slot >= 0;
            r.dense = (uint32_t)slot * P.unit_rows.d + (row - P.unit_rows.div(row) * P.unit_rows.d);
            if (r.computed && (uint32_t)slot >= P.dense_units) {             // not a row of the dense buffers
                if (t == 0) atomicCAS(P.status, 0, OC_ERR_INVALID_ARG);
                r.computed = false;
            }
        }
        r.want_r = r.in && (P.out || (P.h && r.computed));
        r.want_v = Z && r.in && (r.want_r || P.cache_out);
        return r;
    };
    // (vectors past the row's end, and rows that are not wanted, arrive as zeros)
    auto fetch = [&](const RowPlan& r) {
        const uint8_t* xp = (const uint8_t*)P.x + (r.want_r ? (long long)r.row * P.C * EB : 0);
        const uint8_t* vp = !r.want_v ? (const uint8_t*)P.x
                          : r.computed ? (const uint8_t*)P.z + (long long)r.dense * P.C * EB : (const uint8_t*)P.cache + (long long)r.row * P.C * EB;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            const bool there = S::has(j, t, P.nvec);
            const int at = there ? (j * TPR + t) * 16 : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(copy_to + (uint32_t)(j * THREADS * 16)), "l"(xp + at), "r"(there && r.want_r ? 16 : 0) : "memory");
            if (Z)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(copy_to + (uint32_t)((VPT + j) * THREADS * 16)), "l"(vp + at), "r"(there && r.want_v ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    // (n_rows and a CTA's rows past it stay below 2^32: the last set of rows begins before n_rows)
    const uint32_t set0 = blockIdx.x * P.queue;
    const int trips = (int)min(P.queue, P.sets - set0);
    uint32_t base = set0 * ROWS, next_row = base + threadIdx.x / TPR;
    RowPlan R = plan(next_row, slot_at(next_row));
    fetch(R);
    next_row += ROWS;
    int next_slot = slot_at(next_row);
    uint32_t tab_group = 0xFFFFFFFFu;
    for (int trip = 0; trip < trips; ++trip, base += ROWS) {
        const uint32_t last = min(base + ROWS, P.n_rows) - 1u;
        const uint32_t group = P.mod_stride ? P.rows_per_group.div(base) : 0u;
        const bool in_smem = (P.folds & FOLD_KEPT) && (!P.mod_stride || P.rows_per_group.div(last) == group);
        if (in_smem && group != tab_group) {                                 // (the same for the whole CTA)
            __syncthreads();                                                 // everybody is done with the last group's
            for (int at = threadIdx.x * E; at < P.C; at += THREADS * E)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (P.folds & (1 << i)) {
                        f32x2 f[E / 2];
                        fold<PT, E>(P, 1 << i, (long long)group * P.mod_stride, at, f);
                        store_row_smem<E>(tab[i] + at, f);
                    }
            __syncthreads();
            tab_group = group;
        }
        const long long row_at = (long long)R.row * P.C, dense_at = (long long)R.dense * P.C;
        const long long group_at = P.mod_stride && R.in ? (long long)P.rows_per_group.div(R.row) * P.mod_stride : 0;
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (Z && P.cache_out && R.in && (R.computed || P.cache_out != P.cache)) {
            uint8_t* cp = (uint8_t*)P.cache_out + row_at * EB;
#pragma unroll
            for (int j = 0; j < VPT; ++j)
                if (S::has(j, t, P.nvec)) st_v4(cp + (j * TPR + t) * 16, held[(VPT + j) * THREADS]);
        }
        f32x2 r[VPT][E / 2];
        if (Z) {
#pragma unroll
            for (int j = 0; j < VPT; ++j) RowVec<DT>::unpack(held[(VPT + j) * THREADS], r[j]);
            normalise<S, E>(r, P.post_norm, P.post_eps, P.inv_c, P.nvec, t, scratch, parity);
            affine<PT, S, E>(r, P, FOLD_A, FOLD_B, tab[0], tab[1], in_smem, group_at, t);
        } else {
#pragma unroll
            for (int j = 0; j < VPT; ++j)
#pragma unroll
                for (int e = 0; e < E / 2; ++e) r[j][e] = 0;
        }
        const f32x2 res = f2(P.res_scale);
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
            f32x2 x[E / 2];
            RowVec<DT>::unpack(held[j * THREADS], x);
#pragma unroll
            for (int e = 0; e < E / 2; ++e) r[j][e] = f2_fma(res, x[e], r[j][e]);
        }
        if (P.out && R.in) {
#pragma unroll
            for (int j = 0; j < VPT; ++j)
                if (S::has(j, t, P.nvec)) store_row<DT, E>(P.out, row_at + (j * TPR + t) * E, r[j]);
        }
        const RowPlan N = plan(next_row, next_slot);
        if (trip + 1 < trips) fetch(N);
        next_row += ROWS;
        // (the rows after this CTA's last set are another CTA's: no slot, so that their plan here reports none)
        next_slot = trip + 2 < trips ? slot_at(next_row) : -1;
        // a warp (or the warps of one row) none of whose rows goes on is done
        const bool goes_on = P.h && (TPR > 32 ? R.computed : __any_sync(0xFFFFFFFFu, R.computed));
        if (goes_on) {
            normalise<S, E>(r, P.pre_norm, P.pre_eps, P.inv_c, P.nvec, t, scratch, parity);
            affine<PT, S, E>(r, P, FOLD_C, FOLD_D, tab[2], tab[3], in_smem, group_at, t);
            if (P.h_dtype == OC_DTYPE_I8) {
                uint32_t m = 0;
#pragma unroll
                for (int j = 0; j < VPT; ++j) m = max_bits<E>(r[j], m);
                const RowQuant q = row_quant(row_max_bits<TPR>(m, scratch, parity));
                if (R.computed) {
                    if (t == 0) P.h_scale[R.dense] = q.scale;
#pragma unroll
                    for (int j = 0; j < VPT; ++j)
                        if (S::has(j, t, P.nvec)) store_row_s8<E>(P.h, dense_at + (j * TPR + t) * E, r[j], q.inv);
                }
            } else if (R.computed) {
#pragma unroll
                for (int j = 0; j < VPT; ++j)
                    if (S::has(j, t, P.nvec)) {
                        const long long at = dense_at + (j * TPR + t) * E;
                        if (P.h_dtype == OC_DTYPE_BF16) store_row<OC_DTYPE_BF16, E>(P.h, at, r[j]);
                        else store_row<OC_DTYPE_F32, E>(P.h, at, r[j]);
                    }
            }
        }
        R = N;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

struct QuantParams {
    const void* x; const int32_t* idx; int8_t* q; float* scale;
    long long x_stride;
    uint32_t n_rows, x_rows;
    int C, nvec;
    int* status;
};

template <int DT, class S>
__global__ void __launch_bounds__(RowCta<S::tpr>::threads)
quantize_rows_kernel(const __grid_constant__ QuantParams P) {
    constexpr int E = RowVec<DT>::E, TPR = S::tpr, VPT = S::vpt;
    constexpr int ROWS = RowCta<TPR>::rows;
    __shared__ RowScratch scratch_mem[ROWS];
    RowScratch* scratch = TPR > 32 ? scratch_mem + threadIdx.x / TPR : nullptr;
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
    f32x2 r[VPT][E / 2];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (in && S::has(j, t, P.nvec)) v = ld_v4(xp + (j * TPR + t) * 16);
        RowVec<DT>::unpack(v, r[j]);
        m = max_bits<E>(r[j], m);
    }
    const RowQuant q = row_quant(row_max_bits<TPR>(m, scratch, parity));
    if (!in) return;
    if (t == 0) P.scale[row] = q.scale;
#pragma unroll
    for (int j = 0; j < VPT; ++j)
        if (S::has(j, t, P.nvec)) store_row_s8<E>(P.q, (long long)row * P.C + (long long)(j * TPR + t) * E, r[j], q.inv);
}

template <int DT, int PT, bool Z>
static bool launch_block_norm_as(oc_ctx* ctx, BlockNormParams& P, cudaStream_t s) {
    bool ok = true;
    row_split(P.nvec, [&](auto split) {
        using S = decltype(split);
        constexpr int THREADS = RowCta<S::tpr>::threads, ROWS = RowCta<S::tpr>::rows, MOST = 200 * 1024;
        auto* kernel = block_norm_kernel<DT, PT, Z, S>;
        static PerDeviceOnce once;                   // (the context's device is current here)
        ok = once.ensure(ctx->device, [&] {
            const bool good = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST) == cudaSuccess;
            if (!good) cudaGetLastError();
            return good;
        });
        if (!ok) return;
        const long long sets = ((long long)P.n_rows + ROWS - 1) / ROWS;
        constexpr int rows_bytes = (Z ? 2 : 1) * S::vpt * THREADS * 16;
        int kept_bytes = 0;
        for (int i = 0; i < 4; ++i) if (P.folds & (1 << i)) kept_bytes += P.C * 4;
        // (not for rows so wide that one CTA would fill an SM)
        if (kept_bytes && rows_bytes + kept_bytes <= MOST / 2) P.folds |= FOLD_KEPT;
        const int smem = rows_bytes + ((P.folds & FOLD_KEPT) ? kept_bytes : 0);
        // resident CTAs for that much shared memory: asked once and remembered (the question costs as much as a launch)
        static std::atomic<uint64_t> known{0};
        const uint64_t key = ((uint64_t)smem << 16) | (uint64_t)(ctx->device & 0xFF) << 8;
        const uint64_t last = known.load(std::memory_order_relaxed);
        int per_sm = (int)(last & 0xFF);
        if ((last & ~0xFFull) != key || per_sm == 0) {
            if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, THREADS, smem) != cudaSuccess || per_sm < 1) { cudaGetLastError(); ok = false; return; }
            known.store(key | (uint64_t)per_sm, std::memory_order_relaxed);
        }
        // Queues of equal length with every CTA resident, unless that makes long ones: 230400 rows of 320, half of the
        // frames with slots, take 127 us in 740 queues of 20 sets and 100 in queues of 4 (64 rows), which are near one
        // another in DRAM at any time; 106 in queues of 2, which fold the parameters too often, and 109 of 8.  57600
        // rows of 640: 59 us in resident queues of 13 sets, 57 in queues of 4, 62 of 8.  8192 rows of 1536: 23 us in
        // resident queues of 5 sets; 30, 28, 31 and 30 in queues of 2, 3, 4 and 8, which are a round and a bit.
        const long long resident = (long long)ctx->sm_count * per_sm, short_queue = std::max(4, 64 / ROWS);
        const long long queue = sets / short_queue > 2 * resident ? short_queue : (sets + resident - 1) / resident;
        const long long ctas = (sets + queue - 1) / queue;
        P.sets = (uint32_t)sets; P.queue = (uint32_t)queue;
        OC_LAUNCH(kernel, (unsigned)ctas, THREADS, smem, s, P);
    });
    return ok;
}

template <int DT, int PT>
static bool launch_block_norm_z(oc_ctx* ctx, BlockNormParams& P, cudaStream_t s) {
    return P.z ? launch_block_norm_as<DT, PT, true>(ctx, P, s) : launch_block_norm_as<DT, PT, false>(ctx, P, s);
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
    // (more rows per group, or per unit, than there are rows is all of them)
    P.n_rows = (uint32_t)d.n_rows; P.dense_units = (uint32_t)(d.dense_rows / d.unit_rows);
    P.unit_rows = FastDiv((uint32_t)d.unit_rows);
    P.rows_per_group = FastDiv((uint32_t)(d.rows_per_group < d.n_rows ? d.rows_per_group : d.n_rows));
    P.C = (int)d.C; P.nvec = (int)(d.C / e); P.post_norm = d.post_norm; P.pre_norm = d.pre_norm; P.h_dtype = d.h_dtype;
    P.post_eps = d.post_eps; P.pre_eps = d.pre_eps; P.res_scale = d.res_scale; P.inv_c = 1.0f / (float)d.C;
    P.folds = (post_w || gate ? FOLD_A : 0) | (post_b ? FOLD_B : 0) |
              (h ? (pre_w || scale ? FOLD_C : 0) | (pre_b || shift ? FOLD_D : 0) : 0);
    P.status = ctx->d_status;
    if (P.nvec > 3072) return OC_ERR_UNSUPPORTED;
    LaunchScope scope(ctx, OC_K_BLOCK_NORM, s);
    const bool pf = d.param_dtype == OC_DTYPE_F32;
    bool ok;
    if (d.dtype == OC_DTYPE_BF16) {
        ok = pf ? launch_block_norm_z<OC_DTYPE_BF16, OC_DTYPE_F32>(ctx, P, s) : launch_block_norm_z<OC_DTYPE_BF16, OC_DTYPE_BF16>(ctx, P, s);
    } else {
        ok = pf ? launch_block_norm_z<OC_DTYPE_F32, OC_DTYPE_F32>(ctx, P, s) : launch_block_norm_z<OC_DTYPE_F32, OC_DTYPE_BF16>(ctx, P, s);
    }
    return ok ? last_launch_status() : OC_ERR_CUDA;
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
        using S = decltype(split);
        constexpr int THREADS = RowCta<S::tpr>::threads, ROWS = RowCta<S::tpr>::rows;
        const dim3 grid((P.n_rows + ROWS - 1) / ROWS);
        if (dtype == OC_DTYPE_BF16) OC_LAUNCH((quantize_rows_kernel<OC_DTYPE_BF16, S>), grid, THREADS, 0, s, P);
        else OC_LAUNCH((quantize_rows_kernel<OC_DTYPE_F32, S>), grid, THREADS, 0, s, P);
    });
    return last_launch_status();
}

}  // namespace oc
