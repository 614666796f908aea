// Rotary positions with up to three axes on queries and keys, after an optional RMS norm of each head:
//     pair (a, b) of a head, angle = position on the pair's axis * the pair's frequency:
//     a' = a cos - b sin,  b' = b cos + a sin
// A head's d_0 + d_1 + d_2 leading elements are rotated, d_a of them by the position on axis a (time, height,
// width); the rest pass through.  cos and sin come from a table of a few KB with one line per position and axis.
//
// The kernel is bound by the bytes of q and k, so what it is built for is to touch nothing else often: a thread
// owns one unit (W pairs split over two vectors, or the pairs of one vector) of one row, looks its cosines up
// once, and then walks over the heads, which all turn by the same angles.  lph lanes make up a head, for the
// sum of squares of its norm; rows of 32 / lph tokens share a warp, so heads of 72 elements leave few lanes idle.
#include <string.h>

#include "rows.cuh"

namespace oc {

static constexpr int ROPE_WARPS = 8;
static constexpr int ROPE_BATCH = 4;             // heads whose loads are in flight together

struct RopeParams {
    const void* in[2]; void* out[2]; const float* w[2];                     // q, k
    long long in_row[2], in_head[2], out_batch[2], out_row[2], out_head[2]; // elements
    int heads[2];
    const float2* table; const int32_t* idx; const int32_t* pos;
    uint32_t n_rows, rows_per_batch, unit_rows;
    int dims[3], pairs[3];                       // positions of an axis, pairs that it turns
    int axis_base[3];                            // table line 0 of an axis
    int D, P, units, units_rot, lph, rpw, heads_per_cta;
    float sign, eps, inv_d;
    int* status;
};

// N bytes as 32-bit words (2 bytes in the low half of one word)
template <int N> struct RopeRaw { uint32_t v[N < 4 ? 1 : N / 4]; };
template <int N> __device__ __forceinline__ RopeRaw<N> rope_load(const void* p) {
    RopeRaw<N> r;
    if constexpr (N == 16) { const uint4 t = ld_v4(p); r.v[0] = t.x; r.v[1] = t.y; r.v[2] = t.z; r.v[3] = t.w; }
    else if constexpr (N == 8) { const uint2 t = *(const uint2*)p; r.v[0] = t.x; r.v[1] = t.y; }
    else if constexpr (N == 4) r.v[0] = *(const uint32_t*)p;
    else r.v[0] = *(const uint16_t*)p;
    return r;
}
template <int N> __device__ __forceinline__ void rope_store(void* p, const RopeRaw<N>& r) {
    if constexpr (N == 16) st_v4(p, make_uint4(r.v[0], r.v[1], r.v[2], r.v[3]));
    else if constexpr (N == 8) *(uint2*)p = make_uint2(r.v[0], r.v[1]);
    else if constexpr (N == 4) *(uint32_t*)p = r.v[0];
    else *(uint16_t*)p = (uint16_t)r.v[0];
}
template <int DT, int W> __device__ __forceinline__ void rope_widen(const RopeRaw<W * (DT == OC_DTYPE_BF16 ? 2 : 4)>& r, float* f) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (DT == OC_DTYPE_F32) f[i] = __uint_as_float(r.v[i]);
        else f[i] = (i & 1) ? bf16_hi(r.v[i / 2]) : bf16_lo(r.v[i / 2]);
    }
}
template <int DT, int W> __device__ __forceinline__ RopeRaw<W * (DT == OC_DTYPE_BF16 ? 2 : 4)> rope_round(const float* f) {
    RopeRaw<W * (DT == OC_DTYPE_BF16 ? 2 : 4)> r;
    if (DT == OC_DTYPE_F32) {
#pragma unroll
        for (int i = 0; i < W; ++i) r.v[i] = __float_as_uint(f[i]);
    } else if (W == 1) {
        r.v[0] = pack_bf16x2(f[0], 0.0f);
    } else {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) r.v[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    }
    return r;
}

// HALVES: a unit is W pairs, first members in one vector and second members in another.
// ADJACENT: a unit is one vector of W elements, W / 2 pairs.
template <int DT, int HALVES, int W, int UPL, bool NORM>
__global__ void __launch_bounds__(ROPE_WARPS * 32)
rope_kernel(const __grid_constant__ RopeParams P) {
    constexpr int VECS = HALVES ? 2 : 1, NP = HALVES ? W : W / 2, EB = DT == OC_DTYPE_BF16 ? 2 : 4, VB = W * EB;
    const int lane = threadIdx.x & 31, sub = lane / P.lph, u0 = lane - sub * P.lph;
    pdl_enter();
    const uint32_t row = (blockIdx.x * ROPE_WARPS + (threadIdx.x >> 5)) * (uint32_t)P.rpw + sub;
    bool in = sub < P.rpw && row < P.n_rows;
    int at[3] = {0, 0, 0};
    if (in) {
        if (P.pos) {
#pragma unroll
            for (int a = 0; a < 3; ++a) {
                at[a] = __ldg(P.pos + 3 * (long long)row + a);
                if (P.pairs[a] && (uint32_t)at[a] >= (uint32_t)P.dims[a]) in = false;
            }
            if (!in) atomicCAS(P.status, 0, OC_ERR_INVALID_ARG);             // a position that the table does not have
        } else {
            uint32_t unit = P.unit_rows == 1 ? row : row / P.unit_rows, rest = row - unit * P.unit_rows;
            if (P.idx) {
                const int i = __ldg(P.idx + unit);
                in = i >= 0;                                                 // the unused tail of a kept list
                unit = (uint32_t)i;
            }
            if (in) {
                const uint64_t token = (uint64_t)unit * P.unit_rows + rest;
                uint32_t r = (uint32_t)(token % ((uint64_t)P.dims[0] * P.dims[1] * P.dims[2]));
                at[2] = r % P.dims[2]; r /= P.dims[2];
                at[1] = r % P.dims[1]; at[0] = r / P.dims[1];
            }
        }
    }
    // the unit's cosines and sines, and where its vectors lie in a head
    float cs[UPL][NP], sn[UPL][NP];
    int off[UPL][VECS];
    bool have[UPL][VECS];
#pragma unroll
    for (int k = 0; k < UPL; ++k) {
        const int u = u0 + k * P.lph;
        const bool rot = u < P.units_rot;
        if (HALVES) {
            off[k][0] = rot ? W * u : 2 * P.P + 2 * W * (u - P.units_rot);
            off[k][VECS - 1] = rot ? P.P + W * u : off[k][0] + W;
        } else {
            off[k][0] = W * u;
        }
#pragma unroll
        for (int v = 0; v < VECS; ++v) have[k][v] = in && u < P.units && off[k][v] < P.D;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            cs[k][p] = 1.0f; sn[k][p] = 0.0f;
            if (rot && in) {
                int j = NP * u + p, a = 0;
                if (j >= P.pairs[0]) { j -= P.pairs[0]; a = 1; if (j >= P.pairs[1]) { j -= P.pairs[1]; a = 2; } }
                const int line = a == 0 ? at[0] : (a == 1 ? at[1] : at[2]);
                const float2 t = __ldg(P.table + P.axis_base[a] + (long long)line * P.pairs[a] + j);
                cs[k][p] = t.x; sn[k][p] = P.sign * t.y;
            }
        }
    }
    const uint32_t batch = in ? row / P.rows_per_batch : 0, in_batch = in ? row - batch * P.rows_per_batch : 0;
    const int first = blockIdx.y * P.heads_per_cta, last = first + P.heads_per_cta;
#pragma unroll
    for (int m = 0; m < 2; ++m) {                                            // q, then k
        const int base = m ? P.heads[0] : 0;
        const int lo = max(first - base, 0), hi = min(last - base, P.heads[m]);
        const uint8_t* src = (const uint8_t*)P.in[m] + (in ? (long long)row * P.in_row[m] : 0) * EB;
        uint8_t* dst = (uint8_t*)P.out[m] + ((long long)batch * P.out_batch[m] + (long long)in_batch * P.out_row[m]) * EB;
        float w[UPL][VECS][W];
        if (NORM && lo < hi) {
#pragma unroll
            for (int k = 0; k < UPL; ++k)
#pragma unroll
                for (int v = 0; v < VECS; ++v)
#pragma unroll
                    for (int i = 0; i < W; ++i) w[k][v][i] = have[k][v] ? __ldg(P.w[m] + off[k][v] + i) : 0.0f;
        }
        for (int h0 = lo; h0 < hi; h0 += ROPE_BATCH) {
            RopeRaw<VB> raw[ROPE_BATCH][UPL][VECS];
#pragma unroll
            for (int b = 0; b < ROPE_BATCH; ++b)
#pragma unroll
                for (int k = 0; k < UPL; ++k)
#pragma unroll
                    for (int v = 0; v < VECS; ++v) {
                        raw[b][k][v] = RopeRaw<VB>();
                        if (have[k][v] && h0 + b < hi)
                            raw[b][k][v] = rope_load<VB>(src + ((h0 + b) * P.in_head[m] + off[k][v]) * EB);
                    }
#pragma unroll
            for (int b = 0; b < ROPE_BATCH; ++b) {
                if (h0 + b >= hi) break;
                float f[UPL][VECS][W];
                float q = 0.0f;
#pragma unroll
                for (int k = 0; k < UPL; ++k)
#pragma unroll
                    for (int v = 0; v < VECS; ++v) {
                        rope_widen<DT, W>(raw[b][k][v], f[k][v]);
                        if (NORM) {
#pragma unroll
                            for (int i = 0; i < W; ++i) q = fmaf(f[k][v][i], f[k][v][i], q);
                        }
                    }
                if (NORM) {
                    // sum over the head's lph lanes, the upper half of the lanes onto the lower one until one is left
                    for (int s = P.lph; s > 1;) {
                        const int half = (s + 1) >> 1;
                        const float o = __shfl_down_sync(0xFFFFFFFFu, q, half);
                        if (u0 + half < s) q += o;
                        s = half;
                    }
                    q = __shfl_sync(0xFFFFFFFFu, q, sub * P.lph);
                    const float rstd = 1.0f / sqrtf(q * P.inv_d + P.eps);
#pragma unroll
                    for (int k = 0; k < UPL; ++k)
#pragma unroll
                        for (int v = 0; v < VECS; ++v)
#pragma unroll
                            for (int i = 0; i < W; ++i) f[k][v][i] *= rstd * w[k][v][i];
                }
#pragma unroll
                for (int k = 0; k < UPL; ++k) {
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        float& x = HALVES ? f[k][0][p] : f[k][0][2 * p];
                        float& y = HALVES ? f[k][VECS - 1][p] : f[k][0][2 * p + 1];
                        if (u0 + k * P.lph >= P.units_rot) continue;         // passes through, infinities and all
                        const float a = x, c = y;
                        x = fmaf(a, cs[k][p], -c * sn[k][p]);
                        y = fmaf(c, cs[k][p], a * sn[k][p]);
                    }
#pragma unroll
                    for (int v = 0; v < VECS; ++v)
                        if (have[k][v]) rope_store<VB>(dst + ((h0 + b) * P.out_head[m] + off[k][v]) * EB, rope_round<DT, W>(f[k][v]));
                }
            }
        }
    }
}

template <int DT, int HALVES, int W>
static void launch_rope_as(const RopeParams& P, int upl, bool norm, dim3 grid, cudaStream_t s) {
    if (upl == 1) {
        if (norm) OC_LAUNCH((rope_kernel<DT, HALVES, W, 1, true>), grid, ROPE_WARPS * 32, 0, s, P);
        else OC_LAUNCH((rope_kernel<DT, HALVES, W, 1, false>), grid, ROPE_WARPS * 32, 0, s, P);
    } else {
        if (norm) OC_LAUNCH((rope_kernel<DT, HALVES, W, 2, true>), grid, ROPE_WARPS * 32, 0, s, P);
        else OC_LAUNCH((rope_kernel<DT, HALVES, W, 2, false>), grid, ROPE_WARPS * 32, 0, s, P);
    }
}

// Elements per vector: the widest that pairs, heads, strides and pointers allow, 16 bytes at most.
int rope_vector(const oc_rope_desc& d, const void* q, const void* q_out, const void* k, const void* k_out) {
    const int eb = d.dtype == OC_DTYPE_BF16 ? 2 : 4;
    const long long rot = (long long)d.axis_dims[0] + d.axis_dims[1] + d.axis_dims[2];
    uint64_t e = (uint64_t)d.head_dim | (uint64_t)(d.pairing == OC_ROPE_HALVES ? rot / 2 : rot);
    const oc_rope_view* views[4] = {&d.q, &d.q_out, &d.k, &d.k_out};
    uint64_t bytes = (uint64_t)(uintptr_t)q | (uint64_t)(uintptr_t)q_out;
    for (int i = 0; i < (k ? 4 : 2); ++i) e |= (uint64_t)views[i]->row_stride | (uint64_t)views[i]->head_stride | (i & 1 ? (uint64_t)views[i]->batch_stride : 0);
    if (k) bytes |= (uint64_t)(uintptr_t)k | (uint64_t)(uintptr_t)k_out;
    int w = 16 / eb;
    while (w > 1 && ((e & (uint64_t)(w - 1)) || (bytes & (uint64_t)(w * eb - 1)))) w >>= 1;
    return (bytes & (uint64_t)(eb - 1)) ? 0 : w;
}

oc_status launch_rope(oc_ctx* ctx, const oc_rope_desc& d, const float* table, const int32_t* idx, const int32_t* pos,
                      const void* q, void* q_out, const float* q_w, const void* k, void* k_out, const float* k_w, cudaStream_t s) {
    const int w = rope_vector(d, q, q_out, k, k_out);
    const bool halves = d.pairing == OC_ROPE_HALVES;
    if (w == 0 || (!halves && w < 2)) return OC_ERR_ALIGNMENT;
    RopeParams P;
    memset(&P, 0, sizeof(P));
    P.in[0] = q; P.in[1] = k; P.out[0] = q_out; P.out[1] = k_out; P.w[0] = q_w; P.w[1] = k_w;
    const oc_rope_view* in[2] = {&d.q, &d.k}; const oc_rope_view* out[2] = {&d.q_out, &d.k_out};
    for (int m = 0; m < 2; ++m) {
        P.in_row[m] = in[m]->row_stride; P.in_head[m] = in[m]->head_stride;
        P.out_row[m] = out[m]->row_stride; P.out_head[m] = out[m]->head_stride; P.out_batch[m] = out[m]->batch_stride;
    }
    P.heads[0] = d.q_heads; P.heads[1] = k ? d.k_heads : 0;
    P.table = (const float2*)table; P.idx = idx; P.pos = pos;
    P.n_rows = (uint32_t)d.n_rows; P.rows_per_batch = (uint32_t)d.rows_per_batch; P.unit_rows = (uint32_t)d.unit_rows;
    int base = 0;
    for (int a = 0; a < 3; ++a) {
        P.dims[a] = d.axis_len[a]; P.pairs[a] = d.axis_dims[a] / 2; P.axis_base[a] = base;
        base += P.dims[a] * P.pairs[a];
        P.P += P.pairs[a];
    }
    P.D = d.head_dim;
    const int per = halves ? w : w / 2;                                      // pairs of a unit
    const int rest = P.D - 2 * P.P;                                          // elements that pass through
    P.units_rot = P.P / per;
    P.units = P.units_rot + (halves ? (rest + 2 * w - 1) / (2 * w) : rest / w);
    const int upl = P.units > 32 ? 2 : 1;
    if (P.units > 64) return OC_ERR_UNSUPPORTED;
    P.lph = (P.units + upl - 1) / upl; P.rpw = 32 / P.lph;
    P.sign = d.inverse ? -1.0f : 1.0f; P.eps = d.eps; P.inv_d = 1.0f / (float)P.D;
    P.status = ctx->d_status;
    // heads per CTA: all of them when there are rows enough to fill the device, fewer otherwise
    const long long rows_per_cta = (long long)ROPE_WARPS * P.rpw, row_ctas = (d.n_rows + rows_per_cta - 1) / rows_per_cta;
    const int heads = P.heads[0] + P.heads[1];
    const long long want = 4ll * ctx->sm_count;
    int splits = (int)((want + row_ctas - 1) / row_ctas);
    const int most = (heads + ROPE_BATCH - 1) / ROPE_BATCH;
    if (splits > most) splits = most;
    P.heads_per_cta = (heads + splits - 1) / splits;
    splits = (heads + P.heads_per_cta - 1) / P.heads_per_cta;
    if (splits > 65535) return OC_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)row_ctas, (unsigned)splits);
    const bool norm = q_w != nullptr;
    LaunchScope scope(ctx, OC_K_ROPE, s);
    if (d.dtype == OC_DTYPE_BF16) {
        if (halves) {
            if (w == 8) launch_rope_as<OC_DTYPE_BF16, 1, 8>(P, upl, norm, grid, s);
            else if (w == 4) launch_rope_as<OC_DTYPE_BF16, 1, 4>(P, upl, norm, grid, s);
            else if (w == 2) launch_rope_as<OC_DTYPE_BF16, 1, 2>(P, upl, norm, grid, s);
            else launch_rope_as<OC_DTYPE_BF16, 1, 1>(P, upl, norm, grid, s);
        } else {
            if (w == 8) launch_rope_as<OC_DTYPE_BF16, 0, 8>(P, upl, norm, grid, s);
            else if (w == 4) launch_rope_as<OC_DTYPE_BF16, 0, 4>(P, upl, norm, grid, s);
            else launch_rope_as<OC_DTYPE_BF16, 0, 2>(P, upl, norm, grid, s);
        }
    } else if (halves) {
        if (w == 4) launch_rope_as<OC_DTYPE_F32, 1, 4>(P, upl, norm, grid, s);
        else if (w == 2) launch_rope_as<OC_DTYPE_F32, 1, 2>(P, upl, norm, grid, s);
        else launch_rope_as<OC_DTYPE_F32, 1, 1>(P, upl, norm, grid, s);
    } else {
        if (w == 4) launch_rope_as<OC_DTYPE_F32, 0, 4>(P, upl, norm, grid, s);
        else launch_rope_as<OC_DTYPE_F32, 0, 2>(P, upl, norm, grid, s);
    }
    return last_launch_status();
}

}  // namespace oc
