// Rotary positions with up to three axes on queries and keys, after an optional RMS norm of each head:
//     pair (a, b) of a head, angle = position on the pair's axis * the pair's frequency:
//     a' = a cos - b sin,  b' = b cos + a sin
// A head's d_0 + d_1 + d_2 leading elements are rotated, d_a of them by the position on axis a (time, height,
// width); the rest pass through.  cos and sin come from a table of a few KB with one line per position and axis.
//
// The kernel is bound by the bytes of q and k.  A thread owns one unit (8 elements: 4 pairs) of one row, looks its
// cosines up once and walks over the heads, which all turn by the same angles; the next two heads are on their way
// while two are worked on, and 64 registers leave room for 32 warps per SM.  lph lanes make up a head, for the sum of
// squares of its norm; rows of 32 / lph tokens share a warp, so heads of 72 elements leave few lanes idle.
// Measured on 230400 rows of 2 x 5 heads of 64, bf16, 590 MB: 97 us (6.1 TB/s) without and 125 us (4.7) with head
// norms, whose sums and square roots are what a warp then waits for; fp32, 1180 MB: 182 us (6.5 TB/s) and 203 (5.8), though
// its pairs in halves do not fit into 64 registers (32 and 128 bytes spilled).
#include <string.h>

#include "rows.cuh"

namespace oc {

static constexpr int ROPE_WARPS = 4;
static constexpr int ROPE_CTAS = 8;              // of them on an SM
static constexpr int ROPE_HEADS = 4;             // heads that a thread has at least, where rows are few

struct RopeParams {
    const void* in[2]; void* out[2]; const float* w[2];                     // q, k
    long long in_row[2], in_head[2], out_batch[2], out_row[2], out_head[2]; // elements
    int heads[2];
    const float2* table; const int32_t* idx; const int32_t* pos;
    uint32_t n_rows;
    FastDiv rows_per_batch, unit_rows, grid, height, width;                  // grid: tokens of all axes
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
template <int DT, int W> __device__ __forceinline__ void rope_widen(const RopeRaw<W * (DT == OC_DTYPE_BF16 ? 2 : 4)>& r, f32x2* f) {
    if constexpr (W == 1) f[0] = DT == OC_DTYPE_F32 ? f2_bits(r.v[0], 0u) : f2_bits(r.v[0] << 16, 0u);
    else
#pragma unroll
        for (int i = 0; i < W / 2; ++i) f[i] = DT == OC_DTYPE_F32 ? f2_bits(r.v[2 * i], r.v[2 * i + 1]) : f2_bits(r.v[i] << 16, r.v[i] & 0xFFFF0000u);
}
template <int DT, int W> __device__ __forceinline__ RopeRaw<W * (DT == OC_DTYPE_BF16 ? 2 : 4)> rope_round(const f32x2* f) {
    RopeRaw<W * (DT == OC_DTYPE_BF16 ? 2 : 4)> r;
#pragma unroll
    for (int i = 0; i < (W + 1) / 2; ++i) {
        if (DT == OC_DTYPE_BF16) r.v[i] = pack_bf16x2(f[i]);
        else { r.v[2 * i] = __float_as_uint(f2_lo(f[i])); if (W > 1) r.v[2 * i + 1] = __float_as_uint(f2_hi(f[i])); }
    }
    return r;
}

// 1 / sqrt(x): the hardware's approximation (good to 2 ulp) and one step of Newton's method on 1/r^2 - x, which
// takes the place of an IEEE square root and division at a quarter of their instructions.
__device__ __forceinline__ float inv_sqrt(float x) {
    const float r = rsqrtf(x), e = fmaf(-x * r, r, 1.0f);
    return x < __int_as_float(0x7F800000) ? fmaf(0.5f * r, e, r) : r;
}

// HALVES: a unit is W pairs, first members in one vector and second members in another; two neighbouring pairs
// share each packed operation.  ADJACENT: a unit is one vector of W elements, W / 2 pairs, the two members of a pair
// sharing each packed operation.
template <int DT, int HALVES, int W, int UPL, bool NORM>
__global__ void __launch_bounds__(ROPE_WARPS * 32, UPL == 1 ? ROPE_CTAS : 1)
rope_kernel(const __grid_constant__ RopeParams P) {
    constexpr int VECS = HALVES ? 2 : 1, NP = HALVES ? W : W / 2, EB = DT == OC_DTYPE_BF16 ? 2 : 4, VB = W * EB;
    constexpr int NW = (W + 1) / 2;                                          // packed words of a vector
    const int lane = threadIdx.x & 31, sub = lane / P.lph, u0 = lane - sub * P.lph;
    pdl_enter();
    const uint32_t row = (blockIdx.x * ROPE_WARPS + (threadIdx.x >> 5)) * (uint32_t)P.rpw + sub;
    const bool there = sub < P.rpw && row < P.n_rows;                        // (rows past the end run along for the shuffles)
    bool in = there;                                                         // whether the row is written, too
    // where the unit's vectors lie in a head
    int off[UPL][VECS];
    bool have[UPL][VECS], rot[UPL];
#pragma unroll
    for (int k = 0; k < UPL; ++k) {
        const int u = u0 + k * P.lph;
        rot[k] = u < P.units_rot;
        if (HALVES) {
            off[k][0] = rot[k] ? W * u : 2 * P.P + 2 * W * (u - P.units_rot);
            off[k][VECS - 1] = rot[k] ? P.P + W * u : off[k][0] + W;
        } else {
            off[k][0] = W * u;
        }
#pragma unroll
        for (int v = 0; v < VECS; ++v) have[k][v] = there && u < P.units && off[k][v] < P.D;
    }
    // This thread's heads, q and then k, as one sequence; those of the next two are on their way while two are
    // worked on.
    const uint32_t batch = there ? P.rows_per_batch.div(row) : 0, in_batch = there ? row - batch * P.rows_per_batch.d : 0;
    const int first = blockIdx.y * P.heads_per_cta, n = min(P.heads_per_cta, P.heads[0] + P.heads[1] - first);
    const int n_q = min(max(P.heads[0] - first, 0), n);                      // how many of them are q's
    const int q0 = min(first, P.heads[0]), k0 = max(first - P.heads[0], 0);
    const long long r64 = there ? row : 0;
    // (a vector that is not there is never loaded: its zeros stay)
    struct Raw { RopeRaw<VB> v[UPL][VECS]; };
    Raw a0 = {}, a1 = {}, b0 = {}, b1 = {};
    const uint8_t* src = n_q > 0 ? (const uint8_t*)P.in[0] + (r64 * P.in_row[0] + q0 * P.in_head[0] + off[0][0]) * EB
                                 : (const uint8_t*)P.in[1] + (r64 * P.in_row[1] + k0 * P.in_head[1] + off[0][0]) * EB;
    uint8_t* dst = n_q > 0 ? (uint8_t*)P.out[0] + ((long long)batch * P.out_batch[0] + (long long)in_batch * P.out_row[0] + q0 * P.out_head[0] + off[0][0]) * EB
                           : (uint8_t*)P.out[1] + ((long long)batch * P.out_batch[1] + (long long)in_batch * P.out_row[1] + k0 * P.out_head[1] + off[0][0]) * EB;
    long long src_step = (n_q > 0 ? P.in_head[0] : P.in_head[1]) * EB, dst_step = (n_q > 0 ? P.out_head[0] : P.out_head[1]) * EB;
    auto load = [&](int i, Raw& raw) {                                       // heads in order: i = 0, 1, 2, ...
        if (i >= n) return;
        if (i == n_q && i > 0) {
            src = (const uint8_t*)P.in[1] + (r64 * P.in_row[1] + off[0][0]) * EB;
            src_step = P.in_head[1] * EB;
        }
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int v = 0; v < VECS; ++v)
                if (have[k][v]) raw.v[k][v] = rope_load<VB>(src + (off[k][v] - off[0][0]) * EB);
        src += src_step;
    };
    load(0, a0); load(1, a1);                                                // (on their way while the positions are looked up)

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
            uint32_t unit = P.unit_rows.div(row);
            const uint32_t rest = row - unit * P.unit_rows.d;
            if (P.idx) {
                const int i = __ldg(P.idx + unit);
                in = i >= 0;                                                 // the unused tail of a kept list
                unit = (uint32_t)i;
            }
            if (in) {
                const uint64_t token = (uint64_t)unit * P.unit_rows.d + rest;
                uint32_t r = token < 0x80000000ull ? (uint32_t)token - P.grid.div((uint32_t)token) * P.grid.d : (uint32_t)(token % P.grid.d);
                const uint32_t y = P.width.div(r);
                at[2] = r - y * P.width.d;
                at[0] = P.height.div(y); at[1] = y - at[0] * P.height.d;
            }
        }
    }
    // HALVES  x' = x c + y ns, y' = y c + x sn  (two pairs at a time);  ADJACENT  (x', y') = (x, y) c + (y, x) (-s, s)
    constexpr int NC = HALVES ? NW : NP;
    f32x2 c[UPL][NC], sn[UPL][NC], ns[UPL][HALVES ? NC : 1];
#pragma unroll
    for (int k = 0; k < UPL; ++k) {
        float co[NP], si[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p) { co[p] = 1.0f; si[p] = 0.0f; }
        if (rot[k] && in) {
            // pairs NP u .. NP u + NP - 1: mostly of one axis, whose line of the table then has them side by side
            const int j0 = NP * (u0 + k * P.lph), j1 = j0 + NP - 1, s1 = P.pairs[0], s2 = s1 + P.pairs[1];
            const int a = j0 < s1 ? 0 : (j0 < s2 ? 1 : 2), a1 = j1 < s1 ? 0 : (j1 < s2 ? 1 : 2);
            const int start = a == 0 ? 0 : (a == 1 ? s1 : s2), pos = a == 0 ? at[0] : (a == 1 ? at[1] : at[2]);
            const float2* line = P.table + P.axis_base[a] + (long long)pos * P.pairs[a] + (j0 - start);
            if (a == a1 && NP > 1 && ((uintptr_t)line & 15u) == 0) {
#pragma unroll
                for (int p = 0; p + 1 < NP; p += 2) {
                    const float4 t = __ldg((const float4*)(line + p));
                    co[p] = t.x; si[p] = P.sign * t.y; co[p + 1] = t.z; si[p + 1] = P.sign * t.w;
                }
            } else {
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int j = j0 + p, b = j < s1 ? 0 : (j < s2 ? 1 : 2), first = b == 0 ? 0 : (b == 1 ? s1 : s2);
                    const int line_b = b == 0 ? at[0] : (b == 1 ? at[1] : at[2]);
                    const float2 t = __ldg(P.table + P.axis_base[b] + (long long)line_b * P.pairs[b] + (j - first));
                    co[p] = t.x; si[p] = P.sign * t.y;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            if (HALVES) {
                const int p = 2 * i, q = 2 * i + 1 < NP ? 2 * i + 1 : 2 * i;
                c[k][i] = f2(co[p], co[q]); sn[k][i] = f2(si[p], si[q]); ns[k][i] = f2(-si[p], -si[q]);
            } else {
                c[k][i] = f2(co[i]); sn[k][i] = f2(-si[i], si[i]);
            }
        }
    }

    f32x2 w[UPL][VECS][NORM ? NW : 1] = {};
    auto weights = [&](const float* from) {
        const bool wide = W % 4 == 0 && ((uintptr_t)from & 15u) == 0;
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                if (!have[k][v]) continue;                                   // (multiplies zeros)
                if (wide) {
#pragma unroll
                    for (int i = 0; i + 1 < NW; i += 2) {
                        const float4 a = __ldg((const float4*)(from + off[k][v] + 2 * i));
                        w[k][v][i] = f2(a.x, a.y); w[k][v][i + 1] = f2(a.z, a.w);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < NW; ++i)
                        w[k][v][i] = f2(__ldg(from + off[k][v] + 2 * i), W > 1 ? __ldg(from + off[k][v] + 2 * i + (W > 1 ? 1 : 0)) : 0.0f);
                }
            }
    };
    // 1 / rms of two heads at once: their sums wait for their shuffles together
    auto norms = [&](const Raw& x, const Raw& y, float& rx, float& ry) {
        float qx = 0.0f, qy = 0.0f;
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int v = 0; v < VECS; ++v)
#pragma unroll
                for (int j = 0; j < (VB < 4 ? 1 : VB / 4); ++j) {
                    if (DT == OC_DTYPE_BF16) { Chunk<OC_DTYPE_BF16>::word1(x.v[k][v].v[j], qx); Chunk<OC_DTYPE_BF16>::word1(y.v[k][v].v[j], qy); }
                    else { const float p = __uint_as_float(x.v[k][v].v[j]), r = __uint_as_float(y.v[k][v].v[j]); qx = fmaf(p, p, qx); qy = fmaf(r, r, qy); }
                }
        if (P.lph == 8) {                                                    // heads of 64
#pragma unroll
            for (int d = 4; d; d >>= 1) { qx += __shfl_xor_sync(0xFFFFFFFFu, qx, d); qy += __shfl_xor_sync(0xFFFFFFFFu, qy, d); }
        } else {
            // the upper half of the head's lanes onto the lower one until one is left
            for (int s = P.lph; s > 1;) {
                const int half = (s + 1) >> 1;
                const float ox = __shfl_down_sync(0xFFFFFFFFu, qx, half), oy = __shfl_down_sync(0xFFFFFFFFu, qy, half);
                if (u0 + half < s) { qx += ox; qy += oy; }
                s = half;
            }
            qx = __shfl_sync(0xFFFFFFFFu, qx, sub * P.lph); qy = __shfl_sync(0xFFFFFFFFu, qy, sub * P.lph);
        }
        rx = inv_sqrt(qx * P.inv_d + P.eps); ry = inv_sqrt(qy * P.inv_d + P.eps);
    };
    auto work = [&](int i, const Raw& raw, float rms) {
        if (i >= n) return;
        if (NORM && i == n_q && i > 0) weights(P.w[1]);
        f32x2 f[UPL][VECS][NW];
#pragma unroll
        for (int k = 0; k < UPL; ++k)
#pragma unroll
            for (int v = 0; v < VECS; ++v) rope_widen<DT, W>(raw.v[k][v], f[k][v]);
        if (NORM) {
            const f32x2 rstd = f2(rms);
#pragma unroll
            for (int k = 0; k < UPL; ++k)
#pragma unroll
                for (int v = 0; v < VECS; ++v)
#pragma unroll
                    for (int j = 0; j < NW; ++j) f[k][v][j] = f2_mul(f[k][v][j], f2_mul(rstd, w[k][v][j]));
        }
        if (i == n_q && i > 0) {
            dst = (uint8_t*)P.out[1] + ((long long)batch * P.out_batch[1] + (long long)in_batch * P.out_row[1] + off[0][0]) * EB;
            dst_step = P.out_head[1] * EB;
        }
#pragma unroll
        for (int k = 0; k < UPL; ++k) {
            if (rot[k]) {                                                    // (what passes through keeps its infinities to itself)
#pragma unroll
                for (int j = 0; j < NC; ++j) {
                    const f32x2 x = f[k][0][j];
                    if (HALVES) {
                        const f32x2 y = f[k][VECS - 1][j];
                        f[k][0][j] = f2_fma(y, ns[k][j], f2_mul(x, c[k][j]));
                        f[k][VECS - 1][j] = f2_fma(x, sn[k][j], f2_mul(y, c[k][j]));
                    } else {
                        f[k][0][j] = f2_fma(f2(f2_hi(x), f2_lo(x)), sn[k][j], f2_mul(x, c[k][j]));
                    }
                }
            }
#pragma unroll
            for (int v = 0; v < VECS; ++v)
                if (have[k][v] && in) rope_store<VB>(dst + (off[k][v] - off[0][0]) * EB, rope_round<DT, W>(f[k][v]));
        }
        dst += dst_step;
    };
    if (NORM) weights(n_q > 0 ? P.w[0] : P.w[1]);
    float r0 = 1.0f, r1 = 1.0f;
#pragma unroll 1
    for (int i = 0; i < n; i += 4) {
        load(i + 2, b0); load(i + 3, b1);
        if (NORM) norms(a0, a1, r0, r1);                                     // (of a head past the last: of what is still there, unused)
        work(i, a0, r0); work(i + 1, a1, r1);
        load(i + 4, a0); load(i + 5, a1);
        if (NORM) norms(b0, b1, r0, r1);
        work(i + 2, b0, r0); work(i + 3, b1, r1);
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

// Elements per vector: the widest that pairs, heads, strides and pointers allow, 16 bytes at most, and 8 elements
// per unit (units of 16 bf16 elements need 96 registers, which leaves 20 warps of 32: 95 and 125 us without and with head
// norms on 230400 rows of 2 x 5 heads of 64, against 97 and 125 -- too little for kernels of their own).
int rope_vector(const oc_rope_desc& d, const void* q, const void* q_out, const void* k, const void* k_out) {
    const int eb = d.dtype == OC_DTYPE_BF16 ? 2 : 4;
    const long long rot = (long long)d.axis_dims[0] + d.axis_dims[1] + d.axis_dims[2];
    uint64_t e = (uint64_t)d.head_dim | (uint64_t)(d.pairing == OC_ROPE_HALVES ? rot / 2 : rot);
    const oc_rope_view* views[4] = {&d.q, &d.q_out, &d.k, &d.k_out};
    uint64_t bytes = (uint64_t)(uintptr_t)q | (uint64_t)(uintptr_t)q_out;
    for (int i = 0; i < (k ? 4 : 2); ++i) e |= (uint64_t)views[i]->row_stride | (uint64_t)views[i]->head_stride | (i & 1 ? (uint64_t)views[i]->batch_stride : 0);
    if (k) bytes |= (uint64_t)(uintptr_t)k | (uint64_t)(uintptr_t)k_out;
    int w = d.pairing == OC_ROPE_HALVES ? 4 : 16 / eb;
    while (w > 1 && ((e & (uint64_t)(w - 1)) || (bytes & (uint64_t)(w * eb - 1)))) w >>= 1;
    return (bytes & (uint64_t)(eb - 1)) ? 0 : w;
}

oc_status launch_rope(oc_ctx* ctx, const oc_rope_desc& d, const float* table, const int32_t* idx, const int32_t* pos,
                      const void* q, void* q_out, const float* q_w, const void* k, void* k_out, const float* k_w, cudaStream_t s) {
    const int w = rope_vector(d, q, q_out, k, k_out);
    const bool halves = d.pairing == OC_ROPE_HALVES;
    if (w == 0 || (!halves && w < 2)) return OC_ERR_ALIGNMENT;
    RopeParams P = {};
    P.in[0] = q; P.in[1] = k; P.out[0] = q_out; P.out[1] = k_out; P.w[0] = q_w; P.w[1] = k_w;
    const oc_rope_view* in[2] = {&d.q, &d.k}; const oc_rope_view* out[2] = {&d.q_out, &d.k_out};
    for (int m = 0; m < 2; ++m) {
        P.in_row[m] = in[m]->row_stride; P.in_head[m] = in[m]->head_stride;
        P.out_row[m] = out[m]->row_stride; P.out_head[m] = out[m]->head_stride; P.out_batch[m] = out[m]->batch_stride;
    }
    P.heads[0] = d.q_heads; P.heads[1] = k ? d.k_heads : 0;
    P.table = (const float2*)table; P.idx = idx; P.pos = pos;
    P.n_rows = (uint32_t)d.n_rows; P.rows_per_batch = FastDiv((uint32_t)d.rows_per_batch); P.unit_rows = FastDiv((uint32_t)d.unit_rows);
    P.grid = FastDiv((uint32_t)d.axis_len[0] * (uint32_t)d.axis_len[1] * (uint32_t)d.axis_len[2]);
    P.height = FastDiv((uint32_t)d.axis_len[1]); P.width = FastDiv((uint32_t)d.axis_len[2]);
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
    // Heads per CTA: all of them where the rows fill the device, otherwise as few as keep every CTA resident (one more
    // split than that starts a second round: 5120 rows of 48 heads take 19 us in 2 splits, 15 in 3 and 18 in 4).
    const long long rows_per_cta = (long long)ROPE_WARPS * P.rpw, row_ctas = (d.n_rows + rows_per_cta - 1) / rows_per_cta;
    const int heads = P.heads[0] + P.heads[1];
    const long long resident = (long long)(upl == 1 ? ROPE_CTAS : ROPE_CTAS / 2) * ctx->sm_count;
    int splits = row_ctas < resident ? (int)(resident / row_ctas) : 1;
    const int most = (heads + ROPE_HEADS - 1) / ROPE_HEADS;
    if (splits > most) splits = most;
    P.heads_per_cta = (heads + splits - 1) / splits;
    splits = (heads + P.heads_per_cta - 1) / P.heads_per_cta;
    if (splits > 65535) return OC_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)row_ctas, (unsigned)splits);
    const bool norm = q_w != nullptr;
    LaunchScope scope(ctx, OC_K_ROPE, s);
    if (d.dtype == OC_DTYPE_BF16) {
        if (halves) {
            if (w == 4) launch_rope_as<OC_DTYPE_BF16, 1, 4>(P, upl, norm, grid, s);
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
