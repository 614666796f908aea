// Attention of few rows (a sequence's rows times the heads that share one of the cache are at most 16: single tokens)
// over the paged cache: bound by reading the cache once, so nothing but that is waited for.
// A warp takes 16 keys at a time, straight from the pages into registers, the next ones while these are worked on, and
// multiplies with mma.sync m16n8k16: the 16 rows are all there are, and a 128-row tile of tcgen05 would be staged through
// shared memory for an eighth of its rows.  Where a lane's elements lie is chosen so that all loads are contiguous and as
// wide as rows are aligned; the products' inner indices may be in any order as long as both operands share it:
//     scores   lane (n, c) = (lane / 4, lane % 4) holds of key n E elements from 4 E chunk + E c on; a step of the product takes
//              four of them, from the queries the same ones
//     outputs  lane (n, c) holds of keys 4c .. 4c + 3 the EV elements from EV n on; column n of the product's tile j is element
//              EV n + j, its inner index the keys in the order in which the scores' tiles leave the probabilities
// 8 and 4 bits are widened to bf16 exactly; the scales join the scores and the probabilities.  The warps of a CTA, and the
// CTAs of a cluster, split the keys and join (maximum, sum, output) at the end, the latter through distributed shared memory.
#include <string.h>

#include <algorithm>

#include "attention_tc.cuh"

namespace oc {

static constexpr int AF_WARPS = 8, AF_ROWS = 16, AF_STEP = 16;
static constexpr float AF_LAG = 8.0f;                                        // powers of two that a maximum may lag behind

template <int BYTES> struct AfRaw { uint32_t w[BYTES / 4]; };
template <int BYTES> __device__ __forceinline__ AfRaw<BYTES> af_load(const void* p) {
    AfRaw<BYTES> r;
    if constexpr (BYTES == 16) { const uint4 v = ld_nc_v4(p); r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w; }
    else if constexpr (BYTES == 8) asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(p));
    else asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(r.w[0]) : "l"(p));
    return r;
}
// Whole numbers as bf16 pairs: see the tensor-core kernel's copy of the idea: 128 + the low 7 bits, minus 128 or 256 by the sign bit
__device__ __forceinline__ uint32_t af_sub(uint32_t a, uint32_t b) { uint32_t r; asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
__device__ __forceinline__ uint32_t af_i8_pair(uint32_t bytes) {              // bytes 0 and 2
    return af_sub((bytes & 0x007F007Fu) | 0x43004300u, (bytes & 0x00800080u) | 0x43004300u);
}
// Elements e and e + 1 of a run, as a pair
template <int KT, int BYTES> __device__ __forceinline__ uint32_t af_pair(const AfRaw<BYTES>& r, int e) {
    if (KT == OC_DTYPE_BF16) return r.w[e >> 1];
    if (KT == OC_DTYPE_I8) return af_i8_pair(__byte_perm(r.w[e >> 2], 0u, e & 2 ? 0x4342u : 0x4140u));
    const uint32_t x = (r.w[e >> 3] ^ 0x88888888u) >> (4 * (e & 7));
    return af_sub((x & 0xFu) | (x & 0xF0u) << 12 | 0x43004300u, 0x43084308u);
}
// Element e of two runs, as a pair
template <int KT, int BYTES> __device__ __forceinline__ uint32_t af_across(const AfRaw<BYTES>& a, const AfRaw<BYTES>& b, int e) {
    if (KT == OC_DTYPE_BF16) return __byte_perm(a.w[e >> 1], b.w[e >> 1], e & 1 ? 0x7632u : 0x5410u);
    if (KT == OC_DTYPE_I8) {
        const int s = e & 3;
        return af_i8_pair(__byte_perm(a.w[e >> 2], b.w[e >> 2], (uint32_t)(s | s << 4 | (4 + s) << 8 | (4 + s) << 12)));
    }
    const int s = (e & 7) >> 1;                                              // the byte; its low or high half
    const uint32_t x = __byte_perm(a.w[e >> 3], b.w[e >> 3], (uint32_t)(s | s << 4 | (4 + s) << 8 | (4 + s) << 12)) ^ 0x00880088u;
    if ((e & 1) == 0) return af_sub((x & 0x000F000Fu) | 0x43004300u, 0x43084308u);
    return af_sub(((x >> 4) & 0x000F000Fu) | 0x43004300u, 0x43084308u);
}
__device__ __forceinline__ void af_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float af_max(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float af_exp2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

// KT: type of the cache; E, NC: elements of a lane's run of a key, runs; EV, NP: of its values; ROWS: 8 where no more are used
template <int KT, int E, int NC, int EV, int NP, int ROWS>
__global__ void __launch_bounds__(AF_WARPS * 32)
attention_few_kernel(const __grid_constant__ AttnParams P) {
    constexpr bool quant = KT == OC_DTYPE_I8 || KT == OC_DTYPE_I4;
    constexpr int KB = KT == OC_DTYPE_BF16 ? 2 * E : KT == OC_DTYPE_I8 ? E : E / 2, VB = KT == OC_DTYPE_BF16 ? 2 * EV : KT == OC_DTYPE_I8 ? EV : EV / 2;
    constexpr int STEPS = NC * E / 4, DP = NP * 8 * EV, HALVES = ROWS / 8, NT = NP * EV;       // products of scores; columns; tiles of outputs
    extern __shared__ __align__(16) float af_smem[];                         // [warps][16][DP + 4] outputs, then [warps][16][2] maxima and sums
    __shared__ int s_range[2], s_odd;
    __shared__ float s_join[AF_ROWS][2];
    constexpr int OS = DP + 4;
    float* stats = af_smem + AF_WARPS * ROWS * OS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, c = lane & 3, D = P.pages.D;
    pdl_enter();
    const uint32_t rank = P.split > 1 ? cluster_rank() : 0u;
    const uint32_t problem = blockIdx.x / (uint32_t)P.split;
    const uint32_t seq = problem / (uint32_t)P.pages.heads, head = problem - seq * (uint32_t)P.pages.heads;
    const AttnSeq S = attn_seq(P, seq);
    const int rows = S.n * P.group;
    if (rows <= 0) return;                                                   // (the whole cluster)
    if (threadIdx.x == 0) { s_range[0] = 0x7FFFFFFF; s_range[1] = 0; s_odd = 0; }
    __syncthreads();
    // the rows n and n + 8: what they see
    int lo[HALVES], hi[HALVES];
    bool exists[HALVES];
    int low = 0, high = 0x7FFFFFFF;                                          // keys within are seen by all rows
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        const int r = n + 8 * h;
        lo[h] = hi[h] = 0;
        exists[h] = r < rows && attn_bounds(P, S, seq, r / P.group, lo[h], hi[h]);
        if (exists[h] && lo[h] < hi[h]) {
            if (warp == 0 && c == 0) { atomicMin(&s_range[0], lo[h]); atomicMax(&s_range[1], hi[h]); }
            low = max(low, lo[h]); high = min(high, hi[h]);
        }
    }
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) { low = max(low, __shfl_xor_sync(0xFFFFFFFFu, low, d)); high = min(high, __shfl_xor_sync(0xFFFFFFFFu, high, d)); }
    // queries: elements 4E chunk + E c + 4s .. + 3 of step (chunk, s)
    uint32_t q[STEPS][4];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int d = (s / (E / 4)) * 4 * E + E * c + 4 * (s % (E / 4));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t a = 0, b = 0;
            const int r = n + 8 * h;
            if (h < HALVES && r < rows && d < D) {
                const int i = r / P.group;
                const uint16_t* p = (const uint16_t*)P.q + attn_q_at(P, S, seq, i, (int)head * P.group + (r - i * P.group)) + d;
                if (P.wide_q) { const uint2 v = *(const uint2*)p; a = v.x; b = v.y; }
                else { a = (uint32_t)p[0] | (uint32_t)p[1] << 16; b = (uint32_t)p[2] | (uint32_t)p[3] << 16; }
            }
            q[s][h] = a; q[s][2 + h] = b;
        }
    }
    __syncthreads();
    // this CTA's share of the steps of 16 keys, this warp's every eighth
    int k0 = s_range[0] / AF_STEP, k1 = s_range[1] > 0 ? (s_range[1] + AF_STEP - 1) / AF_STEP : 0;
    if (k1 <= k0) k0 = k1 = 0;
    if (P.split > 1) {
        const int all = k1 - k0, a = (int)((long long)all * rank / P.split), b = (int)((long long)all * (rank + 1) / P.split);
        k1 = k0 + b; k0 += a;
    }
    float m[HALVES], l[HALVES], o[NT][4];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) { m[h] = exists[h] && lo[h] < hi[h] ? -INFINITY : 0.0f; l[h] = 0.0f; }
#pragma unroll
    for (int t = 0; t < NT; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.0f;
    struct Step { AfRaw<KB> k[NC][2]; AfRaw<VB> v[NP][4]; float4 ks, vs; } cur, nxt;
    auto find = [&](int k) -> int {                                          // the pool's vector of a step's first key; -1: no such page
        if (k >= k1) return -1;
        const uint32_t key = (uint32_t)k * AF_STEP, pn = P.pages.page_rows.div(key);
        const int page = kv_page(P.pages, seq, pn);
        return page < 0 ? -1 : (int)(kv_vector(P.pages, page, key - pn * P.pages.page_rows.d) + head * P.pages.page_rows.d);
    };
    const long long row_bytes = KT == OC_DTYPE_BF16 ? 2ll * D : KT == OC_DTYPE_I8 ? D : D / 2;
    const int key_n = 4 * (n >> 1) + (n & 1);                                // key of column n of the first tile of scores; the second's: + 2
    auto load = [&](Step& s, int vec) {
#pragma unroll
        for (int ch = 0; ch < NC; ++ch)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s.k[ch][t] = AfRaw<KB>{};
                if (vec >= 0 && (ch * 4 + c) * E < D) s.k[ch][t] = af_load<KB>((const uint8_t*)P.k_pool + (long long)(vec + key_n + 2 * t) * row_bytes + (ch * 4 + c) * KB);
            }
#pragma unroll
        for (int ps = 0; ps < NP; ++ps)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s.v[ps][i] = AfRaw<VB>{};
                if (vec >= 0 && (ps * 8 + n) * EV < D) s.v[ps][i] = af_load<VB>((const uint8_t*)P.v_pool + (long long)(vec + 4 * c + i) * row_bytes + (ps * 8 + n) * VB);
            }
        if (quant) {
            s.ks = s.vs = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (vec >= 0) { s.ks = __ldg((const float4*)(P.k_scale + vec) + c); s.vs = __ldg((const float4*)(P.v_scale + vec) + c); }
        }
    };
    const float cc = P.scale_log2, lag = AF_LAG / cc;
    int k = k0 + warp, vec_next = find(k + AF_WARPS);
    load(cur, find(k));
    for (; k < k1; k += AF_WARPS) {
        load(nxt, vec_next);
        vec_next = find(k + 2 * AF_WARPS);
        float s[2][4] = {};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            const int e = 4 * (st % (E / 4));
#pragma unroll
            for (int t = 0; t < 2; ++t) af_mma(s[t], q[st], af_pair<KT>(cur.k[st / (E / 4)][t], e), af_pair<KT>(cur.k[st / (E / 4)][t], e + 2));
        }
        const int key0 = k * AF_STEP + 4 * c;                                // this lane's keys: key0 .. key0 + 3, s[i / 2][i % 2 + 2 h] of row n + 8h
        const bool cut = k * AF_STEP < low || (k + 1) * AF_STEP > high;
        const float ks[4] = {cur.ks.x, cur.ks.y, cur.ks.z, cur.ks.w}, vs[4] = {cur.vs.x, cur.vs.y, cur.vs.z, cur.vs.w};
        float x[HALVES][4];
        bool hidden[HALVES][4];
        bool grow = false;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[h][i] = s[i >> 1][(i & 1) + 2 * h];
                if (quant) x[h][i] *= ks[i];
                hidden[h][i] = cut && (key0 + i < lo[h] || key0 + i >= hi[h]);
                if (hidden[h][i]) x[h][i] = -INFINITY;
            }
            const float top = af_max(af_max(x[h][0], x[h][1]), af_max(x[h][2], x[h][3]));
            grow |= !(top <= m[h] + lag) && top != -INFINITY;
        }
        if (__any_sync(0xFFFFFFFFu, grow)) {
            // the rows' new maxima (NaN is passed on to the whole row; that of +infinity makes its exponentials NaN)
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                float top = af_max(af_max(x[h][0], x[h][1]), af_max(x[h][2], x[h][3]));
                top = af_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = af_max(af_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2)), m[h]);
                if (top == INFINITY) top = __int_as_float(0x7FFFFFFF);
                const float corr = top == -INFINITY || m[h] == -INFINITY ? (top == top ? 0.0f : top) : af_exp2((m[h] - top) * cc);
                l[h] *= corr;
#pragma unroll
                for (int t = 0; t < NT; ++t) { o[t][2 * h] *= corr; o[t][2 * h + 1] *= corr; }
                m[h] = top;
            }
        }
        uint32_t p[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            const float shift = m[h] == -INFINITY ? 0.0f : -m[h] * cc;
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[i] = af_exp2(fmaf(x[h][i], cc, shift));
                l[h] += e[i];
                if (quant) e[i] = hidden[h][i] ? 0.0f : e[i] * vs[i];        // (0 times a scale that is no number)
            }
            p[h] = pack_bf16x2(e[0], e[1]); p[2 + h] = pack_bf16x2(e[2], e[3]);
        }
        if (!quant && cut) {                                                 // 0 * NaN would reach rows that do not see it
            bool odd = false;
#pragma unroll
            for (int ps = 0; ps < NP; ++ps)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < VB / 4; ++j) {
                        uint32_t& w = cur.v[ps][i].w[j];
                        const bool a = (w & 0x7F80u) == 0x7F80u, b = (w & 0x7F800000u) == 0x7F800000u;
                        odd |= (a || b) && key0 + i < S.len;
                        w &= (a ? 0u : 0xFFFFu) | (b ? 0u : 0xFFFF0000u);
                    }
            if (odd) s_odd = 1;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) af_mma(o[t], p, af_across<KT>(cur.v[t / EV][0], cur.v[t / EV][1], t % EV), af_across<KT>(cur.v[t / EV][2], cur.v[t / EV][3], t % EV));
        cur = nxt;
    }
    // ---- the warps' results side by side: o[t] holds columns EV * (8 pass + 2c) + j and EV * (8 pass + 2c + 1) + j of rows n and n + 8 ----
    float* mine = af_smem + warp * ROWS * OS;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 1);
        l[h] += __shfl_xor_sync(0xFFFFFFFFu, l[h], 2);
        if (c == 0) { stats[(warp * ROWS + n + 8 * h) * 2] = m[h]; stats[(warp * ROWS + n + 8 * h) * 2 + 1] = l[h]; }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int at = (t / EV) * 8 * EV + t % EV;
            mine[(n + 8 * h) * OS + at + EV * (2 * c)] = o[t][2 * h];
            mine[(n + 8 * h) * OS + at + EV * (2 * c + 1)] = o[t][2 * h + 1];
        }
    }
    __syncthreads();
    const int vecs = D / 4;
    // a row's parts, with their maxima and sums: (maximum, sum, 4 columns)
    auto join = [&](int parts, auto stat, auto part, float& top, float& sum) {
        float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        top = -INFINITY; sum = 0.0f;
        for (int k2 = 0; k2 < parts; ++k2) top = af_max(top, stat(k2, 0));
        for (int k2 = 0; k2 < parts; ++k2) {
            const float x2 = stat(k2, 0);
            if (x2 == -INFINITY) continue;
            const float f = af_exp2((x2 - top) * cc);
            const float4 v = part(k2);
            sum = fmaf(f, stat(k2, 1), sum);
            y.x = fmaf(f, v.x, y.x); y.y = fmaf(f, v.y, y.y); y.z = fmaf(f, v.z, y.z); y.w = fmaf(f, v.w, y.w);
        }
        return y;
    };
    auto store = [&](int r, int d, float4 y, float top, float sum, bool odd) {
        const int i = r / P.group, hq = (int)head * P.group + (r - i * P.group);
        int a, b;
        if (!attn_bounds(P, S, seq, i, a, b)) return;
        const bool some = a < b;
        const float inv = 1.0f / sum;                                        // (all scores -infinity: 0 / 0)
        y = some ? make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (odd && some && !quant) {
            y.x += attn_not_finite<KT>(P, seq, head, a, b, d); y.y += attn_not_finite<KT>(P, seq, head, a, b, d + 1);
            y.z += attn_not_finite<KT>(P, seq, head, a, b, d + 2); y.w += attn_not_finite<KT>(P, seq, head, a, b, d + 3);
        }
        attn_store4<OC_DTYPE_BF16>(P, attn_out_at(P, S, seq, i, hq) + d, y);
        if (P.lse && d == 0) P.lse[(S.row0 + i) * P.q_heads + hq] = some ? top * P.scale + logf(sum) : -INFINITY;
    };
    const int used = min(rows, ROWS);
    if (P.split == 1) {
        for (int it = threadIdx.x; it < used * vecs; it += AF_WARPS * 32) {
            const int r = it / vecs, d = 4 * (it - r * vecs);
            float top, sum;
            const float4 y = join(AF_WARPS, [&](int w, int e) { return stats[(w * ROWS + r) * 2 + e]; },
                                  [&](int w) { return *(const float4*)(af_smem + (w * ROWS + r) * OS + d); }, top, sum);
            store(r, d, y, top, sum, s_odd != 0);
        }
        return;
    }
    // the CTA's warps first (in the place of warp 0's part: a thread reads and writes the same elements), then the cluster's CTAs
    for (int it = threadIdx.x; it < used * vecs; it += AF_WARPS * 32) {
        const int r = it / vecs, d = 4 * (it - r * vecs);
        float top, sum;
        const float4 y = join(AF_WARPS, [&](int w, int e) { return stats[(w * ROWS + r) * 2 + e]; },
                              [&](int w) { return *(const float4*)(af_smem + (w * ROWS + r) * OS + d); }, top, sum);
        *(float4*)(af_smem + r * OS + d) = y;
        if (d == 0) { s_join[r][0] = top; s_join[r][1] = sum; }
    }
    cluster_sync();
    int odd = 0;
    for (int k2 = 0; k2 < P.split; ++k2) {
        int w;
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(w) : "r"(cluster_map(smem_u32(&s_odd), (uint32_t)k2)) : "memory");
        odd |= w;
    }
    const uint32_t part_at = smem_u32(af_smem), join_at = smem_u32(&s_join[0][0]);
    for (int it = (int)rank * AF_WARPS * 32 + threadIdx.x; it < used * vecs; it += P.split * AF_WARPS * 32) {
        const int r = it / vecs, d = 4 * (it - r * vecs);
        float top, sum;
        const float4 y = join(P.split, [&](int w, int e) { return cluster_ld(cluster_map(join_at, (uint32_t)w) + 8u * r + 4u * e); },
                              [&](int w) { return cluster_ld4(cluster_map(part_at, (uint32_t)w) + (uint32_t)(r * OS + d) * 4u); }, top, sum);
        store(r, d, y, top, sum, odd != 0);
    }
    cluster_sync();                                                          // nobody reads a retired CTA's memory
}

// ---- host side -------------------------------------------------------------------------------------
template <int KT, int E, int NC, int EV, int NP, int ROWS>
static oc_status launch_few_as(oc_ctx* ctx, AttnParams& P, cudaStream_t s) {
    constexpr int DP = NP * 8 * EV, SMEM = AF_WARPS * ROWS * (DP + 4 + 2) * 4;
    auto* kernel = attention_few_kernel<KT, E, NC, EV, NP, ROWS>;
    static PerDeviceOnce once;                       // (the context's device is current here)
    if (!once.ensure(ctx->device, [&] {
            const bool ok = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) == cudaSuccess &&
                            cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
            if (!ok) cudaGetLastError();
            return ok;
        })) return OC_ERR_CUDA;
    const uint64_t problems = (uint64_t)P.n_seqs * (uint64_t)P.pages.heads;
    if (problems * ATT_SPLIT_MAX > 0x7FFFFFFFull) return OC_ERR_UNSUPPORTED;
    // CTAs enough for the device several times over (sequences differ in length), each with two steps for every warp at least
    int split = 1;
    while (split < ATT_SPLIT_MAX && problems * split < 4ull * ctx->sm_count && (uint64_t)P.pages.seq_rows >= (uint64_t)split * 2 * 2 * AF_WARPS * AF_STEP) split *= 2;
    P.split = split;
    LaunchScope scope(ctx, OC_K_ATTENTION, s);
    PdlLaunch l(dim3((unsigned)(problems * split)), dim3(AF_WARPS * 32), SMEM, s, (unsigned)split);
    cudaLaunchKernelEx(&l.cfg, kernel, (const AttnParams&)P);
    return last_launch_status();
}
template <int KT, int E, int NC, int EV, int NP>
static oc_status launch_few_rows(oc_ctx* ctx, AttnParams& P, cudaStream_t s) {
    return (uint64_t)P.rows_per_batch * (uint64_t)P.group <= 8 ? launch_few_as<KT, E, NC, EV, NP, 8>(ctx, P, s) : launch_few_as<KT, E, NC, EV, NP, 16>(ctx, P, s);
}

bool attention_few_rows(const AttnParams& P) { return (uint64_t)P.rows_per_batch * (uint64_t)P.group <= AF_ROWS; }

oc_status launch_attention_few(oc_ctx* ctx, AttnParams& P, int kv_dtype, cudaStream_t s) {
    const int D = P.pages.D;
    if (kv_dtype == OC_DTYPE_BF16) return D <= 64 ? launch_few_rows<OC_DTYPE_BF16, 8, 2, 8, 1>(ctx, P, s) : launch_few_rows<OC_DTYPE_BF16, 8, 4, 8, 2>(ctx, P, s);
    // runs as wide as the rows' alignment allows (rows of whole numbers are D or D / 2 bytes long), without leaving lanes idle
    if (kv_dtype == OC_DTYPE_I8) {
        if (D == 64) return launch_few_rows<OC_DTYPE_I8, 16, 1, 8, 1>(ctx, P, s);
        if (D > 64 && D % 16 == 0) return launch_few_rows<OC_DTYPE_I8, 16, 2, 16, 1>(ctx, P, s);
        return D <= 64 ? launch_few_rows<OC_DTYPE_I8, 8, 2, 8, 1>(ctx, P, s) : launch_few_rows<OC_DTYPE_I8, 8, 4, 8, 2>(ctx, P, s);
    }
    if (D == 64) return launch_few_rows<OC_DTYPE_I4, 16, 1, 8, 1>(ctx, P, s);
    if (D > 64 && D % 32 == 0) return launch_few_rows<OC_DTYPE_I4, 32, 1, 16, 1>(ctx, P, s);
    if (D > 64 && D % 16 == 0) return launch_few_rows<OC_DTYPE_I4, 16, 2, 16, 1>(ctx, P, s);
    return D <= 64 ? launch_few_rows<OC_DTYPE_I4, 8, 2, 8, 1>(ctx, P, s) : launch_few_rows<OC_DTYPE_I4, 8, 4, 8, 2>(ctx, P, s);
}

}  // namespace oc
