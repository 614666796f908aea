// Attention of few rows (a sequence's rows times the heads that share one of the cache are at most 16: single tokens)
// over the paged cache: bound by reading the cache once, so nothing but that is waited for.
// A warp takes 16 keys at a time, straight from the pages into registers, the next keys on their way as soon as these have
// been multiplied, the next values likewise, and multiplies with mma.sync m16n8k16: S^T = K Q^T and O^T = V^T P^T, so that the
// few rows are the short side of the products (a 128-row tile of tcgen05 would be empty but for them, and go through shared
// memory).  Where a lane's elements lie is chosen so that all loads are contiguous and as wide as rows are aligned; the
// products' indices may be in any order as long as all operands share it:
//     scores   lane (n, c) = (lane / 4, lane % 4) holds of the keys of its two rows n, n + 8 of the product the E elements from
//              4 E chunk + E c on; a step of the product takes four of them, from the queries the same ones
//     outputs  lane (n, c) holds of the keys of columns 2c, 2c + 1, 2c + 8, 2c + 9 the EV elements from EV n on; rows n and n + 8 of
//              tile j are elements EV n + 2j and the next.  P^T comes out of the scores by transposing 8 x 8 pieces (movmatrix)
// Measured in 8 bits on 286000 keys of 8 heads of 128, 4 heads to a key: 604 MB in 166 us (3.64 TB/s), issuing 91 million
// instructions, 82 us of every scheduler's time, most of them for the widening; the rest is waiting with 16 warps on an SM.
// 8 and 4 bits are widened to bf16 exactly; the scales join the scores and the probabilities, which are rounded to bf16 for the
// second product (their sum is of the unrounded ones).  The warps of a CTA, and the
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
// Which elements of a run of 8 make up pair i: neighbours, or in 4 bits those that one mask cuts out of a word.
template <int KT> __device__ __forceinline__ constexpr int af_first(int i) { return KT == OC_DTYPE_I4 ? i : 2 * i; }
template <int KT> __device__ __forceinline__ constexpr int af_second(int i) { return KT == OC_DTYPE_I4 ? i + 4 : 2 * i + 1; }
// (sign bits flipped: whole numbers with an offset)
template <int KT, int BYTES> __device__ __forceinline__ void af_flip(AfRaw<BYTES>& r) {
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) r.w[i] ^= KT == OC_DTYPE_I8 ? 0x80808080u : KT == OC_DTYPE_I4 ? 0x88888888u : 0u;
}
// Pair i of a run
template <int KT, int BYTES> __device__ __forceinline__ uint32_t af_pair(const AfRaw<BYTES>& r, int i) {
    if (KT == OC_DTYPE_BF16) return r.w[i];
    if (KT == OC_DTYPE_I8) return attn_i8_pair(__byte_perm(r.w[i >> 1], 0x43434343u, i & 1 ? 0x4342u : 0x4140u));
    return attn_i4_pair(r.w[i >> 2] >> (4 * (i & 3)));
}
// Element e of two runs
template <int KT, int BYTES> __device__ __forceinline__ uint32_t af_across(const AfRaw<BYTES>& a, const AfRaw<BYTES>& b, int e) {
    if (KT == OC_DTYPE_BF16) return __byte_perm(a.w[e >> 1], b.w[e >> 1], e & 1 ? 0x7632u : 0x5410u);
    const int s = KT == OC_DTYPE_I8 ? e & 3 : (e & 7) >> 1;                  // the byte
    const uint32_t x = __byte_perm(KT == OC_DTYPE_I8 ? a.w[e >> 2] : a.w[e >> 3], KT == OC_DTYPE_I8 ? b.w[e >> 2] : b.w[e >> 3],
                                   (uint32_t)(s | s << 4 | (4 + s) << 8 | (4 + s) << 12));
    if (KT == OC_DTYPE_I8) return attn_i8_pair((x & 0x00FF00FFu) | 0x43004300u);
    return attn_i4_pair(e & 1 ? x >> 4 : x);
}
__device__ __forceinline__ void af_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float af_max(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float af_exp2(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

__device__ __forceinline__ uint32_t af_transpose(uint32_t a) { uint32_t r; asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a)); return r; }

// KT: type of the cache; E, NC: elements of a lane's run of a key, runs; EV, NP: of its values; ROWS: 8 where no more are used
template <int KT, int E, int NC, int EV, int NP, int ROWS>
__global__ void __launch_bounds__(AF_WARPS * 32, KT != OC_DTYPE_BF16 && ROWS == 8 ? 2 : 1)
attention_few_kernel(const __grid_constant__ AttnParams P) {
    constexpr bool quant = KT == OC_DTYPE_I8 || KT == OC_DTYPE_I4;
    constexpr int KB = KT == OC_DTYPE_BF16 ? 2 * E : KT == OC_DTYPE_I8 ? E : E / 2, VB = KT == OC_DTYPE_BF16 ? 2 * EV : KT == OC_DTYPE_I8 ? EV : EV / 2;
    constexpr int STEPS = NC * E / 4, DP = NP * 8 * EV, RT = ROWS / 8, OT = NP * EV / 2;       // products of scores; columns; tiles of rows, of outputs
    extern __shared__ __align__(16) float af_smem[];                         // [warps][rows][DP + 4] outputs, then [warps][rows][2] maxima and sums
    __shared__ int s_bad[ATT_BAD];                                                 // keys with values that are no numbers
    __shared__ float s_join[AF_ROWS][2];
    constexpr int OS = DP + 4;
    float* stats = af_smem + AF_WARPS * ROWS * OS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, c = lane & 3, D = P.pages.D;
    pdl_enter();
    const uint32_t rank = P.split > 1 ? cluster_rank() : 0u;
    const uint32_t problem = blockIdx.x / (uint32_t)P.split;
    uint32_t seq = problem / (uint32_t)P.pages.heads;
    const uint32_t head = problem - seq * (uint32_t)P.pages.heads;
    if (P.long_first) {                                                      // the seq-th longest sequence (at most as many as threads)
        __shared__ int s_len[AF_WARPS * 32], s_seq;
        const int t = threadIdx.x, ns = (int)P.n_seqs;
        if (t < ns) s_len[t] = __ldg(P.kv_len + t);
        __syncthreads();
        if (t < ns) {
            const int mine = s_len[t];
            uint32_t before = 0;
            for (int i = 0; i < ns; ++i) before += s_len[i] > mine || (s_len[i] == mine && i < t);
            if (before == seq) s_seq = t;
        }
        __syncthreads();
        seq = (uint32_t)s_seq;
    }
    const AttnSeq S = attn_seq(P, seq);
    const int rows = S.n * P.group;
    if (rows <= 0) return;                                                   // (the whole cluster)
    // what the rows 8 rt + 2c and the next see
    int lo[RT][2], hi[RT][2];
    float m[RT][2], l[RT][2], o[RT][OT][4];
    int low = 0, high = 0x7FFFFFFF, from = 0x7FFFFFFF, to = 0;               // keys [low, high) are seen by all rows, [from, to) by any
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * rt + 2 * c + e;
            int a = 0, b = 0;
            const bool some = r < rows && attn_bounds(P, S, seq, r / P.group, a, b) && a < b;
            if (some) { low = max(low, a); high = min(high, b); from = min(from, a); to = max(to, b); }
            lo[rt][e] = some ? a : 0; hi[rt][e] = some ? b : 0;
            m[rt][e] = some ? -INFINITY : 0.0f; l[rt][e] = 0.0f;
        }
#pragma unroll
        for (int t = 0; t < OT; ++t) o[rt][t][0] = o[rt][t][1] = o[rt][t][2] = o[rt][t][3] = 0.0f;
    }
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        low = max(low, __shfl_xor_sync(0xFFFFFFFFu, low, d)); high = min(high, __shfl_xor_sync(0xFFFFFFFFu, high, d));
        from = min(from, __shfl_xor_sync(0xFFFFFFFFu, from, d)); to = max(to, __shfl_xor_sync(0xFFFFFFFFu, to, d));
    }
    if (threadIdx.x == 0) attn_bad_none(s_bad);
    // this CTA's share of the steps of 16 keys, this warp's every eighth
    int k0 = from / AF_STEP, k1 = to > 0 ? (to + AF_STEP - 1) / AF_STEP : 0;
    if (k1 <= k0) k0 = k1 = 0;
    if (P.split > 1) {
        const int all = k1 - k0, a = (int)((long long)all * rank / P.split), b = (int)((long long)all * (rank + 1) / P.split);
        k1 = k0 + b; k0 += a;
    }
    auto find = [&](int k) -> int {                                          // the pool's vector of a step's first key; -1: no such page
        if (k >= k1) return -1;
        const uint32_t key = (uint32_t)k * AF_STEP, pn = P.pages.page_rows.div(key);
        const int page = kv_page(P.pages, seq, pn);
        return page < 0 ? -1 : (int)(kv_vector(P.pages, page, key - pn * P.pages.page_rows.d) + head * P.pages.page_rows.d);
    };
    const long long row_bytes = KT == OC_DTYPE_BF16 ? 2ll * D : KT == OC_DTYPE_I8 ? D : D / 2;
    const int key_n = 4 * (n >> 1) + (n & 1);                                // key of row n of the scores' product; row n + 8's: + 2
    AfRaw<KB> rk[NC][2];
    AfRaw<VB> rv[NP][4];
    float ks[2] = {0.0f, 0.0f}, vs[2] = {0.0f, 0.0f};
    // (a lane's runs behind the end of a row are never loaded: their zeros stay)
    const uint8_t* kp = (const uint8_t*)P.k_pool + key_n * row_bytes + c * KB;
    const uint8_t* vp = (const uint8_t*)P.v_pool + 4 * c * row_bytes + n * VB;
#pragma unroll
    for (int ch = 0; ch < NC; ++ch) rk[ch][0] = rk[ch][1] = AfRaw<KB>{};
#pragma unroll
    for (int ps = 0; ps < NP; ++ps) rv[ps][0] = rv[ps][1] = rv[ps][2] = rv[ps][3] = AfRaw<VB>{};
    auto load_k = [&](int vec) {
        if (vec >= 0) {
            const uint8_t* at = kp + (long long)vec * row_bytes;
#pragma unroll
            for (int ch = 0; ch < NC; ++ch)
                if ((ch * 4 + c) * E < D) { rk[ch][0] = af_load<KB>(at + ch * 4 * KB); rk[ch][1] = af_load<KB>(at + 2 * row_bytes + ch * 4 * KB); }
            if (quant) { ks[0] = __ldg(P.k_scale + vec + key_n); ks[1] = __ldg(P.k_scale + vec + key_n + 2); }
        } else {                                                             // a page that is not there, or nothing left
            ks[0] = ks[1] = 0.0f;
            if (!quant)
#pragma unroll
                for (int ch = 0; ch < NC; ++ch) rk[ch][0] = rk[ch][1] = AfRaw<KB>{};
        }
    };
    auto load_v = [&](int vec) {
        if (vec >= 0) {
            const uint8_t* at = vp + (long long)vec * row_bytes;
#pragma unroll
            for (int i = 0; i < 4; ++i)                                      // keys 4c + i: columns 2c, 2c + 1, 2c + 8, 2c + 9
#pragma unroll
                for (int ps = 0; ps < NP; ++ps)
                    if ((ps * 8 + n) * EV < D) rv[ps][i] = af_load<VB>(at + i * row_bytes + ps * 8 * VB);
            if (quant) { vs[0] = __ldg(P.v_scale + vec + key_n); vs[1] = __ldg(P.v_scale + vec + key_n + 2); }
        } else {
            vs[0] = vs[1] = 0.0f;
            if (!quant)
#pragma unroll
                for (int ps = 0; ps < NP; ++ps) rv[ps][0] = rv[ps][1] = rv[ps][2] = rv[ps][3] = AfRaw<VB>{};
        }
    };
    int k = k0 + warp, vec = find(k);
    load_k(vec);
    load_v(vec);
    vec = find(k + AF_WARPS);
    // queries: of row n, elements 4E chunk + E c + 4s .. + 3 of step (chunk, s)
    uint32_t q[RT][STEPS][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int r = 8 * rt + n, i = r / P.group;
        const uint16_t* p = (const uint16_t*)P.q + (r < rows ? attn_q_at(P, S, seq, i, (int)head * P.group + (r - i * P.group)) : 0);
#pragma unroll
        for (int s = 0; s < STEPS; s += 2) {                                 // 8 elements: pairs 2s .. 2s + 3 of the lane's run
            const int d = (s / (E / 4)) * 4 * E + E * c + 4 * (s % (E / 4));
            uint16_t e[8] = {};
            if (r < rows && d < D) {
                if (P.wide_q) { const uint4 v = ld_v4(p + d); memcpy(e, &v, 16); }
                else
#pragma unroll
                    for (int i2 = 0; i2 < 8; ++i2) e[i2] = p[d + i2];
            }
#pragma unroll
            for (int i2 = 0; i2 < 4; ++i2) q[rt][s + (i2 >> 1)][i2 & 1] = (uint32_t)e[af_first<KT>(i2)] | (uint32_t)e[af_second<KT>(i2)] << 16;
        }
    }
    __syncthreads();                                                         // (s_bad)
    const float cc = P.scale_log2, lag = AF_LAG / cc;
    for (; k < k1; k += AF_WARPS) {
        if (quant)
#pragma unroll
            for (int ch = 0; ch < NC; ++ch) { af_flip<KT>(rk[ch][0]); af_flip<KT>(rk[ch][1]); }
        float x[RT][4];                                                      // [0], [1]: key n with the lane's two rows, [2], [3]: key n + 8
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) x[rt][0] = x[rt][1] = x[rt][2] = x[rt][3] = 0.0f;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            const int i = 2 * (st % (E / 4));
            const AfRaw<KB>&r0 = rk[st / (E / 4)][0], &r1 = rk[st / (E / 4)][1];
            const uint32_t a[4] = {af_pair<KT>(r0, i), af_pair<KT>(r1, i), af_pair<KT>(r0, i + 1), af_pair<KT>(r1, i + 1)};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) af_mma(x[rt], a, q[rt][st][0], q[rt][st][1]);
        }
        if (quant)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) { x[rt][0] *= ks[0]; x[rt][1] *= ks[0]; x[rt][2] *= ks[1]; x[rt][3] *= ks[1]; }
        load_k(vec);
        const int vec_v = vec;
        vec = find(k + 2 * AF_WARPS);
        const int key0 = k * AF_STEP;
        const bool cut = key0 < low || key0 + AF_STEP > high;
        bool grow = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (cut) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = key0 + key_n + 2 * (i >> 1);
                    if (key < lo[rt][i & 1] || key >= hi[rt][i & 1]) x[rt][i] = -INFINITY;
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float top = af_max(x[rt][e], x[rt][2 + e]);
                grow |= !(top <= m[rt][e] + lag) && top != -INFINITY;
            }
        }
        if (__any_sync(0xFFFFFFFFu, grow)) {
            // the rows' new maxima (NaN is passed on to the whole row; that of +infinity makes its exponentials NaN)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = af_max(x[rt][e], x[rt][2 + e]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top = af_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                    top = af_max(top, m[rt][e]);
                    if (top == INFINITY) top = __int_as_float(0x7FFFFFFF);
                    const float corr = top == -INFINITY || m[rt][e] == -INFINITY ? (top == top ? 0.0f : top) : af_exp2((m[rt][e] - top) * cc);
                    l[rt][e] *= corr;
#pragma unroll
                    for (int t = 0; t < OT; ++t) { o[rt][t][e] *= corr; o[rt][t][2 + e] *= corr; }
                    m[rt][e] = top;
                }
        }
        // values that are no numbers: 0 * NaN would reach rows that do not see them
        if (quant) {
            if (__any_sync(0xFFFFFFFFu, fmaf(vs[0], 0.0f, vs[1] * 0.0f) != 0.0f))
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (!isfinite(vs[i])) { vs[i] = 0.0f; if (key0 + key_n + 2 * i < S.len) attn_bad_key(P, s_bad, key0 + key_n + 2 * i); }
        } else {
            uint32_t zero[4] = {};                                           // (four sums: one would wait for itself)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int ps = 0; ps < NP; ++ps)
#pragma unroll
                    for (int j = 0; j < VB / 4; ++j) zero[i] = attn_zero2(zero[i], rv[ps][i].w[j]);
            if (attn_bad2(zero[0] | zero[1] | zero[2] | zero[3])) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    bool odd = false;
#pragma unroll
                    for (int ps = 0; ps < NP; ++ps)
#pragma unroll
                        for (int j = 0; j < VB / 4; ++j) {
                            uint32_t& w = rv[ps][i].w[j];
                            const bool a = (w & 0x7F80u) == 0x7F80u, b = (w & 0x7F800000u) == 0x7F800000u;
                            odd |= a || b;
                            w &= (a ? 0u : 0xFFFFu) | (b ? 0u : 0xFFFF0000u);
                        }
                    if (odd && key0 + 4 * c + i < S.len) attn_bad_key(P, s_bad, key0 + 4 * c + i);
                }
            }
            __syncwarp();
        }
        uint32_t p[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float mm = m[rt][i & 1];
                e[i] = af_exp2(fmaf(x[rt][i], cc, mm == -INFINITY ? 0.0f : -mm * cc));
                l[rt][i & 1] += e[i];
                if (quant) e[i] *= vs[i >> 1];
            }
            p[rt][0] = af_transpose(pack_bf16x2(e[0], e[1])); p[rt][1] = af_transpose(pack_bf16x2(e[2], e[3]));
        }
        if (quant)
#pragma unroll
            for (int ps = 0; ps < NP; ++ps) { af_flip<KT>(rv[ps][0]); af_flip<KT>(rv[ps][1]); af_flip<KT>(rv[ps][2]); af_flip<KT>(rv[ps][3]); }
#pragma unroll
        for (int t = 0; t < OT; ++t) {
            const AfRaw<VB>* r = rv[2 * t / EV];
            const int e = 2 * t % EV;
            const uint32_t a[4] = {af_across<KT>(r[0], r[1], e), af_across<KT>(r[0], r[1], e + 1), af_across<KT>(r[2], r[3], e), af_across<KT>(r[2], r[3], e + 1)};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) af_mma(o[rt][t], a, p[rt][0], p[rt][1]);
        }
        load_v(vec_v);
    }
    // ---- the warps' results side by side ----
    float* mine = af_smem + warp * ROWS * OS;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * rt + 2 * c + e;
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[rt][e] += __shfl_xor_sync(0xFFFFFFFFu, l[rt][e], d);
            if (n == 0) { stats[(warp * ROWS + r) * 2] = m[rt][e]; stats[(warp * ROWS + r) * 2 + 1] = l[rt][e]; }
#pragma unroll
            for (int t = 0; t < OT; ++t)
                *(float2*)(mine + r * OS + (2 * t / EV) * 8 * EV + EV * n + 2 * t % EV) = make_float2(o[rt][t][e], o[rt][t][2 + e]);
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
    int bad0 = 0, bad1 = 0;
    auto store = [&](int r, int d, float4 y, float top, float sum) {
        const int i = r / P.group, hq = (int)head * P.group + (r - i * P.group);
        int a, b;
        if (!attn_bounds(P, S, seq, i, a, b)) return;
        const bool some = a < b;
        const float inv = 1.0f / sum;                                        // (all scores -infinity: 0 / 0)
        y = some ? make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (some) {
            a = max(a, bad0); b = min(b, bad1);
            if (a < b) attn_add4(y, attn_not_finite<KT>(P, s_bad, seq, head, a, b, d));
        }
        attn_store4<OC_DTYPE_BF16>(P, attn_out_at(P, S, seq, i, hq) + d, y);
        if (P.lse && d == 0) P.lse[(S.row0 + i) * P.q_heads + hq] = some ? top * P.scale + logf(sum) : -INFINITY;
    };
    const int used = min(rows, ROWS);
    if (P.split == 1) {
        bad0 = s_bad[0]; bad1 = s_bad[1];
        for (int it = threadIdx.x; it < used * vecs; it += AF_WARPS * 32) {
            const int r = it / vecs, d = 4 * (it - r * vecs);
            float top, sum;
            const float4 y = join(AF_WARPS, [&](int w, int e) { return stats[(w * ROWS + r) * 2 + e]; },
                                  [&](int w) { return *(const float4*)(af_smem + (w * ROWS + r) * OS + d); }, top, sum);
            store(r, d, y, top, sum);
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
    cluster_bad(s_bad, P.split, bad0, bad1);
    const uint32_t part_at = smem_u32(af_smem), join_at = smem_u32(&s_join[0][0]);
    for (int it = (int)rank * AF_WARPS * 32 + threadIdx.x; it < used * vecs; it += P.split * AF_WARPS * 32) {
        const int r = it / vecs, d = 4 * (it - r * vecs);
        float top, sum;
        const float4 y = join(P.split, [&](int w, int e) { return cluster_ld(cluster_map(join_at, (uint32_t)w) + 8u * r + 4u * e); },
                              [&](int w) { return cluster_ld4(cluster_map(part_at, (uint32_t)w) + (uint32_t)(r * OS + d) * 4u); }, top, sum);
        store(r, d, y, top, sum);
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
    // CTAs for twice the device, each with two steps for every warp at least.  16 sequences of up to 32768 tokens, 8 heads of 128 in
    // 8 bits (128 problems): clusters of 1, 2, 4, 8 and 16 CTAs take 431, 318, 185, 193 and 261 us: a cluster waits until an
    // equal number of places is free at once, and its CTAs end together.
    int split = 1;
    while (split < ATT_SPLIT_MAX && problems * split < 2ull * ctx->sm_count && (uint64_t)P.pages.seq_rows >= (uint64_t)split * 2 * 2 * AF_WARPS * AF_STEP) split *= 2;
    P.split = split;
    // (where all CTAs are not resident at once, the long sequences' come first)
    P.long_first = P.kv_len && P.n_seqs > 1 && P.n_seqs <= AF_WARPS * 32 && problems * split > (uint64_t)ctx->sm_count;
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
