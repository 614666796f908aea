// Device helpers of the kernels that hold a whole row in registers (norms, 8-bit quantisation): a row of
// nvec 16-byte vectors belongs to TPR threads, thread t holding vectors t, t + TPR, ... (VPT of them).
#pragma once
#include "common.cuh"

namespace oc {

// threads per CTA
template <int TPR> struct RowCta { static constexpr int threads = TPR >= 128 ? TPR : (TPR == 64 ? 256 : 128), rows = threads / TPR; };

// Two fp32 values in one 64-bit register, and the instructions that work on both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 f2(float lo, float hi) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi)); return r; }
__device__ __forceinline__ f32x2 f2(float v) { return f2(v, v); }
__device__ __forceinline__ float f2_lo(f32x2 v) { float a, b; asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); return a; }
__device__ __forceinline__ float f2_hi(f32x2 v) { float a, b; asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); return b; }
__device__ __forceinline__ f32x2 f2_add(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 f2_mul(f32x2 a, f32x2 b) { f32x2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f32x2 f2_fma(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 f2_bits(uint32_t lo, uint32_t hi) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi)); return r; }

// One 16-byte vector of a row as pairs of floats.
template <int DT> struct RowVec;
template <> struct RowVec<OC_DTYPE_BF16> {
    static constexpr int E = 8;                                              // elements
    static __device__ __forceinline__ void unpack(const uint4& v, f32x2* f) {
        f[0] = f2_bits(v.x << 16, v.x & 0xFFFF0000u); f[1] = f2_bits(v.y << 16, v.y & 0xFFFF0000u);
        f[2] = f2_bits(v.z << 16, v.z & 0xFFFF0000u); f[3] = f2_bits(v.w << 16, v.w & 0xFFFF0000u);
    }
};
template <> struct RowVec<OC_DTYPE_F32> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void unpack(const uint4& v, f32x2* f) { f[0] = f2_bits(v.x, v.y); f[1] = f2_bits(v.z, v.w); }
};

// n / d for n < 2^31 with a multiplication (d >= 1): with 2^(L-1) < d <= 2^L and mul = ceil(2^(31+L) / d), the
// product exceeds n 2^(31+L) / d by less than 2^(31+L) / d.
struct FastDiv {
    uint32_t d, mul, shift;
    FastDiv() = default;
    explicit FastDiv(uint32_t d_) : d(d_), mul(0), shift(0) {
        if (d == 1) return;
        uint32_t L = 1;
        while (L < 31 && (1u << L) < d) ++L;
        mul = (uint32_t)(((1ull << (31 + L)) + d - 1) / d);
        shift = L - 1;
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return d == 1 ? n : __umulhi(n, mul) >> shift; }
};

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint4 ld_v4(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// E consecutive parameters starting at element `at` (a multiple of E), widened to fp32.  Parameters are
// read by every row, so they go through the read-only path and stay in L1.
template <int PT, int E>
__device__ __forceinline__ void load_param(const void* base, long long at, f32x2* f) {
    if (PT == OC_DTYPE_F32) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i) RowVec<OC_DTYPE_F32>::unpack(__ldg((const uint4*)((const float*)base + at) + i), f + 2 * i);
    } else if (E == 8) {
        RowVec<OC_DTYPE_BF16>::unpack(__ldg((const uint4*)((const uint16_t*)base + at)), f);
    } else {
        const uint2 v = __ldg((const uint2*)((const uint16_t*)base + at));
        f[0] = f2_bits(v.x << 16, v.x & 0xFFFF0000u); f[1] = f2_bits(v.y << 16, v.y & 0xFFFF0000u);
    }
}

// E consecutive floats of a row rounded to type DT and stored at element `at`.
__device__ __forceinline__ uint32_t pack_bf16x2(f32x2 v) { return pack_bf16x2(f2_lo(v), f2_hi(v)); }
template <int DT, int E>
__device__ __forceinline__ void store_row(void* base, long long at, const f32x2* f) {
    if (DT == OC_DTYPE_F32) {
#pragma unroll
        for (int i = 0; i < E / 4; ++i)
            st_v4((float*)base + at + 4 * i, make_uint4(__float_as_uint(f2_lo(f[2 * i])), __float_as_uint(f2_hi(f[2 * i])),
                                                        __float_as_uint(f2_lo(f[2 * i + 1])), __float_as_uint(f2_hi(f[2 * i + 1]))));
    } else if (E == 8) {
        st_v4((uint16_t*)base + at, make_uint4(pack_bf16x2(f[0]), pack_bf16x2(f[1]), pack_bf16x2(f[2]), pack_bf16x2(f[3])));
    } else {
        *(uint2*)((uint16_t*)base + at) = make_uint2(pack_bf16x2(f[0]), pack_bf16x2(f[1]));
    }
}

template <int E> __device__ __forceinline__ void store_row_smem(float* to, const f32x2* f) {
#pragma unroll
    for (int i = 0; i < E / 4; ++i) *(float4*)(to + 4 * i) = make_float4(f2_lo(f[2 * i]), f2_hi(f[2 * i]), f2_lo(f[2 * i + 1]), f2_hi(f[2 * i + 1]));
}

// Sum / maximum over the TPR threads of a row; every one of them gets the same result (butterflies within a
// warp, then a fixed order over the warps: no atomics, so a row's result never depends on scheduling).
// Rows wider than a warp meet at a barrier of their own threads, and `scratch` holds one word per warp and parity.
struct RowScratch { uint32_t w[2][16]; };
template <int TPR, class Op>
__device__ __forceinline__ uint32_t row_reduce(uint32_t v, Op op, RowScratch* scratch, int& parity) {
    constexpr int W = TPR < 32 ? TPR : 32;
#pragma unroll
    for (int d = W / 2; d >= 1; d >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    if (TPR > 32) {
        // (two buffers taken in turn: a warp that is ahead writes the other one, and the barrier of that
        //  reduction keeps it from coming back before everybody has read this one)
        uint32_t* w = scratch->w[parity];
        parity ^= 1;
        if ((threadIdx.x & 31) == 0) w[(threadIdx.x % TPR) >> 5] = v;
        asm volatile("bar.sync %0, %1;" :: "r"(1 + (int)threadIdx.x / TPR), "n"(TPR > 32 ? TPR : 32) : "memory");
        v = w[0];
#pragma unroll
        for (int i = 1; i < TPR / 32; ++i) v = op(v, w[i]);
    }
    return v;
}
template <int TPR>
__device__ __forceinline__ float row_sum(float v, RowScratch* s, int& parity) {
    return __uint_as_float(row_reduce<TPR>(__float_as_uint(v),
        [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }, s, parity));
}
// Largest magnitude, from the magnitudes' bit patterns: the order of the patterns is that of the values, with
// infinity above every number and NaN above infinity, so a row that holds either says so.
template <int TPR>
__device__ __forceinline__ uint32_t row_max_bits(uint32_t v, RowScratch* s, int& parity) {
    return row_reduce<TPR>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }, s, parity);
}

// A row's 8-bit form: scale = max|x| / 127, q = rint(x * 127 / max|x|).  A row whose largest magnitude is below
// 2^-100 has no useful scale (its reciprocal leaves the range) and becomes zeros with scale 0.  A row with an
// infinity or a NaN keeps that in its scale, so that whatever is multiplied with it shows it; its q are zeros.
struct RowQuant { float scale, inv; };
__device__ __forceinline__ RowQuant row_quant(uint32_t max_bits) {
    const float m = __uint_as_float(max_bits);
    RowQuant r;
    if (max_bits >= 0x7F800000u) { r.scale = m; r.inv = 0.0f; }
    else if (m < 7.8886091e-31f) { r.scale = 0.0f; r.inv = 0.0f; }
    else { r.scale = m * (1.0f / 127.0f); r.inv = 127.0f / m; }
    return r;
}
template <int E>
__device__ __forceinline__ uint32_t max_bits(const f32x2* f, uint32_t m) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) m = max(m, max(__float_as_uint(f2_lo(f[i])) & 0x7FFFFFFFu, __float_as_uint(f2_hi(f[i])) & 0x7FFFFFFFu));
    return m;
}
// (inv = 0 has to give q = 0 even where x is not finite: 0 * inf is NaN, which cvt.rni.s32 turns into 0)
__device__ __forceinline__ uint32_t pack_s8x4(f32x2 a, f32x2 b, float inv) {
    const f32x2 x = f2_mul(a, f2(inv)), y = f2_mul(b, f2(inv));
    return ((uint32_t)__float2int_rn(f2_lo(x)) & 0xFFu) | (((uint32_t)__float2int_rn(f2_hi(x)) & 0xFFu) << 8) |
           (((uint32_t)__float2int_rn(f2_lo(y)) & 0xFFu) << 16) | ((uint32_t)__float2int_rn(f2_hi(y)) << 24);
}
template <int E>
__device__ __forceinline__ void store_row_s8(void* base, long long at, const f32x2* f, float inv) {
    int8_t* p = (int8_t*)base + at;
    if (E == 8) *(uint2*)p = make_uint2(pack_s8x4(f[0], f[1], inv), pack_s8x4(f[2], f[3], inv));
    else *(uint32_t*)p = pack_s8x4(f[0], f[1], inv);
}

// The split of a row of more than MIN vectors over TPR threads with up to VPT each.
template <int TPR, int VPT, int MIN> struct RowSplit {
    static constexpr int tpr = TPR, vpt = VPT;
    // whether thread t has a j-th vector (known without looking for all but the last few)
    static __device__ __forceinline__ bool has(int j, int t, int nvec) { return (j + 1) * TPR <= MIN + 1 || j * TPR + t < nvec; }
};
// Picks the row split for nvec vectors: as few threads as hold the row in 3 to 6 vectors each, so that several 16-byte
// loads per thread are in flight and few lanes idle, and more of them where 5 or 6 vectors' registers leave too few
// warps on an SM.  oc_block_norm on 8192 rows, half of them with a slot, in us, this split | the neighbouring one:
//     vectors of a row          80          128         144         192         256         320         400
//     threads                32 | 16     32 | 64     32 | 64     64 | 32     64 | 128    64 | 128   256 | 128
//     bf16, z and cache    12.7 | 13.7 17.2 | 18.4 22.6 | 20.8 23.1 | 26.5 29.1 | 40.0 42.0 | 49.1 52.6 | 58.7
//     fp32, z and cache    11.6 | 10.9 15.8 | 16.9 18.0 | 17.2 21.6 | 23.8 28.9 | 36.6 36.5 | 41.8 49.1 | 51.4
//     bf16, norm alone      7.9 | 6.7   8.7 | 11.5  9.9 | 13.2 13.8 | 12.2 16.6 | 24.6 22.8 | 29.3 35.7 | 35.2
//     fp32, norm alone      7.0 | 5.5   7.2 | 9.8   8.4 | 10.8 10.9 | 8.2  11.2 | 21.0 14.1 | 22.7 29.0 | 26.1
// One rule serves all four: it costs at most 8 % with z, and up to a third on some widths of the norm alone.  Calls f with
// the split; false if the row is too wide (more than 3072 vectors).
template <class F>
inline bool row_split(long long nvec, F&& f) {
    if (nvec <= 8) f(RowSplit<8, 1, 0>());
    else if (nvec <= 16) f(RowSplit<8, 2, 8>());
    else if (nvec <= 24) f(RowSplit<8, 3, 16>());
    else if (nvec <= 32) f(RowSplit<8, 4, 24>());
    else if (nvec <= 40) f(RowSplit<8, 5, 32>());
    else if (nvec <= 48) f(RowSplit<8, 6, 40>());
    else if (nvec <= 64) f(RowSplit<16, 4, 48>());
    else if (nvec <= 96) f(RowSplit<32, 3, 64>());
    else if (nvec <= 128) f(RowSplit<32, 4, 96>());
    else if (nvec <= 160) f(RowSplit<32, 5, 128>());
    else if (nvec <= 192) f(RowSplit<64, 3, 160>());
    else if (nvec <= 256) f(RowSplit<64, 4, 192>());
    else if (nvec <= 384) f(RowSplit<64, 6, 256>());
    else if (nvec <= 512) f(RowSplit<256, 2, 384>());
    else if (nvec <= 768) f(RowSplit<256, 3, 512>());
    else if (nvec <= 1536) f(RowSplit<512, 3, 768>());
    else if (nvec <= 3072) f(RowSplit<512, 6, 1536>());
    else return false;
    return true;
}

}  // namespace oc
