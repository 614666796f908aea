// Device helpers of the kernels that hold a whole row in registers (norms, 8-bit quantisation): a row of
// nvec 16-byte vectors belongs to TPR threads, thread t holding vectors t, t + TPR, ... (VPT of them).
#pragma once
#include "common.cuh"

namespace oc {

static constexpr int ROW_THREADS = 256;          // threads per CTA while a row fits one warp

// One 16-byte vector of a row as floats.
template <int DT> struct RowVec;
template <> struct RowVec<OC_DTYPE_BF16> {
    static constexpr int E = 8;                                              // elements
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
        f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
    }
};
template <> struct RowVec<OC_DTYPE_F32> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void unpack(const uint4& v, float* f) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
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
__device__ __forceinline__ void load_param(const void* base, long long at, float* f) {
    if (PT == OC_DTYPE_F32) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const float4 v = __ldg((const float4*)((const float*)base + at + i));
            f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
        }
    } else if (E == 8) {
        RowVec<OC_DTYPE_BF16>::unpack(__ldg((const uint4*)((const uint16_t*)base + at)), f);
    } else {
        const uint2 v = __ldg((const uint2*)((const uint16_t*)base + at));
        f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    }
}

// E consecutive floats of a row rounded to type DT and stored at element `at`.
template <int DT, int E>
__device__ __forceinline__ void store_row(void* base, long long at, const float* f) {
    if (DT == OC_DTYPE_F32) {
#pragma unroll
        for (int i = 0; i < E; i += 4)
            st_v4((float*)base + at + i, make_uint4(__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]), __float_as_uint(f[i + 3])));
    } else if (E == 8) {
        st_v4((uint16_t*)base + at, make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])));
    } else {
        *(uint2*)((uint16_t*)base + at) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
    }
}

// Sum / maximum over the TPR threads of a row; every one of them gets the same result (butterflies within a
// warp, then a fixed order over the warps: no atomics, so a row's result never depends on scheduling).
// Rows wider than a warp take the whole CTA, and `scratch` holds one word per warp and parity.
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
        if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = v;
        __syncthreads();
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
// (inv = 0 has to give q = 0 even where x is not finite: 0 * inf is NaN, which cvt.rni.s32 turns into 0)
__device__ __forceinline__ uint32_t pack_s8x4(const float* f, float inv) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= ((uint32_t)__float2int_rn(f[i] * inv) & 0xFFu) << (8 * i);
    return r;
}
template <int E>
__device__ __forceinline__ void store_row_s8(void* base, long long at, const float* f, float inv) {
    int8_t* p = (int8_t*)base + at;
    if (E == 8) *(uint2*)p = make_uint2(pack_s8x4(f, inv), pack_s8x4(f + 4, inv));
    else *(uint32_t*)p = pack_s8x4(f, inv);
}

// Picks the row split for nvec vectors: the fewest threads that hold the row in at most 6 vectors each, so that
// few lanes idle and several 16-byte loads per thread are in flight.  Calls f with the two sizes as
// std::integral_constant; false if the row is too wide (more than 3072 vectors).
template <int TPR, int VPT> struct RowSplit { static constexpr int tpr = TPR, vpt = VPT; };
template <class F>
inline bool row_split(long long nvec, F&& f) {
    if (nvec <= 8) f(RowSplit<8, 1>());
    else if (nvec <= 16) f(RowSplit<8, 2>());
    else if (nvec <= 24) f(RowSplit<8, 3>());
    else if (nvec <= 32) f(RowSplit<8, 4>());
    else if (nvec <= 40) f(RowSplit<8, 5>());
    else if (nvec <= 48) f(RowSplit<8, 6>());
    else if (nvec <= 64) f(RowSplit<16, 4>());
    else if (nvec <= 80) f(RowSplit<16, 5>());
    else if (nvec <= 96) f(RowSplit<16, 6>());
    else if (nvec <= 128) f(RowSplit<32, 4>());
    else if (nvec <= 160) f(RowSplit<32, 5>());
    else if (nvec <= 192) f(RowSplit<32, 6>());
    else if (nvec <= 256) f(RowSplit<128, 2>());
    else if (nvec <= 384) f(RowSplit<128, 3>());
    else if (nvec <= 768) f(RowSplit<128, 6>());
    else if (nvec <= 1536) f(RowSplit<512, 3>());
    else if (nvec <= 3072) f(RowSplit<512, 6>());
    else return false;
    return true;
}

}  // namespace oc
