// Matrix product in 8-bit integers with one scale per token and one per output channel:
//     out[dst(m), n] = a_scale[m] * w_scale[n] * sum_k a[m, k] * w[n, k] + bias[n]
// The sums are exact (32-bit integers), the scales and the bias are applied in fp32, the result is rounded once.
//
// Many tokens: tcgen05.mma kind::i8 (8-bit operands, 32-bit accumulators in tensor memory).  One persistent CTA
// (or CTA pair, cta_group::2) per SM walks over output tiles of 128 x N_TILE (256 x 256 for a pair):
//   warp 0       copies: TMA boxes of 128 bytes of K by 128 rows, 128-byte swizzle, into a ring of stages
//   warp 1       the MMAs (128 bytes of K = four steps of 32); owns the tensor memory
//   warps 2..17  epilogue: thread = row, four warps side by side, a quarter of the columns each; scales, bias,
//                rounding, then through shared memory: rows that keep their order leave as TMA boxes, others as
//                whole 64-byte pieces to where out_idx says
// Two accumulators take turns, so the epilogue of a tile runs under the MMAs of the next.
// One or two tokens: one warp per pair of output channels, dp4a, the weights read once as they lie.
// K and N tails are zero-filled by TMA and not stored.  Every wait is bounded (OC_ERR_TIMEOUT in the status word).
// Measured in short runs at full clock | for seconds on end, under the power limit: 8192 x 6400 x 8192 273 us (3.1 POP/s) |
// 311 (2.8 POP/s at 1.26 GHz, 0.9 of 16384 operations per SM and clock); 5120 x 1536 x 4608 28 | 33; 57600 x 640 x 5120
// 157 | 188 (1.25 GHz; 139 on zeros, which draw less power), of which 590 MB of output alone take 90 to 100.  The ring
// form of 256 columns spills 52 bytes.
#include <string.h>

#include <algorithm>
#include <mutex>

#include "rows.cuh"
#include "tc_ptx.cuh"

namespace oc {

static constexpr int I8_BM = 128, I8_BK = 128;                      // rows of a CTA's tile; bytes of K per stage
static constexpr int I8_EPI_WARPS = 16, I8_THREADS = 64 + 32 * I8_EPI_WARPS;
static constexpr int I8_A_BYTES = I8_BM * I8_BK;
static constexpr int I8_STAGES_MAX = 8;

// An epilogue warp stages 64 bytes of each of its 32 rows at a time.  128 would save a wait, but the shared memory is
// worth more as ring: loads that compete with 148 SMs' stores come back late.  57600 x 640 x 5120 takes 157 us with 64
// bytes and seven stages (resident form) and 181 with 128 bytes and the five that they leave; 8192 x 1536 x 6144 55 with
// six stages (ring form) and 61 with five.  (64 bytes and five stages: 170 and 56; four: 182 and 58.)
static constexpr int I8_SEG = 64, I8_OUT_STAGE = 32 * I8_SEG;

struct I8Params {
    CUtensorMap mapA, mapW;      // {K, rows}: boxes {128, 128} and {128, rows of W per CTA}
    CUtensorMap mapOut;          // {N, M}: box {64 bytes, 32}; used when rows keep their order
    const float *a_scale, *w_scale, *bias;
    const int32_t* out_idx;
    void* out;
    long long out_stride;
    int M, N, out_rows;
    int kblocks, m_tiles, n_tiles, n_stages;
    int a_bytes;                 // of A per stage: fewer than a tile's where there are not that many tokens
    int rows_of_walkers, main_rows;    // see I8Walk
    int wide, tma_out;           // rows of `out` may be stored in 16-byte pieces; by TMA
    int* status;
};

template <bool PAIR>
__device__ __forceinline__ void tma_load_2d_elected(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar, uint32_t issue) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %5, 0;\n\t"
                     "@e cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
                     :: "r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar), "r"(issue) : "memory");
    else
        asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %5, 0;\n\t"
                     "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t}"
                     :: "r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar), "r"(issue) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tc_mma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate, uint32_t issue) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
                     "@e tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(issue) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
                     "@e tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     :: "r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(issue) : "memory");
}
// Where 16-byte piece j of a staged row lies: TMA's swizzle for rows of 64 bytes, which also spreads the pieces that
// a warp's lanes write, one row each, over all banks.
__device__ __forceinline__ uint32_t i8_staged(int row, int j) { return (uint32_t)(row * I8_SEG + ((j ^ ((row >> 1) & 3)) << 4)); }
// arrive on `bar` (of both CTAs in a pair) once every MMA issued so far has retired
template <bool PAIR>
__device__ __forceinline__ void tc_commit_all(uint32_t bar, uint32_t issue) {
    if (PAIR)
        asm volatile("{\n\t.reg .pred e;\n\t.reg .b16 both;\n\tmov.b16 both, 3;\n\tsetp.ne.b32 e, %1, 0;\n\t"
                     "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], both;\n\t}"
                     :: "r"(bar), "r"(issue) : "memory");
    else
        tc_commit<false>(bar, issue);
}

// The tiles of a walker.  Whole rows of `out` are written at about the same time, which is what DRAM writes fastest
// (walks in groups of 9 and of 3 tile columns cost a 57600 x 5120 output 8 and 16 % in the ring form), and each row of A
// is read from DRAM once.
//   ring form      tile after tile along a row of tiles; W comes back from L2 for every tile
//   resident form  a walker keeps its tile column, so that its rows of W stay in shared memory (57600 x 640 x 5120:
//                  157 us, ring form 194): the walkers form as many whole rows of tiles as
//                  there are (`rows_of_walkers`), which go down the first `main_rows` rows together; the walkers
//                  left over share out the other rows, column after column
struct I8Walk {
    int n_tiles, m_tiles, tile, step, end, column, above;            // column: of a walker that keeps it, or -1
    template <bool RES> __device__ __forceinline__ void start(const I8Params& P, int walker, int walkers) {
        n_tiles = P.n_tiles; m_tiles = P.m_tiles; column = -1; above = 0;
        if (!RES) { tile = walker; step = walkers; end = m_tiles * n_tiles; return; }
        const int mains = P.rows_of_walkers * n_tiles;
        if (walker < mains) { tile = walker / n_tiles; column = walker - tile * n_tiles; step = P.rows_of_walkers; end = P.main_rows; return; }
        above = P.main_rows;
        const long long rest = (long long)(m_tiles - above) * n_tiles, x = walker - mains, of = walkers - mains;
        tile = (int)(rest * x / of); end = (int)(rest * (x + 1) / of); step = 1;
    }
    template <bool RES> __device__ __forceinline__ bool next(int& m, int& n) {
        if (tile >= end) return false;
        if (!RES) { m = tile / n_tiles; n = tile - m * n_tiles; }
        else if (column >= 0) { m = tile; n = column; }
        else { const int rows = m_tiles - above; n = tile / rows; m = above + tile - n * rows; }
        tile += step;
        return true;
    }
};

template <int N_TILE, bool PAIR, bool RES, int OT>
__global__ void __launch_bounds__(I8_THREADS, 1)
linear_int8_kernel(const __grid_constant__ I8Params P) {
    constexpr int W_ROWS = PAIR ? N_TILE / 2 : N_TILE;               // rows of W that this CTA fetches
    constexpr int W_BYTES = W_ROWS * I8_BK;
    constexpr int STAGE_BYTES = RES ? I8_A_BYTES : I8_A_BYTES + W_BYTES;
    constexpr int TMEM_COLS = 2 * N_TILE;
    constexpr int OB = OT == OC_DTYPE_F32 ? 4 : 2;
    constexpr int WC = N_TILE >= 128 ? N_TILE / 4 : 32;              // columns of an epilogue warp
    constexpr int PASS = I8_SEG / OB, PARTS = N_TILE / WC;           // columns that it stages together; warps side by side
    constexpr int LPR = I8_SEG / 16, RPI = 32 / LPR;                 // lanes that store a staged row; rows per store
    extern __shared__ __align__(1024) uint8_t i8_smem[];
    const uint32_t w_bytes = RES ? (uint32_t)(P.kblocks * W_BYTES) : 0u;       // W of this walker's column, in front of the ring
    uint8_t* after = i8_smem + w_bytes + (size_t)P.n_stages * STAGE_BYTES;
    uint8_t* out_stage = after;                                      // [warps][32 rows][64 bytes]
    float* col_tab = (float*)(after + I8_EPI_WARPS * I8_OUT_STAGE);  // [parts][scale, bias][WC]
    uint64_t* bars = (uint64_t*)(col_tab + 2 * N_TILE);
    const uint32_t resident = smem_u32(i8_smem), tiles = resident + w_bytes;
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * I8_STAGES_MAX;
    const uint32_t bar_acc_full = bar_empty + 8 * I8_STAGES_MAX, bar_acc_empty = bar_acc_full + 16, bar_drain = bar_acc_empty + 16;
    const uint32_t bar_w_full = bar_drain + 8, bar_w_empty = bar_drain + 16;
    uint32_t* tmem_slot = (uint32_t*)(bars + 2 * I8_STAGES_MAX + 7);
    volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;
    const int STAGES = P.n_stages;

    if ((tiles & 1023u) != 0) {                                      // never expected; refuse rather than compute garbage
        if (threadIdx.x == 0) atomicCAS(P.status, 0, OC_ERR_ALIGNMENT);
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < I8_STAGES_MAX; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(bar_acc_full + 8 * b, 1); mbar_init(bar_acc_empty + 8 * b, (PAIR ? 2 : 1) * I8_EPI_WARPS); }
        mbar_init(bar_drain, 1); mbar_init(bar_w_full, 1); mbar_init(bar_w_empty, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tma_prefetch_map(&P.mapA);
        tma_prefetch_map(&P.mapW);
        if (P.tma_out) tma_prefetch_map(&P.mapOut);
    }
    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            tmem_alloc_cta1(smem_u32(tmem_slot), TMEM_COLS);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();                                    // the other CTA's barriers exist before anything signals them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();                                                      // the operands may come from the kernel before this one
    if (threadIdx.x == 0) pdl_launch_dependents();
    I8Walk walk;
    walk.template start<RES>(P, PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x);
    int m, n;

    if (warp == 0) {
        // ================================ copies ================================================
        // The whole warp runs this and an elected lane issues: addresses and coordinates then are warp-uniform, where a
        // lone lane would have them moved for every copy, which takes it longer than the copies' MMAs.
        const uint32_t issue = elect_one();
        int stage = 0, held = -1; uint32_t phase = 0, armed = 0, w_phase = 0;
        bool ok = true, have = walk.template next<RES>(m, n);
        while (ok && have) {
            const int row0 = m * (PAIR ? 2 * I8_BM : I8_BM) + (int)rank * I8_BM, col0 = n * N_TILE + (int)rank * W_ROWS;
            if (RES && n != held) {                                  // another column: its W, once the last one's MMAs are over
                if (held >= 0) {
                    if (!__all_sync(0xFFFFFFFFu, mbar_wait(bar_w_empty, w_phase, abort_flag))) { ok = false; break; }
                    w_phase ^= 1u;
                }
                held = n;
                for (int kb = 0; kb < P.kblocks; ++kb)
                    tma_load_2d_elected<PAIR>(resident + (uint32_t)(kb * W_BYTES), &P.mapW, kb * I8_BK, col0, PAIR ? map_to_cta(bar_w_full, 0) : bar_w_full, issue);
                if (leader) mbar_arrive_expect_tx_elected(bar_w_full, (PAIR ? 2 : 1) * w_bytes, issue);
            }
            for (int kb = 0; kb < P.kblocks; ++kb) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(bar_empty + 8 * stage, phase ^ 1u, abort_flag))) { ok = false; break; }
                const uint32_t dst = tiles + (uint32_t)(stage * STAGE_BYTES), full = bar_full + 8 * stage;
                const uint32_t bar = PAIR ? map_to_cta(full, 0) : full;               // both CTAs' copies report to the leader
                // (the copies first: the barrier cannot complete before the arrival that carries their byte count)
                tma_load_2d_elected<PAIR>(dst, &P.mapA, kb * I8_BK, row0, bar, issue);
                if (!RES) tma_load_2d_elected<PAIR>(dst + I8_A_BYTES, &P.mapW, kb * I8_BK, col0, bar, issue);
                if (leader) mbar_arrive_expect_tx_elected(full, (PAIR ? 2 : 1) * (uint32_t)(P.a_bytes + (RES ? 0 : W_BYTES)), issue);
                armed |= 1u << stage;
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                if (kb == 0) have = walk.template next<RES>(m, n);
            }
        }
        if (!ok && lane == 0) {
            atomicCAS(P.status, 0, OC_ERR_TIMEOUT);
            *abort_flag = 1;
            // copies already issued still write this CTA's shared memory: a bounded chance to land
            const unsigned long long t0 = global_ns();
            if (leader) {
                for (int s = 0; s < STAGES; ++s)
                    if (armed & (1u << s))
                        while (!mbar_try_wait(bar_full + 8 * s, s < stage ? phase : phase ^ 1u) && global_ns() - t0 < 20000000ull) {}
            }
            if (!leader || RES) while (global_ns() - t0 < 2000000ull) {}       // (the peer's, and W's, report elsewhere)
        }
    } else if (warp == 1) {
        // ================================ MMAs ==================================================
        if (leader) {
            constexpr uint32_t IDESC = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N_TILE >> 3) << 17) |
                                       ((uint32_t)((PAIR ? 2 * I8_BM : I8_BM) >> 4) << 24);       // D = s32, A = B = s8, K-major
            const uint32_t issue = elect_one();
            int stage = 0, held = -1; uint32_t phase = 0, it = 0, w_phase = 0;
            bool ok = true, have = walk.template next<RES>(m, n);
            while (ok && have) {
                const int column = n;
                have = walk.template next<RES>(m, n);
                const uint32_t buf = it & 1u, acc_phase = (it >> 1) & 1u;
                ++it;
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(bar_acc_empty + 8 * buf, acc_phase ^ 1u, abort_flag))) { ok = false; break; }
                if (RES && column != held) {
                    if (!__all_sync(0xFFFFFFFFu, mbar_wait(bar_w_full, w_phase, abort_flag))) { ok = false; break; }
                    w_phase ^= 1u; held = column;
                }
                tc_fence_after();
                const uint32_t d = tmem_base + buf * N_TILE;
                for (int kb = 0; kb < P.kblocks; ++kb) {
                    if (!__all_sync(0xFFFFFFFFu, mbar_wait(bar_full + 8 * stage, phase, abort_flag))) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a_addr = tiles + (uint32_t)(stage * STAGE_BYTES);
                    const uint64_t a_desc = make_smem_desc(a_addr), b_desc = make_smem_desc(RES ? resident + (uint32_t)(kb * W_BYTES) : a_addr + I8_A_BYTES);
#pragma unroll
                    for (int k = 0; k < 4; ++k)                      // 32 bytes of K at a time along the swizzled rows
                        tc_mma_i8<PAIR>(d, a_desc + 2 * k, b_desc + 2 * k, IDESC, (uint32_t)((kb | k) != 0), issue);
                    tc_commit_all<PAIR>(bar_empty + 8 * stage, issue);
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
                if (ok) tc_commit_all<PAIR>(bar_acc_full + 8 * buf, issue);
                if (RES && ok && have && n != column) tc_commit_all<PAIR>(bar_w_empty, issue);
            }
            if (!ok && lane == 0) { atomicCAS(P.status, 0, OC_ERR_TIMEOUT); *abort_flag = 1; }
            // every MMA retires before tensor memory is released
            tc_commit<PAIR>(PAIR ? map_to_cta(bar_drain, 0) : bar_drain, issue);
            const unsigned long long t0 = global_ns();
            while (!mbar_try_wait(bar_drain, 0) && global_ns() - t0 < WAIT_LIMIT_NS) {}
        }
    } else {
        // ================================ epilogue ==============================================
        const int ew = warp - 2, quarter = warp & 3, part = ew >> 2; // TMEM lanes of this warp; which of the columns
        const bool works = part < PARTS;                             // (narrow tiles do not occupy all warps)
        const uint32_t acc_empty = PAIR ? map_to_cta(bar_acc_empty, 0) : bar_acc_empty;          // the leader's
        const uint32_t stage_base = smem_u32(out_stage + ew * I8_OUT_STAGE);
        float* tab = col_tab + (works ? part : 0) * 2 * WC;          // scales and biases of the part's columns
        // What a tile needs beside its sums is fetched a tile ahead: the latency passes under the tile before.
        // (the part's four warps fetch a column each: its scale, or with the upper lanes its bias)
        const int et = (ew & 3) * 32 + lane;
        struct Ahead { float col, sa; int dst; } ah;
        auto fetch = [&](int m_, int n_) {
            const int c = n_ * N_TILE + part * WC + et % WC;
            const float* from = et < WC ? P.w_scale : P.bias;
            ah.col = et < 2 * WC && works && from && c < P.N ? __ldg(from + c) : 0.0f;
            const int r = m_ * (PAIR ? 2 * I8_BM : I8_BM) + (int)rank * I8_BM + quarter * 32 + lane;
            ah.dst = -1; ah.sa = 0.0f;
            if (r < P.M) { ah.sa = __ldg(P.a_scale + r); ah.dst = P.out_idx ? __ldg(P.out_idx + r) : r; }
        };
        uint32_t it = 0;
        int tab_n = -1;                                              // the tile column that the table is of
        bool ok = true, have = walk.template next<RES>(m, n);
        if (have) fetch(m, n);
        while (have) {
            const uint32_t buf = it & 1u, acc_phase = (it >> 1) & 1u;
            ++it;
            const int row0 = m * (PAIR ? 2 * I8_BM : I8_BM) + (int)rank * I8_BM + quarter * 32, col0 = n * N_TILE + part * WC;
            if (works && n != tab_n) {
                asm volatile("bar.sync %0, 128;" :: "r"(1 + part) : "memory");       // the part is done with the table
                if (et < 2 * WC) tab[et] = ah.col;
                asm volatile("bar.sync %0, 128;" :: "r"(1 + part) : "memory");
                tab_n = n;
            }
            const float sa = ah.sa;
            int dst = ah.dst;
            if (dst >= P.out_rows) { atomicCAS(P.status, 0, OC_ERR_INVALID_ARG); dst = -1; }
            have = walk.template next<RES>(m, n);
            if (have) fetch(m, n);
            // (a warp that has given up keeps meeting the others at the barriers, and waits for nothing else)
            if (ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(bar_acc_full + 8 * buf, acc_phase, abort_flag));
            if (!ok) continue;
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * N_TILE + (uint32_t)(part * WC);
            // The sums go into registers at once and the accumulator back to the MMAs; scaling and storing them then
            // delays nobody but this warp.
            uint32_t v[WC];
            if (works) {
#pragma unroll
                for (int c = 0; c < WC; c += 32) tmem_ld32(t_row + (uint32_t)c, v + c);
                tmem_ld_wait();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) { if (PAIR) mbar_arrive_cluster(acc_empty + 8 * buf); else mbar_arrive(acc_empty + 8 * buf); }
            if (works) {
#pragma unroll
                for (int pass = 0; pass < WC / PASS; ++pass) {
                    uint32_t* o = v + pass * PASS;
                    const float4* sw = (const float4*)(tab + pass * PASS);
                    const float4* bs = (const float4*)(tab + WC + pass * PASS);
                    const f32x2 s2 = f2(sa);
#pragma unroll
                    for (int j = 0; j < PASS; j += 4) {
                        const float4 w = sw[j / 4], b = bs[j / 4];
                        const f32x2 lo = f2_fma(f2_mul(f2((float)(int)o[j], (float)(int)o[j + 1]), s2), f2(w.x, w.y), f2(b.x, b.y));
                        const f32x2 hi = f2_fma(f2_mul(f2((float)(int)o[j + 2], (float)(int)o[j + 3]), s2), f2(w.z, w.w), f2(b.z, b.w));
                        if (OT == OC_DTYPE_F32) {
                            o[j] = __float_as_uint(f2_lo(lo)); o[j + 1] = __float_as_uint(f2_hi(lo));
                            o[j + 2] = __float_as_uint(f2_lo(hi)); o[j + 3] = __float_as_uint(f2_hi(hi));
                        } else {
                            o[j / 2] = pack_bf16x2(lo);
                            o[j / 2 + 1] = pack_bf16x2(hi);
                        }
                    }
                    // the piece staged before has left (it had this one's arithmetic to do so)
                    if (P.tma_out && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < I8_SEG / 16; ++j)
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(stage_base + i8_staged(lane, j)),
                                     "r"(o[4 * j]), "r"(o[4 * j + 1]), "r"(o[4 * j + 2]), "r"(o[4 * j + 3]) : "memory");
                    if (P.tma_out) {
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) {
                            // (rows and columns past the end are clipped; a box wholly outside starts past the last row or column)
                            if (row0 < P.M && col0 + pass * PASS < P.N)
                                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                                             :: "l"(&P.mapOut), "r"(col0 + pass * PASS), "r"(row0), "r"(stage_base) : "memory");
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                        continue;
                    }
                    __syncwarp();
                    if (!P.wide) {                                   // rows of `out` that are not 16-byte aligned: element by element
                        constexpr int COLS = PASS < 32 ? PASS : 32;  // lanes of a row; two rows at a time where it is short
#pragma unroll 8
                        for (int r = 0; r < COLS; ++r) {
                            const int row = r * (32 / COLS) + lane / COLS, at = (lane % COLS) * OB, col = col0 + pass * PASS + lane % COLS;
                            const int d = __shfl_sync(0xFFFFFFFFu, dst, row);
                            const uint32_t from = stage_base + i8_staged(row, at >> 4) + (uint32_t)(at & 15);
                            const bool keep = d >= 0 && col < P.N;
                            if (OB == 4) {
                                uint32_t x;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(from) : "memory");
                                if (keep) ((uint32_t*)P.out)[(long long)d * P.out_stride + col] = x;
                            } else {
                                uint16_t x;
                                asm volatile("ld.shared.b16 %0, [%1];" : "=h"(x) : "r"(from) : "memory");
                                if (keep) ((uint16_t*)P.out)[(long long)d * P.out_stride + col] = x;
                            }
                        }
                        continue;
                    }
                    const int col = col0 + pass * PASS + (lane % LPR) * (16 / OB);
#pragma unroll
                    for (int i = 0; i < 32 / RPI; ++i) {
                        const int row = i * RPI + lane / LPR;
                        const int d = __shfl_sync(0xFFFFFFFFu, dst, row);
                        uint4 x;
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(stage_base + i8_staged(row, lane % LPR)) : "memory");
                        if (d >= 0 && col < P.N) {
                            uint8_t* p = (uint8_t*)P.out + ((long long)d * P.out_stride + col) * OB;
                            if (col + 16 / OB <= P.N) {
                                st_v4(p, x);
                            } else {                                 // the row's last, partial 16 bytes
                                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                                for (int e = 0; e < P.N - col; ++e) {
                                    if (OB == 4) ((uint32_t*)p)[e] = w[e];
                                    else ((uint16_t*)p)[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
                                }
                            }
                        }
                    }
                }
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");                 // its pieces are written
        if (!ok && lane == 0) { atomicCAS(P.status, 0, OC_ERR_TIMEOUT); *abort_flag = 1; }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();                                    // nobody signals a barrier of, or reads operands from, a retired CTA
    tc_fence_after();
    if (warp == 1) {
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(TMEM_COLS) : "memory");
        else tmem_dealloc_cta1(tmem_base, TMEM_COLS);
    }
}

// ---- few tokens ------------------------------------------------------------------------------------
static constexpr int I8S_WARPS = 8, I8S_CH = 2;                      // warps per CTA, output channels per warp
// 1536 x 9216 weights: 1 token 3.4 us and 2 tokens 4.6 this way, 5.1 with tensor-core tiles; 4 tokens 4.8 against 4.8,
// 8 tokens 10.3 against 4.8
static constexpr int I8S_TOKENS = 2;

struct I8SmallParams {
    const int8_t *a, *w;
    const float *a_scale, *w_scale, *bias;
    const int32_t* out_idx;
    void* out;
    long long out_stride;
    int M, N, K, out_rows;
    int* status;
};

template <int MR, int OT>
__global__ void __launch_bounds__(I8S_WARPS * 32)
linear_int8_small_kernel(const __grid_constant__ I8SmallParams P) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n0 = (blockIdx.x * I8S_WARPS + warp) * I8S_CH;
    pdl_enter();
    if (n0 >= P.N) return;
    int acc[I8S_CH][MR] = {};
    const int chunks = P.K >> 4;
#pragma unroll 4
    for (int c = lane; c < chunks; c += 32) {
        uint4 w[I8S_CH];
#pragma unroll
        for (int i = 0; i < I8S_CH; ++i)
            w[i] = n0 + i < P.N ? ld_nc_v4(P.w + (long long)(n0 + i) * P.K + c * 16) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            const uint4 a = m < P.M ? __ldg((const uint4*)(P.a + (long long)m * P.K + c * 16)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < I8S_CH; ++i) {
                acc[i][m] = __dp4a((int)w[i].x, (int)a.x, acc[i][m]);
                acc[i][m] = __dp4a((int)w[i].y, (int)a.y, acc[i][m]);
                acc[i][m] = __dp4a((int)w[i].z, (int)a.z, acc[i][m]);
                acc[i][m] = __dp4a((int)w[i].w, (int)a.w, acc[i][m]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int i = 0; i < I8S_CH; ++i) {
            const int sum = __reduce_add_sync(0xFFFFFFFFu, acc[i][m]);
            const int n = n0 + i;
            if (lane == (m * I8S_CH + i) && m < P.M && n < P.N) {
                const int d = P.out_idx ? __ldg(P.out_idx + m) : m;
                if (d >= P.out_rows) { atomicCAS(P.status, 0, OC_ERR_INVALID_ARG); }
                else if (d >= 0) {
                    const float v = fmaf((float)sum * __ldg(P.a_scale + m), __ldg(P.w_scale + n), P.bias ? __ldg(P.bias + n) : 0.0f);
                    const long long at = (long long)d * P.out_stride + n;
                    if (OT == OC_DTYPE_F32) ((float*)P.out)[at] = v;
                    else ((uint16_t*)P.out)[at] = (uint16_t)pack_bf16x2(v, 0.0f);
                }
            }
        }
}

template <int OT>
static void launch_small(const I8SmallParams& P, cudaStream_t s) {
    const dim3 grid((unsigned)((P.N + I8S_WARPS * I8S_CH - 1) / (I8S_WARPS * I8S_CH)));
    if (P.M == 1) OC_LAUNCH((linear_int8_small_kernel<1, OT>), grid, I8S_WARPS * 32, 0, s, P);
    else OC_LAUNCH((linear_int8_small_kernel<2, OT>), grid, I8S_WARPS * 32, 0, s, P);
}

// ---- host side -------------------------------------------------------------------------------------
typedef CUresult (*I8EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                               const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                               CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static I8EncodeFn i8_encode_fn() {
    static I8EncodeFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = (I8EncodeFn)p;
        else
            cudaGetLastError();
    });
    return fn;
}
static bool i8_encode(I8EncodeFn enc, CUtensorMap* map, const void* p, int64_t K, int64_t rows, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)K};
    const cuuint32_t box[2] = {(cuuint32_t)I8_BK, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static bool i8_encode_out(I8EncodeFn enc, CUtensorMap* map, void* p, int dtype, int64_t N, int64_t M, int64_t stride) {
    const bool f32 = dtype == OC_DTYPE_F32;
    const cuuint64_t dims[2] = {(cuuint64_t)N, (cuuint64_t)M};
    const cuuint64_t strides[1] = {(cuuint64_t)stride * (f32 ? 4 : 2)};
    const cuuint32_t box[2] = {(cuuint32_t)(f32 ? I8_SEG / 4 : I8_SEG / 2), 32}, estr[2] = {1, 1};
    return strides[0] < (1ull << 40) &&
           enc(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int N_TILE, bool PAIR, bool RES, int OT>
static oc_status launch_tiles_as(oc_ctx* ctx, I8Params& P, cudaStream_t s) {
    constexpr int W_BYTES = (PAIR ? N_TILE / 2 : N_TILE) * I8_BK, STAGE_BYTES = RES ? I8_A_BYTES : I8_A_BYTES + W_BYTES;
    constexpr int REST = I8_EPI_WARPS * I8_OUT_STAGE + 2 * N_TILE * 4 + (2 * I8_STAGES_MAX + 7) * 8 + 16;
    const int w_bytes = RES ? P.kblocks * W_BYTES : 0, fit = (227 * 1024 - REST - w_bytes) / STAGE_BYTES;
    const int stages = fit < I8_STAGES_MAX ? fit : I8_STAGES_MAX, smem = w_bytes + stages * STAGE_BYTES + REST;
    static PerDeviceOnce once;                       // (the context's device is current here)
    auto* kernel = linear_int8_kernel<N_TILE, PAIR, RES, OT>;
    if (!once.ensure(ctx->device, [&] {
            const bool ok = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024) == cudaSuccess;
            if (!ok) cudaGetLastError();
            return ok;
        })) return OC_ERR_CUDA;
    P.n_stages = stages;
    const long long tiles = (long long)P.m_tiles * P.n_tiles, walkers = PAIR ? ctx->sm_count / 2 : ctx->sm_count;
    const unsigned grid = (unsigned)(tiles < walkers ? tiles : walkers) * (PAIR ? 2u : 1u);
    if (RES) {
        // each row of walkers takes its share of the rows, the walkers left over the rest
        P.rows_of_walkers = (int)(walkers / P.n_tiles);
        const long long share = (tiles + walkers - 1) / walkers * P.rows_of_walkers;
        P.main_rows = (int)(share < P.m_tiles && walkers % P.n_tiles ? share : (P.rows_of_walkers ? P.m_tiles : 0));
    }
    LaunchScope scope(ctx, OC_K_LINEAR_I8, s);
    PdlLaunch l(dim3(grid), dim3(I8_THREADS), (size_t)smem, s, PAIR ? 2u : 0u);
    cudaLaunchKernelEx(&l.cfg, kernel, (const I8Params&)P);
    return last_launch_status();
}
template <int N_TILE, bool PAIR, bool RES>
static oc_status launch_tiles(oc_ctx* ctx, I8Params& P, int out_dtype, cudaStream_t s) {
    return out_dtype == OC_DTYPE_F32 ? launch_tiles_as<N_TILE, PAIR, RES, OC_DTYPE_F32>(ctx, P, s)
                                     : launch_tiles_as<N_TILE, PAIR, RES, OC_DTYPE_BF16>(ctx, P, s);
}

oc_status launch_linear_int8(oc_ctx* ctx, const int8_t* a, const float* a_scale, int64_t M, int64_t K, const int8_t* w,
                             const float* w_scale, int64_t N, const float* bias, void* out, int out_dtype, int64_t out_rows,
                             int64_t out_stride, const int32_t* out_idx, cudaStream_t s) {
    if (M <= I8S_TOKENS) {
        I8SmallParams P;
        P.a = a; P.w = w; P.a_scale = a_scale; P.w_scale = w_scale; P.bias = bias; P.out_idx = out_idx; P.out = out;
        P.out_stride = out_stride; P.M = (int)M; P.N = (int)N; P.K = (int)K; P.out_rows = (int)out_rows; P.status = ctx->d_status;
        LaunchScope scope(ctx, OC_K_LINEAR_I8, s);
        if (out_dtype == OC_DTYPE_F32) launch_small<OC_DTYPE_F32>(P, s);
        else launch_small<OC_DTYPE_BF16>(P, s);
        return last_launch_status();
    }
    I8EncodeFn enc = i8_encode_fn();
    if (!enc) return OC_ERR_UNSUPPORTED;
    I8Params P;
    memset(&P, 0, sizeof(P));
    // The form whose waves over the device take the least time: a fixed part, and for each wave its steps of 128 bytes
    // of K or its output, whichever is longer.  The figures (us) were read off 22 shapes of 1 to 14400 tokens timed
    // with every form; they name the fastest, or one within 7 %, on all of them (1024 x 1536 x 1536: 5.9 us in
    // 128 x 128 tiles, 8.4 in pairs; 2048 x 1536 x 4608: 16.0 against 13.7; 64 x 1536 x 9216: 5.3 against 5.0 in
    // 128 x 64; 128 x 1536 x 1536: 5.4 against 4.7 in 128 x 32).
    struct Form { int rows, cols, w_rows, per_walker; double fixed, step, tile; };
    static const Form forms[4] = {{256, 256, 128, 2, 3.5, 0.417, 2.2}, {128, 128, 128, 1, 2.5, 0.28, 1.4},
                                  {128, 64, 64, 1, 2.5, 0.206, 1.05}, {128, 32, 32, 1, 2.5, 0.19, 0.9}};
    int best = 1;
    double best_cost = 1e300;
    const int kblocks = (int)((K + I8_BK - 1) / I8_BK);
    for (int f = M > 128 ? 0 : 1; f < 4; ++f) {
        const long long tiles = ((M + forms[f].rows - 1) / forms[f].rows) * ((N + forms[f].cols - 1) / forms[f].cols);
        const long long walkers = ctx->sm_count / forms[f].per_walker;
        const double cost = forms[f].fixed + (double)((tiles + walkers - 1) / walkers) * std::max(kblocks * forms[f].step, forms[f].tile);
        if (cost < best_cost) { best_cost = cost; best = f; }
    }
    const Form& F = forms[best];
    // (the rows of a tile that no token has are left as they are in shared memory: their sums are not stored)
    const int a_box = M < I8_BM ? (int)(M + 7) / 8 * 8 : I8_BM;
    P.a_bytes = a_box * I8_BK;
    if (!i8_encode(enc, &P.mapA, a, K, M, a_box) || !i8_encode(enc, &P.mapW, w, K, N, F.w_rows)) return OC_ERR_UNSUPPORTED;
    P.a_scale = a_scale; P.w_scale = w_scale; P.bias = bias; P.out_idx = out_idx; P.out = out; P.out_stride = out_stride;
    P.M = (int)M; P.N = (int)N; P.out_rows = (int)out_rows; P.kblocks = kblocks; P.status = ctx->d_status;
    P.wide = ((uintptr_t)out | (uint64_t)out_stride * (out_dtype == OC_DTYPE_F32 ? 4u : 2u)) % 16 == 0;
    // (a TMA store clips at 16 bytes, not at an element: a row's end in mid-piece is stored by hand)
    P.tma_out = P.wide && !out_idx && N * (out_dtype == OC_DTYPE_F32 ? 4 : 2) % 16 == 0 &&
                i8_encode_out(enc, &P.mapOut, out, out_dtype, N, M, out_stride);
    const long long mt = (M + F.rows - 1) / F.rows, nt = (N + F.cols - 1) / F.cols;
    if (mt * nt > 0x7FFFFFFFll - 1024) return OC_ERR_UNSUPPORTED;
    P.m_tiles = (int)mt; P.n_tiles = (int)nt;
    switch (best) {
        case 0:
            // W stays in shared memory where a column's share leaves room for five stages of A, and there are tiles
            // enough to use it on
            if (kblocks <= 7 && mt * nt >= 4 * (ctx->sm_count / 2)) return launch_tiles<256, true, true>(ctx, P, out_dtype, s);
            return launch_tiles<256, true, false>(ctx, P, out_dtype, s);
        case 1: return launch_tiles<128, false, false>(ctx, P, out_dtype, s);
        case 2: return launch_tiles<64, false, false>(ctx, P, out_dtype, s);
        default: return launch_tiles<32, false, false>(ctx, P, out_dtype, s);
    }
}

}  // namespace oc
