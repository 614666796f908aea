// The C-ABI layer: argument validation, context, launch bookkeeping, Layered Cache store, and the
// host-buffer convenience call.  No kernel lives here.
#include <initializer_list>
#include <math.h>
#include <string.h>

#include <new>

#include <algorithm>
#include <cmath>
#include "common.cuh"

namespace oc {

// ---- launch bookkeeping ------------------------------------------------------------------------
static cudaEvent_t take_event(oc_ctx* c) {
    if (!c->free_events.empty()) { cudaEvent_t e = c->free_events.back(); c->free_events.pop_back(); return e; }
    cudaEvent_t e = nullptr;
    if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
    return e;
}

LaunchScope::LaunchScope(oc_ctx* c, int kernel, cudaStream_t stream) : ctx(c), k(kernel), s(stream) {
    ctx->prof[k].launches += 1;
    if (ctx->profile_on) {
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(s, &cap) != cudaSuccess) { cudaGetLastError(); cap = cudaStreamCaptureStatusNone; }
        capturing = cap == cudaStreamCaptureStatusActive;
        e0 = take_event(ctx); e1 = take_event(ctx);
        // in a capture the records become event-record nodes of the graph (external events), so that the
        // bracket is taken again on every replay
        if (e0 && e1) cudaEventRecordWithFlags(e0, s, capturing ? cudaEventRecordExternal : cudaEventRecordDefault);
    }
}
LaunchScope::~LaunchScope() {
    if (e0 && e1) {
        cudaEventRecordWithFlags(e1, s, capturing ? cudaEventRecordExternal : cudaEventRecordDefault);
        if (capturing) ctx->prof[k].captured.emplace_back(e0, e1);
        else ctx->prof[k].pending.emplace_back(e0, e1);
    } else {
        if (e0) ctx->free_events.push_back(e0);
        if (e1) ctx->free_events.push_back(e1);
    }
}

// ---- geometry ----------------------------------------------------------------------------------
oc_status make_geo(const oc_layout* L, Geo* g) {
    if (!L || !g) return OC_ERR_INVALID_ARG;
    if (L->kind < OC_KIND_TOKEN || L->kind > OC_KIND_BLOCK) return OC_ERR_INVALID_ARG;
    if (L->dtype != OC_DTYPE_F32 && L->dtype != OC_DTYPE_BF16) return OC_ERR_INVALID_ARG;
    if (L->B <= 0 || L->T <= 0 || L->H <= 0 || L->W <= 0 || L->C <= 0) return OC_ERR_INVALID_ARG;
    if (!(L->eps >= 0.0f) || !isfinite(L->eps)) return OC_ERR_INVALID_ARG;
    g->kind = L->kind; g->dtype = L->dtype; g->B = L->B; g->T = L->T; g->H = L->H; g->W = L->W; g->C = L->C;
    g->sy = L->sy; g->sx = L->sx; g->oy = L->oy; g->ox = L->ox; g->gy = L->gy; g->gx = L->gx;
    g->self_match = L->self_match ? 1 : 0; g->frame_stat = L->frame_stat; g->eps = L->eps;
    g->elem_bytes = L->dtype == OC_DTYPE_F32 ? 4 : 2;
    if (((int64_t)L->C * g->elem_bytes) % 16 != 0) return OC_ERR_ALIGNMENT;
    const int64_t n_tok = (int64_t)L->B * L->T * L->H * L->W;
    if (n_tok > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
    if (L->kind == OC_KIND_FRAME) {
        if (L->frame_stat != OC_FRAME_MEAN_POS_COS && L->frame_stat != OC_FRAME_FLAT_COS) return OC_ERR_INVALID_ARG;
        // patch-local Frame Cache (Section 3.3): gy x gx equal patches per frame, one group per
        // patch position of a batch element; a layout that leaves gy = gx = 0 means whole frames
        g->gy = L->gy > 0 ? L->gy : 1; g->gx = L->gx > 0 ? L->gx : 1;
        if (L->gy < 0 || L->gx < 0 || L->H % g->gy != 0 || L->W % g->gx != 0) return OC_ERR_INVALID_ARG;
        g->sy = g->sx = 1; g->oy = g->ox = 0; g->self_match = 0;
        g->Hp = L->H / g->gy; g->Wp = L->W / g->gx; g->Hs = g->Hp; g->Ws = g->Wp;
        g->n_groups = (int64_t)L->B * g->gy * g->gx; g->units_per_group = L->T; g->reps_per_group = (L->T + 1) / 2;
        g->n_units = g->n_groups * L->T;
        if (g->n_units > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
        return OC_OK;
    }
    if (L->gy <= 0 || L->gx <= 0) return OC_ERR_INVALID_ARG;
    if (L->kind == OC_KIND_BLOCK && L->self_match) return OC_ERR_INVALID_ARG;
    if (L->H % L->gy != 0 || L->W % L->gx != 0) return OC_ERR_INVALID_ARG;
    g->Hp = L->H / L->gy; g->Wp = L->W / L->gx;
    if (g->self_match) {
        if (L->gy != 1 || L->gx != 1) return OC_ERR_UNSUPPORTED;
        g->sy = g->sx = 1; g->oy = g->ox = 0;
        g->Hs = g->Hp; g->Ws = g->Wp;
    } else {
        if (L->sy <= 0 || L->sx <= 0 || (int64_t)L->sy * L->sx < 2) return OC_ERR_INVALID_ARG;
        if (L->oy < 0 || L->oy >= L->sy || L->ox < 0 || L->ox >= L->sx) return OC_ERR_INVALID_ARG;
        if (g->Hp % L->sy != 0 || g->Wp % L->sx != 0) return OC_ERR_INVALID_ARG;
        g->Hs = g->Hp / L->sy; g->Ws = g->Wp / L->sx;
    }
    if (L->kind == OC_KIND_TOKEN) {
        g->n_groups = (int64_t)L->B * L->T * L->gy * L->gx;
        g->units_per_group = (int64_t)g->Hp * g->Wp;
        g->reps_per_group = (int64_t)g->Hs * g->Ws;
    } else {
        // a patch confines the selection; matching stays inside the sy x sx neighbourhood, which a
        // patch never cuts (Hp % sy == 0, Wp % sx == 0 above)
        g->n_groups = (int64_t)L->B * L->gy * L->gx;
        g->units_per_group = (int64_t)g->Hp * g->Wp;
        g->reps_per_group = (int64_t)g->Hs * g->Ws;
        if ((int64_t)L->H * L->W * L->B > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
    }
    g->n_units = g->n_groups * g->units_per_group;
    return OC_OK;
}

GroupMap make_group_map(const Geo& g) {
    GroupMap m;
    m.kind = g.kind; m.self_match = g.self_match; m.H = g.H; m.W = g.W; m.gy = g.gy; m.gx = g.gx;
    m.Hp = g.Hp; m.Wp = g.Wp; m.sy = g.sy; m.sx = g.sx; m.oy = g.oy; m.ox = g.ox;
    m.units_per_group = (int)g.units_per_group;
    m.frames = nullptr; m.n_reuse_single = 0;
    return m;
}

static oc_status check_rows(const oc_rows* r) {
    if (!r) return OC_ERR_INVALID_ARG;
    if (r->seg_bytes <= 0 || r->n_seg <= 0 || r->unit_pitch <= 0 || r->units_per_outer <= 0) return OC_ERR_INVALID_ARG;
    if (r->seg_stride < 0 || r->outer_pitch < 0) return OC_ERR_INVALID_ARG;
    if ((r->seg_bytes | r->seg_stride | r->unit_pitch | r->outer_pitch) & 15) return OC_ERR_ALIGNMENT;
    if (r->n_seg > 65535 || r->seg_bytes * r->n_seg > (1ll << 34)) return OC_ERR_UNSUPPORTED;
    return OC_OK;
}

static inline bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

}  // namespace oc

using namespace oc;

extern "C" {

const char* oc_status_str(oc_status s) {
    switch (s) {
        case OC_OK: return "OC_OK";
        case OC_ERR_INVALID_ARG: return "OC_ERR_INVALID_ARG";
        case OC_ERR_ALIGNMENT: return "OC_ERR_ALIGNMENT";
        case OC_ERR_UNSUPPORTED: return "OC_ERR_UNSUPPORTED";
        case OC_ERR_WORKSPACE: return "OC_ERR_WORKSPACE";
        case OC_ERR_CUDA: return "OC_ERR_CUDA";
        case OC_ERR_TIMEOUT: return "OC_ERR_TIMEOUT";
        case OC_ERR_OOM: return "OC_ERR_OOM";
        case OC_CACHE_MISS: return "OC_CACHE_MISS";
        default: return "OC_UNKNOWN_STATUS";
    }
}

const char* oc_kernel_name(int k) {
    static const char* names[OC_K_COUNT] = {"norms", "match_tc", "match_simt", "match_finalize", "frame_pair",
                                            "frame_finalize", "block_partial", "block_finalize", "select",
                                            "gather", "restore", "copy", "linear", "block_norm", "rope", "quantize",
                                            "linear_int8", "kv_put", "kv_get", "attention"};
    return (k >= 0 && k < OC_K_COUNT) ? names[k] : "unknown";
}

oc_status oc_layout_check(const oc_layout* layout) {
    Geo g;
    return make_geo(layout, &g);
}

oc_status oc_layout_counts(const oc_layout* layout, int64_t* n_groups, int64_t* units_per_group,
                           int64_t* reps_per_group) {
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    if (n_groups) *n_groups = g.n_groups;
    if (units_per_group) *units_per_group = g.units_per_group;
    if (reps_per_group) *reps_per_group = g.reps_per_group;
    return OC_OK;
}

oc_status oc_match_workspace_bytes(const oc_layout* layout, size_t* bytes) {
    if (!bytes) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    *bytes = match_workspace_bytes(g);
    return OC_OK;
}

oc_status oc_rows_from_layout(const oc_layout* layout, int channels, int elem_bytes, oc_rows* rows) {
    if (!rows || channels <= 0 || (elem_bytes != 1 && elem_bytes != 2 && elem_bytes != 4 && elem_bytes != 8))
        return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    const int64_t cb = (int64_t)channels * elem_bytes;
    if (cb % 16 != 0) return OC_ERR_ALIGNMENT;
    const int64_t P = (int64_t)g.H * g.W;
    if (g.kind == OC_KIND_TOKEN) {
        *rows = oc_rows{cb, 1, 0, cb, (int64_t)1 << 40, 0};
    } else if (g.kind == OC_KIND_FRAME) {
        if (g.gy * g.gx == 1) *rows = oc_rows{P * cb, 1, 0, P * cb, (int64_t)1 << 40, 0};
        // a patch of a frame: Hp segments of Wp*C' elements; the gx patches of a patch row sit side by
        // side and patch rows follow one another at one pitch through frames and batch elements
        else *rows = oc_rows{g.Wp * cb, g.Hp, (int64_t)g.W * cb, g.Wp * cb, g.gx, (int64_t)g.Hp * g.W * cb};
    } else {
        *rows = oc_rows{cb, g.T, P * cb, cb, P, (int64_t)g.T * P * cb};
    }
    return OC_OK;
}

int oc_layer_cache_would_hit(int stored_step, int step, int interval) {
    const long long d = (long long)step - (long long)stored_step;
    return d >= 0 && d < (long long)interval;
}

// ---- context -----------------------------------------------------------------------------------
oc_status oc_create(oc_ctx** out, int device, size_t workspace_bytes) {
    if (!out || device < 0) return OC_ERR_INVALID_ARG;
    *out = nullptr;
    int n = 0;
    if (cudaGetDeviceCount(&n) != cudaSuccess || device >= n) { cudaGetLastError(); return OC_ERR_CUDA; }
    DeviceGuard guard(device);
    if (!guard.ok) return OC_ERR_CUDA;
    cudaDeviceProp prop;
    if (cudaGetDeviceProperties(&prop, device) != cudaSuccess) return OC_ERR_CUDA;
    if (prop.major != 10) return OC_ERR_UNSUPPORTED;      // the kernels are built for sm_100a only
    oc_ctx* c = new (std::nothrow) oc_ctx();
    if (!c) return OC_ERR_OOM;
    c->device = device; c->sm_count = prop.multiProcessorCount;
    if (cudaMalloc(&c->d_status, 256) != cudaSuccess) { delete c; cudaGetLastError(); return OC_ERR_OOM; }
    cudaMemset(c->d_status, 0, 256);
    if (cudaMalloc(&c->d_span, 512 * sizeof(unsigned long long)) != cudaSuccess) {
        cudaFree(c->d_status); delete c; cudaGetLastError(); return OC_ERR_OOM;
    }
    cudaMemset(c->d_span, 0, 512 * sizeof(unsigned long long));
    if (workspace_bytes) {
        if (cudaMalloc(&c->workspace, workspace_bytes) != cudaSuccess) {
            cudaGetLastError();
            cudaFree(c->d_span); cudaFree(c->d_status); delete c;
            return OC_ERR_OOM;
        }
        c->workspace_bytes = workspace_bytes;
    }
    *out = c;
    return OC_OK;
}

oc_status oc_destroy(oc_ctx* c) {
    if (!c) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    cudaDeviceSynchronize();
    for (auto& kv : c->layers) cudaFree(kv.second.ptr);
    for (int k = 0; k < OC_K_COUNT; ++k) {
        for (auto& p : c->prof[k].pending) { cudaEventDestroy(p.first); cudaEventDestroy(p.second); }
        for (auto& p : c->prof[k].captured) { cudaEventDestroy(p.first); cudaEventDestroy(p.second); }
    }
    for (auto e : c->free_events) cudaEventDestroy(e);
    cudaFree(c->stage);
    cudaFree(c->workspace);
    for (auto e : c->chunk_events) cudaEventDestroy(e);
    if (c->copy_stream) cudaStreamDestroy(c->copy_stream);
    cudaFree(c->d_span);
    cudaFree(c->d_status);
    delete c;
    return cuda_ok(cudaGetLastError());
}

oc_status oc_device_status(oc_ctx* c, int* code) {
    if (!c || !code) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    int v = 0;
    if (cudaDeviceSynchronize() != cudaSuccess) return OC_ERR_CUDA;
    if (cudaMemcpy(&v, c->d_status, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) return OC_ERR_CUDA;
    if (v != 0) cudaMemset(c->d_status, 0, sizeof(int));
    *code = v;
    return OC_OK;
}

oc_status oc_selftest_per_device_once(int n_devices, int n_rounds, int fail_dev, int* runs, int* ok) {
    if (n_devices < 1 || n_devices > oc::PerDeviceOnce::MAX_DEV || n_rounds < 1 || !runs || !ok) return OC_ERR_INVALID_ARG;
    oc::PerDeviceOnce once;
    for (int d = 0; d < n_devices; ++d) { runs[d] = 0; ok[d] = 0; }
    for (int r = 0; r < n_rounds; ++r)
        for (int d = 0; d < n_devices; ++d)
            if (once.ensure(d, [&] { ++runs[d]; return d != fail_dev; })) ++ok[d];
    return OC_OK;
}

oc_status oc_selftest_bounded_wait(oc_ctx* c, unsigned int limit_us, void* stream) {
    if (!c || limit_us == 0 || limit_us > 1000000u) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_bounded_wait_selftest(c, (unsigned long long)limit_us * 1000ull, (cudaStream_t)stream);
}

oc_status oc_tc_plan_override(oc_ctx* c, int on, int pair, int tiles_per_cta, int pieces_per_row, int single_accumulator,
                              int candidates_resident) {
    if (!c) return OC_ERR_INVALID_ARG;
    if (on && ((pair != 0 && pair != 1) || (tiles_per_cta != 1 && tiles_per_cta != 2) || pieces_per_row < 1))
        return OC_ERR_INVALID_ARG;
    c->tc_plan_forced = on != 0;
    c->tc_plan_pair = pair; c->tc_plan_tiles = tiles_per_cta; c->tc_plan_pieces = pieces_per_row;
    c->tc_plan_no_narrow = single_accumulator ? 1 : 0;
    c->tc_plan_a_res = candidates_resident < 0 ? -1 : (candidates_resident ? 1 : 0);
    return OC_OK;
}

oc_status oc_tc_plan_describe(oc_ctx* c, const oc_layout* layout, int32_t* out) {
    if (!c || !out) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return tc_plan_describe(c, g, out);
}

oc_status oc_profile_enable(oc_ctx* c, int on) {
    if (!c) return OC_ERR_INVALID_ARG;
    c->profile_on = on == 1;
    c->span_on = on == 2;
    return OC_OK;
}

static void drain(oc_ctx* c, int k) {
    for (auto& p : c->prof[k].pending) {
        float ms = 0.f;
        if (cudaEventSynchronize(p.second) == cudaSuccess && cudaEventElapsedTime(&ms, p.first, p.second) == cudaSuccess)
            c->prof[k].total_ms += ms;
        c->free_events.push_back(p.first); c->free_events.push_back(p.second);
    }
    c->prof[k].pending.clear();
}

oc_status oc_profile_reset(oc_ctx* c) {
    if (!c) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    for (int k = 0; k < OC_K_COUNT; ++k) { drain(c, k); c->prof[k].launches = 0; c->prof[k].total_ms = 0.0; }
    c->span_count = 0;
    return OC_OK;
}

oc_status oc_profile_read(oc_ctx* c, int k, int64_t* launches, double* total_ms) {
    if (!c || k < 0 || k >= OC_K_COUNT) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    drain(c, k);
    if (launches) *launches = c->prof[k].launches;
    if (total_ms) *total_ms = c->prof[k].total_ms;
    return OC_OK;
}

oc_status oc_profile_captured_read(oc_ctx* c, int k, int64_t* launches, double* total_ms) {
    if (!c || k < 0 || k >= OC_K_COUNT) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    double sum = 0.0;
    int64_t n = 0;
    for (auto& p : c->prof[k].captured) {
        float ms = 0.f;
        if (cudaEventSynchronize(p.second) == cudaSuccess && cudaEventElapsedTime(&ms, p.first, p.second) == cudaSuccess) {
            sum += ms; ++n;
        } else {
            cudaGetLastError();                  // captured but its graph has not run yet
        }
    }
    if (launches) *launches = n;
    if (total_ms) *total_ms = sum;
    return OC_OK;
}

oc_status oc_profile_span_read(oc_ctx* c, int k, int64_t* launches, double* total_ms) {
    if (!c || k < 0 || k >= OC_K_COUNT) return OC_ERR_INVALID_ARG;
    if (k != OC_K_MATCH_TC) return OC_ERR_UNSUPPORTED;
    DeviceGuard guard(c->device);
    if (!guard.ok || cudaDeviceSynchronize() != cudaSuccess) return OC_ERR_CUDA;
    const long long n = c->span_count < 256 ? c->span_count : 256;
    std::vector<unsigned long long> h(512);
    if (cudaMemcpy(h.data(), c->d_span, 512 * sizeof(unsigned long long), cudaMemcpyDeviceToHost) != cudaSuccess)
        return OC_ERR_CUDA;
    double ns = 0.0;
    long long counted = 0;
    for (long long i = 0; i < n; ++i) {
        const long long slot = (c->span_count - 1 - i) & 255;
        const unsigned long long entry = ~h[2 * slot], exit = h[2 * slot + 1];
        if (h[2 * slot] != 0 && exit >= entry) { ns += (double)(exit - entry); ++counted; }
    }
    if (launches) *launches = counted;
    if (total_ms) *total_ms = ns * 1e-6;
    return OC_OK;
}

// ---- hot path ----------------------------------------------------------------------------------
oc_status oc_match(oc_ctx* c, const oc_layout* layout, const void* x, float* best_sim, int32_t* best_idx,
                   float* aux_sim, float* pair_sim, void* stream) {
    if (!c || !x || !best_sim || !best_idx) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    if (misaligned(x)) return OC_ERR_ALIGNMENT;
    if (pair_sim && g.kind != OC_KIND_FRAME) return OC_ERR_INVALID_ARG;
    if (aux_sim && g.kind == OC_KIND_BLOCK) return OC_ERR_INVALID_ARG;
    if (match_workspace_bytes(g) > c->workspace_bytes) return OC_ERR_WORKSPACE;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    if (g.kind == OC_KIND_TOKEN) return launch_match_token(c, g, x, best_sim, best_idx, aux_sim, s);
    if (g.kind == OC_KIND_FRAME) return launch_match_frame(c, g, x, best_sim, best_idx, aux_sim, pair_sim, s);
    return launch_match_block(c, g, x, best_sim, best_idx, s);
}

oc_status oc_match_frame_levels(oc_ctx* c, const oc_layout* layout, const void* x, int n_levels,
                                const int32_t* grids, float* best_sim, int32_t* best_idx, float* pos_sim,
                                float* pair_sim, void* stream) {
    if (!c || !x || !best_sim || !best_idx || !grids || n_levels < 1 || n_levels > OC_MAX_FRAME_LEVELS)
        return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    if (g.kind != OC_KIND_FRAME) return OC_ERR_INVALID_ARG;
    long long units = 0;
    for (int l = 0; l < n_levels; ++l) {
        const int gy = grids[2 * l], gx = grids[2 * l + 1];
        if (gy <= 0 || gx <= 0 || g.gy % gy != 0 || g.gx % gx != 0) return OC_ERR_INVALID_ARG;
        units += (long long)g.B * g.T * gy * gx;
    }
    if (units > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
    if (misaligned(x)) return OC_ERR_ALIGNMENT;
    if (match_workspace_bytes(g) > c->workspace_bytes) return OC_ERR_WORKSPACE;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_match_frame_levels(c, g, x, n_levels, grids, best_sim, best_idx, pos_sim, pair_sim, (cudaStream_t)stream);
}

oc_status oc_linear_gather_scatter(oc_ctx* c, const void* a, int64_t a_rows, int64_t K, const int32_t* a_idx,
                                   int64_t n_rows, const void* w, int64_t N, void* out, int64_t out_rows,
                                   const int32_t* out_idx, void* stream) {
    if (!c || !a || !w || !out || a_rows <= 0 || K <= 0 || N <= 0 || n_rows < 0 || out_rows <= 0) return OC_ERR_INVALID_ARG;
    if (K % 8 != 0 || N % 8 != 0) return OC_ERR_ALIGNMENT;
    if (misaligned(a) || misaligned(w) || misaligned(out)) return OC_ERR_ALIGNMENT;
    if (!a_idx && n_rows > a_rows) return OC_ERR_INVALID_ARG;
    if (N < 128 || a_rows > 0x7FFFFFFFll || out_rows > 0x7FFFFFFFll || K > 0x7FFFFFFFll || N > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_linear_gs(c, a, a_rows, K, a_idx, n_rows, w, N, out, out_rows, out_idx, (cudaStream_t)stream);
}

// ---- the wrapped block on kept tokens -------------------------------------------------------------
static inline bool float_type(int t) { return t == OC_DTYPE_F32 || t == OC_DTYPE_BF16; }
static inline bool norm_kind(int k) { return k == OC_NORM_NONE || k == OC_NORM_RMS || k == OC_NORM_LAYER; }
static inline bool bad_eps(float e) { return !(e >= 0.0f) || !isfinite(e); }
static const int64_t ROWS_MAX = 0x7FFFFFFFll;

oc_status oc_block_norm(oc_ctx* c, const oc_block_norm_desc* d, const void* x, const void* z, const int32_t* slot_of,
                        const void* cache, void* cache_out, void* out, const void* post_w, const void* post_b,
                        const void* gate, const void* pre_w, const void* pre_b, const void* scale, const void* shift,
                        void* h, float* h_scale, void* stream) {
    if (!c || !d) return OC_ERR_INVALID_ARG;
    if (!float_type(d->dtype) || !float_type(d->param_dtype) || !norm_kind(d->post_norm) || !norm_kind(d->pre_norm)) return OC_ERR_INVALID_ARG;
    if (!float_type(d->h_dtype) && d->h_dtype != OC_DTYPE_I8) return OC_ERR_INVALID_ARG;
    if (bad_eps(d->post_eps) || bad_eps(d->pre_eps) || !isfinite(d->res_scale)) return OC_ERR_INVALID_ARG;
    if (d->n_rows < 0 || d->C <= 0 || d->rows_per_group <= 0 || d->mod_stride < 0 || d->unit_rows <= 0 || d->dense_rows < 0) return OC_ERR_INVALID_ARG;
    if (d->n_rows > ROWS_MAX || d->dense_rows > ROWS_MAX || d->C > ROWS_MAX) return OC_ERR_UNSUPPORTED;
    if (d->n_rows % d->unit_rows != 0 || d->dense_rows % d->unit_rows != 0) return OC_ERR_INVALID_ARG;
    if (d->n_rows == 0) return OC_OK;                                       // (empty tensors have no addresses)
    // (so have z and h where every unit is reused: the cache then says that there is a z)
    const bool none_dense = slot_of && d->dense_rows == 0, empty_z = none_dense && !z && cache;
    if (!x || (!out && !h && !cache_out && !none_dense)) return OC_ERR_INVALID_ARG;
    if (!z && !empty_z && (cache || cache_out || gate || post_w || post_b || d->post_norm != OC_NORM_NONE)) return OC_ERR_INVALID_ARG;
    if (z && slot_of && !cache) return OC_ERR_INVALID_ARG;                  // reused rows would come from nowhere
    if ((z || h) && !slot_of && d->dense_rows < d->n_rows) return OC_ERR_INVALID_ARG;
    if (h && d->h_dtype == OC_DTYPE_I8 && !h_scale) return OC_ERR_INVALID_ARG;
    if (out && (out == z || out == cache || out == cache_out)) return OC_ERR_INVALID_ARG;
    if (cache_out && (cache_out == x || cache_out == z)) return OC_ERR_INVALID_ARG;
    if (h && (h == x || h == z || h == cache || h == cache_out || h == out)) return OC_ERR_INVALID_ARG;
    const int64_t eb = d->dtype == OC_DTYPE_F32 ? 4 : 2;
    if (d->C * eb % 16 != 0 || (h && d->h_dtype == OC_DTYPE_I8 && d->C % 16 != 0)) return OC_ERR_ALIGNMENT;
    const void* rows[] = {x, z, cache, cache_out, out, h};
    for (const void* p : rows) if (p && misaligned(p)) return OC_ERR_ALIGNMENT;
    // parameters are read as many elements at a time as 16 bytes of a row hold
    const int64_t pb = d->param_dtype == OC_DTYPE_F32 ? 4 : 2, param_align = std::min<int64_t>(16, 16 / eb * pb);
    const void* params[] = {post_w, post_b, gate, pre_w, pre_b, scale, shift};
    for (const void* p : params) if ((uintptr_t)p & (uintptr_t)(param_align - 1)) return OC_ERR_ALIGNMENT;
    if ((gate || scale || shift) && d->mod_stride * pb % param_align != 0) return OC_ERR_ALIGNMENT;
    if (((uintptr_t)slot_of & 3u) || ((uintptr_t)h_scale & 3u)) return OC_ERR_ALIGNMENT;
    if (!out && !h && !cache_out) return OC_OK;                             // the rows of no unit
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    // (no row of an empty z is read: any address stands for it)
    return launch_block_norm(c, *d, x, empty_z ? cache : z, slot_of, cache, cache_out, out, post_w, post_b, gate, pre_w, pre_b, scale, shift,
                             h, h_scale, (cudaStream_t)stream);
}

// Sizes and axes of a rotation; the number of (cos, sin) pairs of its table.
static oc_status check_rope(const oc_rope_desc* d, int64_t* table_pairs) {
    if (!d || !float_type(d->dtype) || d->head_dim <= 0 || (d->pairing != OC_ROPE_ADJACENT && d->pairing != OC_ROPE_HALVES)) return OC_ERR_INVALID_ARG;
    int64_t rot = 0, n = 0, grid = 1;
    for (int a = 0; a < 3; ++a) {
        if (d->axis_dims[a] < 0 || d->axis_dims[a] % 2 != 0 || d->axis_len[a] < 1) return OC_ERR_INVALID_ARG;
        rot += d->axis_dims[a];
        n += (int64_t)d->axis_len[a] * (d->axis_dims[a] / 2);
        if (grid <= ROWS_MAX) grid *= d->axis_len[a];
    }
    if (rot == 0 || rot > d->head_dim) return OC_ERR_INVALID_ARG;
    if (n > ROWS_MAX || grid > ROWS_MAX) return OC_ERR_UNSUPPORTED;
    *table_pairs = n;
    return OC_OK;
}

oc_status oc_rope_table_size(const oc_rope_desc* d, int64_t* n_floats) {
    int64_t n;
    if (!n_floats) return OC_ERR_INVALID_ARG;
    oc_status st = check_rope(d, &n);
    if (st != OC_OK) return st;
    *n_floats = 2 * n;
    return OC_OK;
}

oc_status oc_rope_table(const oc_rope_desc* d, double theta, float* table) {
    int64_t n;
    if (!table || !(theta > 0.0) || !std::isfinite(theta)) return OC_ERR_INVALID_ARG;
    oc_status st = check_rope(d, &n);
    if (st != OC_OK) return st;
    for (int a = 0; a < 3; ++a)
        for (int p = 0; p < d->axis_len[a]; ++p)
            for (int j = 0; j < d->axis_dims[a] / 2; ++j) {
                const double angle = p * std::pow(theta, -2.0 * j / d->axis_dims[a]);
                *table++ = (float)std::cos(angle);
                *table++ = (float)std::sin(angle);
            }
    return OC_OK;
}

oc_status oc_rope(oc_ctx* c, const oc_rope_desc* d, const float* table, const int32_t* idx, const int32_t* pos, const void* q,
                  void* q_out, const float* q_w, const void* k, void* k_out, const float* k_w, void* stream) {
    if (!c) return OC_ERR_INVALID_ARG;
    int64_t n;
    oc_status st = check_rope(d, &n);
    if (st != OC_OK) return st;
    if (d->q_heads <= 0 || (k && d->k_heads <= 0) || d->n_rows < 0 || d->rows_per_batch <= 0 || d->unit_rows <= 0) return OC_ERR_INVALID_ARG;
    if (d->n_rows == 0) return OC_OK;                                       // (empty tensors have no addresses)
    if (!table || !q || !q_out) return OC_ERR_INVALID_ARG;
    if ((k != nullptr) != (k_out != nullptr) || (idx && pos)) return OC_ERR_INVALID_ARG;
    if ((q_w != nullptr) != (k_w != nullptr) && k) return OC_ERR_INVALID_ARG;
    if (k_w && !k) return OC_ERR_INVALID_ARG;
    if (q_w && bad_eps(d->eps)) return OC_ERR_INVALID_ARG;
    const oc_rope_view* views[4] = {&d->q, &d->q_out, &d->k, &d->k_out};
    for (int i = 0; i < (k ? 4 : 2); ++i)
        if (views[i]->batch_stride < 0 || views[i]->row_stride < 0 || views[i]->head_stride < 0) return OC_ERR_INVALID_ARG;
    // (several heads, rows or batch elements of an output cannot lie in one place)
    for (int i = 1; i < (k ? 4 : 2); i += 2) {
        const oc_rope_view& o = *views[i];
        if (((i == 1 ? d->q_heads : d->k_heads) > 1 && o.head_stride == 0) || (std::min(d->rows_per_batch, d->n_rows) > 1 && o.row_stride == 0) ||
            (d->n_rows > d->rows_per_batch && o.batch_stride == 0)) return OC_ERR_INVALID_ARG;
    }
    if (d->n_rows > ROWS_MAX || d->rows_per_batch > ROWS_MAX || d->unit_rows > ROWS_MAX || d->q_heads > 65535 || d->k_heads > 65535) return OC_ERR_UNSUPPORTED;
    if (((uintptr_t)table & 7u) || ((uintptr_t)idx & 3u) || ((uintptr_t)pos & 3u) || ((uintptr_t)q_w & 3u) || ((uintptr_t)k_w & 3u)) return OC_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_rope(c, *d, table, idx, pos, q, q_out, q_w, k, k_out, k_w, (cudaStream_t)stream);
}

oc_status oc_quantize_rows(oc_ctx* c, const void* x, int dtype, int64_t x_rows, int64_t x_stride, const int32_t* idx,
                           int64_t n_rows, int64_t K, int8_t* q, float* scale, void* stream) {
    if (!c || !float_type(dtype) || n_rows < 0 || K <= 0 || x_rows < 0 || x_stride < K) return OC_ERR_INVALID_ARG;
    if (n_rows == 0) return OC_OK;                                          // (empty tensors have no addresses)
    if (!x || !q || !scale || (!idx && n_rows > x_rows)) return OC_ERR_INVALID_ARG;
    if (n_rows > ROWS_MAX || x_rows > ROWS_MAX || K > ROWS_MAX) return OC_ERR_UNSUPPORTED;
    if (K % 16 != 0 || x_stride * (dtype == OC_DTYPE_F32 ? 4 : 2) % 16 != 0 || misaligned(x) || misaligned(q)) return OC_ERR_ALIGNMENT;
    if (((uintptr_t)scale & 3u) || ((uintptr_t)idx & 3u)) return OC_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_quantize_rows(c, x, dtype, x_rows, x_stride, idx, n_rows, K, q, scale, (cudaStream_t)stream);
}

oc_status oc_linear_int8(oc_ctx* c, const int8_t* a, const float* a_scale, int64_t M, int64_t K, const int8_t* w,
                         const float* w_scale, int64_t N, const float* bias, void* out, int out_dtype, int64_t out_rows,
                         int64_t out_stride, const int32_t* out_idx, void* stream) {
    if (!c || !float_type(out_dtype) || M < 0 || K <= 0 || N <= 0 || out_rows < 0 || out_stride < N) return OC_ERR_INVALID_ARG;
    if (M == 0) return OC_OK;                                               // (empty tensors have no addresses)
    if (!a || !a_scale || !w || !w_scale || !out || (!out_idx && out_rows < M)) return OC_ERR_INVALID_ARG;
    // (rows and columns are counted in whole tiles of up to 256, in 32 bits)
    if (M > ROWS_MAX - 512 || N > ROWS_MAX - 512 || out_rows > ROWS_MAX || K > 131056) return OC_ERR_UNSUPPORTED;
    if (K % 16 != 0 || misaligned(a) || misaligned(w)) return OC_ERR_ALIGNMENT;
    if ((uintptr_t)out & (out_dtype == OC_DTYPE_F32 ? 3u : 1u)) return OC_ERR_ALIGNMENT;
    if (((uintptr_t)a_scale & 3u) || ((uintptr_t)w_scale & 3u) || ((uintptr_t)bias & 3u) || ((uintptr_t)out_idx & 3u)) return OC_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_linear_int8(c, a, a_scale, M, K, w, w_scale, N, bias, out, out_dtype, out_rows, out_stride, out_idx, (cudaStream_t)stream);
}

// ---- the paged cache and the attention over it ----------------------------------------------------
static inline bool kv_quantised(const oc_kv_desc* k) { return k->dtype == OC_DTYPE_I8 || k->dtype == OC_DTYPE_I4; }
static inline int64_t elem_size(int dtype) { return dtype == OC_DTYPE_F32 ? 4 : 2; }

static oc_status check_kv(const oc_kv_desc* k, bool table) {
    if (!k || (!float_type(k->dtype) && !kv_quantised(k))) return OC_ERR_INVALID_ARG;
    if (k->heads <= 0 || k->head_dim <= 0 || k->n_seqs < 0 || k->seq_rows < 0 || k->page_rows <= 0 || k->n_pages < 0 || k->table_stride < 0) return OC_ERR_INVALID_ARG;
    if (k->head_dim % 8 != 0 || k->page_rows % 16 != 0) return OC_ERR_ALIGNMENT;
    if (k->head_dim > 256 || k->heads > 65535 || k->n_seqs > ROWS_MAX || k->seq_rows > ROWS_MAX || k->page_rows > ROWS_MAX || k->n_pages > ROWS_MAX ||
        k->table_stride > ROWS_MAX) return OC_ERR_UNSUPPORTED;
    if (k->n_seqs * k->seq_rows > ROWS_MAX || k->heads * k->page_rows > ROWS_MAX || k->heads * k->page_rows * k->n_pages > ROWS_MAX) return OC_ERR_UNSUPPORTED;
    if (k->n_pages == 0 && k->n_seqs * k->seq_rows > 0) return OC_ERR_INVALID_ARG;
    const int64_t pages = (k->seq_rows + k->page_rows - 1) / k->page_rows;      // of a sequence
    if (table ? (k->n_seqs > 1 && k->table_stride < pages) : k->n_seqs * pages > k->n_pages) return OC_ERR_INVALID_ARG;
    return OC_OK;
}

oc_status oc_kv_bytes(const oc_kv_desc* k, size_t* pool, size_t* scales) {
    if (!pool || !scales) return OC_ERR_INVALID_ARG;
    // (a stride of 0 between several sequences: a cache without a table)
    oc_status st = check_kv(k, !k || k->table_stride > 0 || k->n_seqs <= 1);
    if (st != OC_OK) return st;
    const size_t vectors = (size_t)(k->n_pages * k->heads * k->page_rows);
    *pool = k->dtype == OC_DTYPE_I4 ? vectors * (size_t)(k->head_dim / 2) : vectors * (size_t)k->head_dim * (k->dtype == OC_DTYPE_I8 ? 1u : (size_t)elem_size(k->dtype));
    *scales = kv_quantised(k) ? vectors * 4 : 0;
    return OC_OK;
}

// Pools and scales of a call (v: whether there is a second tensor).
static oc_status check_pools(const oc_kv_desc* k, const void* k_pool, const float* k_scale, const void* v_pool, const float* v_scale, bool v) {
    if (!k_pool || (v && !v_pool)) return OC_ERR_INVALID_ARG;
    if (kv_quantised(k) ? (!k_scale || (v && !v_scale)) : (k_scale || v_scale)) return OC_ERR_INVALID_ARG;
    if (!v && (v_pool || v_scale)) return OC_ERR_INVALID_ARG;
    if (misaligned(k_pool) || (v && misaligned(v_pool)) || misaligned(k_scale) || misaligned(v_scale)) return OC_ERR_ALIGNMENT;
    return OC_OK;
}

// Strides of rows on the dense side; those of an output lead to a place of its own for every head, row and batch element.
static bool bad_view(const oc_rope_view& w, int64_t heads, int64_t rows, int64_t rows_per_batch, bool output, bool batches) {
    if (w.batch_stride < 0 || w.row_stride < 0 || w.head_stride < 0) return true;
    if (!output) return false;
    return (heads > 1 && w.head_stride == 0) || (std::min(rows, rows_per_batch) > 1 && w.row_stride == 0) || (batches && rows > rows_per_batch && w.batch_stride == 0);
}

// Whether an output begins where another output or an input does.
static bool same_place(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
    for (auto o = outputs.begin(); o != outputs.end(); ++o) {
        if (!*o) continue;
        if (std::find(o + 1, outputs.end(), *o) != outputs.end() || std::find(inputs.begin(), inputs.end(), *o) != inputs.end()) return true;
    }
    return false;
}
static bool same_strides(const oc_rope_view& a, const oc_rope_view& b, int64_t heads, int64_t rows, int64_t rows_per_batch, bool batches) {
    return (heads <= 1 || a.head_stride == b.head_stride) && (std::min(rows, rows_per_batch) <= 1 || a.row_stride == b.row_stride) &&
           (!batches || rows <= rows_per_batch || a.batch_stride == b.batch_stride);
}

static oc_status kv_move(oc_ctx* c, bool put, const oc_kv_desc* cache, const oc_kv_rows* rows, const int32_t* page_table, const int32_t* idx,
                         const void* k, const void* k_pool, const float* k_scale, const void* v, const void* v_pool, const float* v_scale, void* stream) {
    if (!c || !rows || !float_type(rows->dtype) || rows->n_rows < 0 || rows->rows_per_batch <= 0) return OC_ERR_INVALID_ARG;
    oc_status st = check_kv(cache, page_table != nullptr);
    if (st != OC_OK) return st;
    if (!kv_quantised(cache) && cache->dtype != rows->dtype) return OC_ERR_INVALID_ARG;
    if (rows->n_rows == 0) return OC_OK;                                    // (empty tensors have no addresses)
    if (!k || (v != nullptr) != (v_pool != nullptr)) return OC_ERR_INVALID_ARG;
    if (!idx && rows->n_rows > cache->n_seqs * cache->seq_rows) return OC_ERR_INVALID_ARG;
    if (bad_view(rows->k, cache->heads, rows->n_rows, rows->rows_per_batch, !put, true) ||
        (v && bad_view(rows->v, cache->heads, rows->n_rows, rows->rows_per_batch, !put, true))) return OC_ERR_INVALID_ARG;
    if (cache->n_seqs * cache->seq_rows == 0) return OC_OK;                 // (no row can name a token)
    st = check_pools(cache, k_pool, k_scale, v_pool, v_scale, v != nullptr);
    if (st != OC_OK) return st;
    if (k == k_pool || (v && v == v_pool)) return OC_ERR_INVALID_ARG;
    if (v && (put ? v_pool == k_pool || (v_scale && v_scale == k_scale) : v == k)) return OC_ERR_INVALID_ARG;  // (both would be written to one place)
    if (rows->n_rows > ROWS_MAX || rows->rows_per_batch > ROWS_MAX) return OC_ERR_UNSUPPORTED;
    const uintptr_t el = (uintptr_t)elem_size(rows->dtype) - 1;
    if (((uintptr_t)k & el) || ((uintptr_t)v & el) || ((uintptr_t)page_table & 3u) || ((uintptr_t)idx & 3u)) return OC_ERR_ALIGNMENT;
    if (put ? same_place({k_pool, v_pool, k_scale, v_scale}, {k, v, page_table, idx}) : same_place({k, v}, {k_pool, v_pool, k_scale, v_scale, page_table, idx})) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_kv_move(c, put, *cache, *rows, page_table, idx, k, k_pool, k_scale, v, v_pool, v_scale, (cudaStream_t)stream);
}

oc_status oc_kv_put(oc_ctx* c, const oc_kv_desc* cache, const oc_kv_rows* rows, const int32_t* page_table, const int32_t* idx,
                    const void* k, void* k_pool, float* k_scale, const void* v, void* v_pool, float* v_scale, void* stream) {
    return kv_move(c, true, cache, rows, page_table, idx, k, k_pool, k_scale, v, v_pool, v_scale, stream);
}

oc_status oc_kv_get(oc_ctx* c, const oc_kv_desc* cache, const oc_kv_rows* rows, const int32_t* page_table, const int32_t* idx,
                    const void* k_pool, const float* k_scale, void* k, const void* v_pool, const float* v_scale, void* v, void* stream) {
    return kv_move(c, false, cache, rows, page_table, idx, k, k_pool, k_scale, v, v_pool, v_scale, stream);
}

oc_status oc_attention(oc_ctx* c, const oc_kv_desc* cache, const oc_attention_desc* d, const int32_t* page_table,
                       const int32_t* kv_len, const int32_t* q_start, const int32_t* idx, const void* q, const void* k_pool,
                       const float* k_scale, const void* v_pool, const float* v_scale, void* out, float* lse, void* stream) {
    if (!c || !d || !float_type(d->dtype) || d->q_heads <= 0 || d->n_rows < 0 || d->rows_per_batch <= 0 || d->unit < 0) return OC_ERR_INVALID_ARG;
    if (!(d->scale > 0.0f) || !(d->scale < 0x1p127f)) return OC_ERR_INVALID_ARG;          // (times log2(e) it is finite)
    oc_status st = check_kv(cache, page_table != nullptr);
    if (st != OC_OK) return st;
    if (!kv_quantised(cache) && cache->dtype != d->dtype) return OC_ERR_INVALID_ARG;
    if (d->q_heads % cache->heads != 0) return OC_ERR_INVALID_ARG;
    if (d->n_rows == 0 || cache->n_seqs == 0) return OC_OK;                 // (empty tensors have no addresses)
    if (!q || !out) return OC_ERR_INVALID_ARG;
    if (bad_view(d->q, d->q_heads, d->n_rows, d->rows_per_batch, false, !q_start) ||
        bad_view(d->out, d->q_heads, q_start ? d->n_rows : std::min(d->n_rows, cache->n_seqs * d->rows_per_batch), q_start ? d->n_rows : d->rows_per_batch, true, !q_start))
        return OC_ERR_INVALID_ARG;
    // (a cache of no tokens has no addresses either: its rows become zeros)
    if (cache->seq_rows > 0) {
        st = check_pools(cache, k_pool, k_scale, v_pool, v_scale, true);
        if (st != OC_OK) return st;
    }
    if (out == k_pool || out == v_pool) return OC_ERR_INVALID_ARG;
    if (cache->seq_rows > ROWS_MAX - 4096) return OC_ERR_UNSUPPORTED;       // (the kernels' tiles of keys end before 2^31)
    if (cache->head_dim > 128 || d->n_rows > ROWS_MAX || d->rows_per_batch > ROWS_MAX || d->q_heads > 65535) return OC_ERR_UNSUPPORTED;
    if (d->n_rows * d->q_heads > ROWS_MAX) return OC_ERR_UNSUPPORTED;
    const uintptr_t el = (uintptr_t)elem_size(d->dtype) - 1;
    if (((uintptr_t)q & el) || ((uintptr_t)out & el) || ((uintptr_t)lse & 3u) || ((uintptr_t)page_table & 3u) || ((uintptr_t)kv_len & 3u) ||
        ((uintptr_t)q_start & 3u) || ((uintptr_t)idx & 3u)) return OC_ERR_ALIGNMENT;
    if (same_place({out, lse}, {k_pool, v_pool, k_scale, v_scale, page_table, kv_len, q_start, idx}) || lse == q) return OC_ERR_INVALID_ARG;
    if (out == q && !same_strides(d->q, d->out, d->q_heads, d->n_rows, q_start ? d->n_rows : d->rows_per_batch, !q_start)) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_attention(c, *cache, *d, page_table, kv_len, q_start, idx, q, k_pool, k_scale, v_pool, v_scale, out, lse, (cudaStream_t)stream);
}

// ---- Token Cache on the frame pairs of Frame Cache (Section 3.2.3) ---------------------------------
static oc_status joint_geo(const oc_layout* layout, Geo* g) {
    oc_status st = make_geo(layout, g);
    if (st != OC_OK) return st;
    if (g->kind != OC_KIND_TOKEN || g->self_match) return OC_ERR_INVALID_ARG;
    if (g->gy != 1 || g->gx != 1 || g->dtype != OC_DTYPE_BF16) return OC_ERR_UNSUPPORTED;
    return OC_OK;
}

oc_status oc_joint_workspace_bytes(const oc_layout* layout, size_t* bytes) {
    if (!bytes) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = joint_geo(layout, &g);
    if (st != OC_OK) return st;
    *bytes = joint_workspace_bytes(g);
    return OC_OK;
}

oc_status oc_joint_groups(oc_ctx* c, const oc_layout* layout, const float* frame_best_sim,
                          const int32_t* frame_best_idx, const int32_t* frame_slot_of, int32_t* frames, void* stream) {
    if (!c || !frame_best_sim || !frame_best_idx || !frame_slot_of || !frames) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = joint_geo(layout, &g);
    if (st != OC_OK) return st;
    if (((uintptr_t)frames & 7u) != 0) return OC_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_joint_groups(c, g.B, g.T, frame_best_sim, frame_best_idx, frame_slot_of, (int2*)frames, (cudaStream_t)stream);
}

oc_status oc_match_joint(oc_ctx* c, const oc_layout* layout, const void* x, const int32_t* frames, float* best_sim,
                         int32_t* best_idx, void* stream) {
    if (!c || !x || !frames || !best_sim || !best_idx) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = joint_geo(layout, &g);
    if (st != OC_OK) return st;
    if (misaligned(x) || ((uintptr_t)frames & 7u) != 0) return OC_ERR_ALIGNMENT;
    if (joint_workspace_bytes(g) > c->workspace_bytes) return OC_ERR_WORKSPACE;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_match_joint(c, g, x, (const int2*)frames, best_sim, best_idx, (cudaStream_t)stream);
}

oc_status oc_select_joint(oc_ctx* c, const oc_layout* layout, const int32_t* frames, const float* best_sim,
                          const int32_t* best_idx, int mode, float thr, int64_t n_reuse_pair, int64_t n_reuse_single,
                          int64_t y_stride, int32_t* kept_idx, int32_t* kept_count, int32_t* match_map,
                          int32_t* slot_of, void* stream) {
    if (!c || !frames || !best_sim || !best_idx || !kept_idx || !kept_count || !match_map || !slot_of)
        return OC_ERR_INVALID_ARG;
    if (mode != OC_SELECT_THRESHOLD && mode != OC_SELECT_COUNT) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = joint_geo(layout, &g);
    if (st != OC_OK) return st;
    const int64_t P = (int64_t)g.H * g.W;
    if (n_reuse_pair < 0 || n_reuse_single < 0 || y_stride <= 0 || y_stride > 2 * P) return OC_ERR_INVALID_ARG;
    // capacity: a pair keeps at least 2P - min(n_reuse_pair, 7P/4-ish candidates), a single frame P - ...
    const int64_t cand_single = P - g.reps_per_group, cand_pair = 2 * P - g.reps_per_group;
    const int64_t keep_pair = mode == OC_SELECT_COUNT ? 2 * P - (n_reuse_pair < cand_pair ? n_reuse_pair : cand_pair) : 2 * P;
    const int64_t keep_single = mode == OC_SELECT_COUNT ? P - (n_reuse_single < cand_single ? n_reuse_single : cand_single) : P;
    if (y_stride < keep_pair || y_stride < keep_single) return OC_ERR_INVALID_ARG;
    if ((int64_t)g.B * g.T * y_stride > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
    if (((uintptr_t)frames & 7u) != 0) return OC_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_select_joint(c, g, (const int2*)frames, best_sim, best_idx, mode, thr, n_reuse_pair, n_reuse_single,
                               y_stride, kept_idx, kept_count, match_map, slot_of, (cudaStream_t)stream);
}

oc_status oc_select(oc_ctx* c, const oc_layout* layout, const float* best_sim, const int32_t* best_idx, int mode,
                    float thr, int64_t n_reuse, int64_t y_stride, int32_t* kept_idx, int32_t* kept_count,
                    int32_t* match_map, int32_t* slot_of, void* stream) {
    if (!c || !best_sim || !best_idx || !kept_idx || !kept_count || !match_map || !slot_of) return OC_ERR_INVALID_ARG;
    if (mode != OC_SELECT_THRESHOLD && mode != OC_SELECT_COUNT) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    if (n_reuse < 0 || y_stride <= 0 || y_stride > g.units_per_group) return OC_ERR_INVALID_ARG;
    if (mode == OC_SELECT_THRESHOLD && isnan(thr)) return OC_ERR_INVALID_ARG;
    if (mode == OC_SELECT_COUNT && g.self_match) return OC_ERR_UNSUPPORTED;
    const int64_t n_cand = g.self_match ? g.units_per_group : g.units_per_group - g.reps_per_group;
    const int64_t min_keep = mode == OC_SELECT_COUNT ? g.units_per_group - (n_reuse < n_cand ? n_reuse : n_cand)
                                                     : g.units_per_group;
    if (y_stride < min_keep) return OC_ERR_INVALID_ARG;   // the dense buffer could overflow
    if (g.n_groups * y_stride > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_select(c, g, best_sim, best_idx, mode, thr, n_reuse, y_stride, kept_idx, kept_count, match_map,
                         slot_of, (cudaStream_t)stream);
}

oc_status oc_gather(oc_ctx* c, const oc_rows* rows, const void* x, const int32_t* kept_idx, int64_t n_slots, void* y,
                    void* stream) {
    if (!c || !x || !kept_idx || !y || n_slots < 0) return OC_ERR_INVALID_ARG;
    oc_status st = check_rows(rows);
    if (st != OC_OK) return st;
    if (misaligned(x) || misaligned(y)) return OC_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_gather(c, *rows, x, kept_idx, n_slots, y, (cudaStream_t)stream);
}

oc_status oc_restore(oc_ctx* c, const oc_rows* rows, const void* z, const void* cache, int64_t n_units,
                     const int32_t* slot_of, const int32_t* match_map, void* out, int src_mode, void* stream) {
    if (!c || !z || !slot_of || !out || n_units < 0) return OC_ERR_INVALID_ARG;
    if (src_mode != OC_RESTORE_FROM_CACHE && src_mode != OC_RESTORE_FROM_REPRESENTATIVE) return OC_ERR_INVALID_ARG;
    if (src_mode == OC_RESTORE_FROM_CACHE && !cache) return OC_ERR_INVALID_ARG;
    if (src_mode == OC_RESTORE_FROM_REPRESENTATIVE && !match_map) return OC_ERR_INVALID_ARG;
    if (n_units > 0x7FFFFFFFll) return OC_ERR_UNSUPPORTED;
    oc_status st = check_rows(rows);
    if (st != OC_OK) return st;
    if (misaligned(z) || misaligned(out) || (cache && misaligned(cache))) return OC_ERR_ALIGNMENT;
    if (out == z) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    return launch_restore(c, *rows, z, cache, n_units, slot_of, match_map ? match_map : slot_of, out, src_mode,
                          (cudaStream_t)stream);
}

// ---- Layered Cache -----------------------------------------------------------------------------
oc_status oc_layer_cache_put(oc_ctx* c, int layer, int step, const void* src, size_t bytes, void* stream) {
    if (!c || !src || bytes == 0) return OC_ERR_INVALID_ARG;
    if (misaligned(src)) return OC_ERR_ALIGNMENT;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    LayerEntry& e = c->layers[layer];
    if (e.capacity < bytes) {
        // stream-ordered users of the old buffer must finish before it is released
        if (e.ptr) { cudaStreamSynchronize((cudaStream_t)stream); cudaFree(e.ptr); e.ptr = nullptr; e.capacity = 0; e.bytes = 0; }
        void* p = nullptr;
        if (cudaMalloc(&p, bytes) != cudaSuccess) { cudaGetLastError(); c->layers.erase(layer); return OC_ERR_OOM; }
        e.ptr = p; e.capacity = bytes;
    }
    oc_status st = launch_copy(c, src, e.ptr, bytes, (cudaStream_t)stream);
    if (st != OC_OK) return st;
    e.bytes = bytes; e.step = step;
    return OC_OK;
}

oc_status oc_layer_cache_get(oc_ctx* c, int layer, int step, int interval, void* dst, const void** view,
                             size_t* bytes, void* stream) {
    if (!c) return OC_ERR_INVALID_ARG;
    if (dst && misaligned(dst)) return OC_ERR_ALIGNMENT;
    auto it = c->layers.find(layer);
    if (it == c->layers.end() || it->second.bytes == 0) return OC_CACHE_MISS;
    const LayerEntry& e = it->second;
    if (!oc_layer_cache_would_hit(e.step, step, interval)) return OC_CACHE_MISS;
    if (view) *view = e.ptr;
    if (bytes) *bytes = e.bytes;
    if (dst) {
        DeviceGuard guard(c->device);
        if (!guard.ok) return OC_ERR_CUDA;
        return launch_copy(c, e.ptr, dst, e.bytes, (cudaStream_t)stream);
    }
    return OC_OK;
}

oc_status oc_layer_cache_clear(oc_ctx* c) {
    if (!c) return OC_ERR_INVALID_ARG;
    DeviceGuard guard(c->device);
    cudaDeviceSynchronize();
    for (auto& kv : c->layers) cudaFree(kv.second.ptr);
    c->layers.clear();
    return cuda_ok(cudaGetLastError());
}

// ---- Layered Cache schedule proposal (host only) -------------------------------------------------
oc_status oc_schedule_propose(const double* latency, const double* quality_loss, int64_t n, double target_speedup,
                              int32_t* chosen, int64_t* n_chosen, double* saved) {
    if (!latency || !quality_loss || !chosen || !n_chosen || n < 0 || n > 0x7FFFFFFF) return OC_ERR_INVALID_ARG;
    if (!(target_speedup >= 1.0)) return OC_ERR_INVALID_ARG;
    for (int64_t i = 0; i < n; ++i)
        if (!(latency[i] > 0.0) || !std::isfinite(latency[i]) || !std::isfinite(quality_loss[i])) return OC_ERR_INVALID_ARG;
    // Algorithm 1 as a prefix-sum problem: rank the candidates by quality loss per unit of latency
    // (a stable ranking keeps equal scores in candidate order), accumulate their latencies along the
    // ranking, and the answer is the shortest prefix whose sum reaches the latency budget -- the
    // whole ranking when even that does not.
    std::vector<int32_t> ranking((size_t)n);
    std::vector<double> score((size_t)n);
    for (int64_t i = 0; i < n; ++i) { ranking[(size_t)i] = (int32_t)i; score[(size_t)i] = quality_loss[i] / latency[i]; }
    std::stable_sort(ranking.begin(), ranking.end(), [&score](int32_t a, int32_t b) { return score[(size_t)a] < score[(size_t)b]; });
    std::vector<double> prefix((size_t)n + 1);
    double total = 0.0;                                   // (summed in candidate order, like the budget's definition)
    for (int64_t i = 0; i < n; ++i) total += latency[i];
    prefix[0] = 0.0;
    for (int64_t r = 0; r < n; ++r) prefix[(size_t)r + 1] = prefix[(size_t)r] + latency[ranking[(size_t)r]];
    const double budget = (1.0 - 1.0 / target_speedup) * total;
    // first prefix length whose sum is >= budget (prefix sums of positive terms ascend)
    const int64_t len = std::lower_bound(prefix.begin(), prefix.end(), budget) - prefix.begin();
    const int64_t k = len > n ? n : len;
    for (int64_t r = 0; r < k; ++r) chosen[r] = ranking[(size_t)r];
    *n_chosen = k;
    if (saved) *saved = prefix[(size_t)k];
    return OC_OK;
}

// ---- host-buffer call --------------------------------------------------------------------------
oc_status oc_cache_step_host(oc_ctx* c, const oc_layout* layout, int mode, float thr, int64_t n_reuse,
                             const void* x_host, const void* cache_host, void* out_host, int32_t* kept_count_host,
                             void* stream) {
    if (!c || !x_host || !cache_host || !out_host) return OC_ERR_INVALID_ARG;
    if (mode != OC_SELECT_THRESHOLD && mode != OC_SELECT_COUNT) return OC_ERR_INVALID_ARG;
    Geo g;
    oc_status st = make_geo(layout, &g);
    if (st != OC_OK) return st;
    if (match_workspace_bytes(g) > c->workspace_bytes) return OC_ERR_WORKSPACE;
    oc_rows rows;
    st = oc_rows_from_layout(layout, g.C, g.elem_bytes, &rows);
    if (st != OC_OK) return st;
    DeviceGuard guard(c->device);
    if (!guard.ok) return OC_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;

    const size_t tensor_bytes = (size_t)g.B * g.T * g.H * g.W * g.C * g.elem_bytes;
    const size_t nu = (size_t)g.n_units, ng = (size_t)g.n_groups;
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    // staging: x | cache | out | y | best_sim | best_idx | kept_idx | match_map | slot_of | kept_count
    const size_t need = 4 * up(tensor_bytes) + 5 * up(nu * 4) + up(ng * 4);
    if (c->stage_bytes < need) {
        cudaStreamSynchronize(s);
        cudaFree(c->stage); c->stage = nullptr; c->stage_bytes = 0;
        if (cudaMalloc(&c->stage, need) != cudaSuccess) { cudaGetLastError(); return OC_ERR_OOM; }
        c->stage_bytes = need;
    }
    uint8_t* p = (uint8_t*)c->stage;
    void* dx = p; p += up(tensor_bytes);
    void* dcache = p; p += up(tensor_bytes);
    void* dout = p; p += up(tensor_bytes);
    void* dy = p; p += up(tensor_bytes);
    float* dsim = (float*)p; p += up(nu * 4);
    int32_t* didx = (int32_t*)p; p += up(nu * 4);
    int32_t* dkept = (int32_t*)p; p += up(nu * 4);
    int32_t* dmap = (int32_t*)p; p += up(nu * 4);
    int32_t* dslot = (int32_t*)p; p += up(nu * 4);
    int32_t* dcount = (int32_t*)p;

    // Pinned (page-locked, device-mapped) host buffers are read and written by the restore kernel
    // itself: of the cache only the rows of reused units then cross the bus, and the output streams
    // to the host while those rows stream in (the link is full duplex).  Pageable buffers go through
    // staging copies.
    auto mapped = [](const void* h) -> void* {
        cudaPointerAttributes a;
        if (cudaPointerGetAttributes(&a, h) != cudaSuccess) { cudaGetLastError(); return nullptr; }
        return (a.type == cudaMemoryTypeHost && ((uintptr_t)a.devicePointer & 15) == 0) ? a.devicePointer : nullptr;
    };
    void* cache_dev = mapped(cache_host);
    void* out_dev = mapped(out_host);

    // Token Cache groups never span frames, so the call is cut into up to 8 chunks of whole frames:
    // all host->device copies of x are queued at once on a second stream, and chunk k is matched,
    // selected, gathered and restored (its output streaming back to the host) while the copies of the
    // chunks after it are still arriving.  Other kinds, and single frames, are one chunk.
    const int64_t frames = (int64_t)g.B * g.T;
    int n_chunks = (g.kind == OC_KIND_TOKEN && frames > 1) ? (int)(frames < 8 ? frames : 8) : 1;
    if (n_chunks > 1) {
        if (!c->copy_stream && cudaStreamCreateWithFlags(&c->copy_stream, cudaStreamNonBlocking) != cudaSuccess) {
            cudaGetLastError(); n_chunks = 1;
        }
        while (n_chunks > 1 && (int)c->chunk_events.size() < n_chunks + 1) {
            cudaEvent_t e;
            if (cudaEventCreateWithFlags(&e, cudaEventDisableTiming) != cudaSuccess) { cudaGetLastError(); n_chunks = 1; break; }
            c->chunk_events.push_back(e);
        }
    }
    if (n_chunks == 1) {
        if (cudaMemcpyAsync(dx, x_host, tensor_bytes, cudaMemcpyHostToDevice, s) != cudaSuccess) return OC_ERR_CUDA;
        if (!cache_dev && cudaMemcpyAsync(dcache, cache_host, tensor_bytes, cudaMemcpyHostToDevice, s) != cudaSuccess)
            return OC_ERR_CUDA;
        st = oc_match(c, layout, dx, dsim, didx, nullptr, nullptr, stream);
        if (st != OC_OK) return st;
        st = oc_select(c, layout, dsim, didx, mode, thr, n_reuse, g.units_per_group, dkept, dcount, dmap, dslot, stream);
        if (st != OC_OK) return st;
        st = oc_gather(c, &rows, dx, dkept, (int64_t)nu, dy, stream);
        if (st != OC_OK) return st;
        st = oc_restore(c, &rows, dy, cache_dev ? cache_dev : dcache, (int64_t)nu, dslot, dmap, out_dev ? out_dev : dout,
                        OC_RESTORE_FROM_CACHE, stream);
        if (st != OC_OK) return st;
        if (!out_dev && cudaMemcpyAsync(out_host, dout, tensor_bytes, cudaMemcpyDeviceToHost, s) != cudaSuccess)
            return OC_ERR_CUDA;
    } else {
        const int64_t fpc = (frames + n_chunks - 1) / n_chunks;              // frames per chunk
        const size_t frame_bytes = tensor_bytes / (size_t)frames;
        const size_t units_pf = nu / (size_t)frames, groups_pf = ng / (size_t)frames;
        cudaStream_t cs = c->copy_stream;
        // the copies may not overtake earlier work of the caller's stream on the staging buffers
        if (cudaEventRecord(c->chunk_events[n_chunks], s) != cudaSuccess ||
            cudaStreamWaitEvent(cs, c->chunk_events[n_chunks], 0) != cudaSuccess) return OC_ERR_CUDA;
        for (int k = 0; k < n_chunks; ++k) {
            const int64_t f0 = k * fpc, f1 = (f0 + fpc < frames) ? f0 + fpc : frames;
            if (f0 >= f1) { n_chunks = k; break; }
            const size_t off = (size_t)f0 * frame_bytes, len = (size_t)(f1 - f0) * frame_bytes;
            if (cudaMemcpyAsync((uint8_t*)dx + off, (const uint8_t*)x_host + off, len, cudaMemcpyHostToDevice, cs) != cudaSuccess)
                return OC_ERR_CUDA;
            if (!cache_dev && cudaMemcpyAsync((uint8_t*)dcache + off, (const uint8_t*)cache_host + off, len,
                                              cudaMemcpyHostToDevice, cs) != cudaSuccess) return OC_ERR_CUDA;
            if (cudaEventRecord(c->chunk_events[k], cs) != cudaSuccess) return OC_ERR_CUDA;
        }
        for (int k = 0; k < n_chunks; ++k) {
            const int64_t f0 = k * fpc, f1 = (f0 + fpc < frames) ? f0 + fpc : frames;
            oc_layout sub = *layout;
            sub.B = (int)(f1 - f0); sub.T = 1;
            oc_rows sub_rows;
            st = oc_rows_from_layout(&sub, g.C, g.elem_bytes, &sub_rows);
            if (st != OC_OK) return st;
            const size_t off = (size_t)f0 * frame_bytes, uoff = (size_t)f0 * units_pf, goff = (size_t)f0 * groups_pf;
            const int64_t sub_units = (int64_t)((size_t)(f1 - f0) * units_pf);
            if (cudaStreamWaitEvent(s, c->chunk_events[k], 0) != cudaSuccess) return OC_ERR_CUDA;
            st = oc_match(c, &sub, (uint8_t*)dx + off, dsim + uoff, didx + uoff, nullptr, nullptr, stream);
            if (st != OC_OK) return st;
            st = oc_select(c, &sub, dsim + uoff, didx + uoff, mode, thr, n_reuse, g.units_per_group, dkept + uoff,
                           dcount + goff, dmap + uoff, dslot + uoff, stream);
            if (st != OC_OK) return st;
            st = oc_gather(c, &sub_rows, (uint8_t*)dx + off, dkept + uoff, sub_units, (uint8_t*)dy + off, stream);
            if (st != OC_OK) return st;
            st = oc_restore(c, &sub_rows, (uint8_t*)dy + off, (uint8_t*)(cache_dev ? cache_dev : dcache) + off, sub_units,
                            dslot + uoff, dmap + uoff, (uint8_t*)(out_dev ? out_dev : dout) + off, OC_RESTORE_FROM_CACHE, stream);
            if (st != OC_OK) return st;
            if (!out_dev && cudaMemcpyAsync((uint8_t*)out_host + off, (uint8_t*)dout + off, (size_t)(f1 - f0) * frame_bytes,
                                            cudaMemcpyDeviceToHost, s) != cudaSuccess) return OC_ERR_CUDA;
        }
    }
    if (kept_count_host &&
        cudaMemcpyAsync(kept_count_host, dcount, ng * 4, cudaMemcpyDeviceToHost, s) != cudaSuccess) return OC_ERR_CUDA;
    if (cudaStreamSynchronize(s) != cudaSuccess) return OC_ERR_CUDA;
    return OC_OK;
}

}  // extern "C"
