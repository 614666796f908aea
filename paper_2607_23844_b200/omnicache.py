"""ctypes binding of the OmniCache C-ABI (``include/omnicache.h``); same names, marshalling only.

Every function here turns torch tensors into raw device pointers and the current torch stream into a
``cudaStream_t`` and calls the shared library: all arithmetic and data movement happen in the CUDA
kernels.  There is no CPU fallback: a missing library raises at import, a failing call raises
``OmniCacheError``.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libomnicache_b200.so")

OK, ERR_INVALID_ARG, ERR_ALIGNMENT, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_OOM, CACHE_MISS = range(9)
KIND_TOKEN, KIND_FRAME, KIND_BLOCK = 0, 1, 2
DTYPE_F32, DTYPE_BF16, DTYPE_I8 = 0, 1, 2
SELECT_THRESHOLD, SELECT_COUNT = 0, 1
RESTORE_FROM_CACHE, RESTORE_FROM_REPRESENTATIVE = 0, 1
FRAME_MEAN_POS_COS, FRAME_FLAT_COS = 0, 1
(K_NORMS, K_MATCH_TC, K_MATCH_SIMT, K_MATCH_FIN, K_FRAME, K_FRAME_FIN, K_BLOCK, K_BLOCK_FIN, K_SELECT,
 K_GATHER, K_RESTORE, K_COPY, K_LINEAR, K_BLOCK_NORM, K_ROPE, K_QUANT, K_LINEAR_I8) = range(17)
K_COUNT = 17
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
ROPE_ADJACENT, ROPE_HALVES = 0, 1

EXPORTS = (
    "oc_status_str", "oc_layout_check", "oc_layout_counts", "oc_match_workspace_bytes",
    "oc_rows_from_layout", "oc_layer_cache_would_hit", "oc_kernel_name", "oc_create", "oc_destroy",
    "oc_device_status", "oc_profile_enable", "oc_profile_reset", "oc_profile_read", "oc_profile_span_read",
    "oc_profile_captured_read", "oc_match", "oc_match_frame_levels",
    "oc_select", "oc_gather", "oc_restore", "oc_layer_cache_put", "oc_layer_cache_get",
    "oc_layer_cache_clear", "oc_cache_step_host", "oc_match_frame_noalloc", "oc_selftest_bounded_wait", "oc_selftest_per_device_once",
    "oc_schedule_propose", "oc_joint_workspace_bytes", "oc_joint_groups", "oc_match_joint", "oc_select_joint",
    "oc_linear_gather_scatter", "oc_tc_plan_override", "oc_tc_plan_describe",
    "oc_block_norm", "oc_rope_table_size", "oc_rope_table", "oc_rope", "oc_quantize_rows", "oc_linear_int8",
)


class OmniCacheError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)}")


class CLayout(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("kind", "dtype", "B", "T", "H", "W", "C", "sy", "sx", "oy", "ox",
                                      "gy", "gx", "self_match", "frame_stat")] + [("eps", C.c_float)]


class CRows(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("seg_bytes", "n_seg", "seg_stride", "unit_pitch",
                                        "units_per_outer", "outer_pitch")]


class CBlockNorm(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("dtype", "h_dtype", "param_dtype", "post_norm", "pre_norm")] +
                [(n, C.c_float) for n in ("post_eps", "pre_eps", "res_scale")] +
                [(n, C.c_int64) for n in ("n_rows", "C", "rows_per_group", "mod_stride", "unit_rows", "dense_rows")])


class CRopeView(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("batch_stride", "row_stride", "head_stride")]


class CRope(C.Structure):
    _fields_ = ([(n, C.c_int) for n in ("dtype", "head_dim", "q_heads", "k_heads", "pairing", "inverse")] +
                [("axis_dims", C.c_int * 3), ("axis_len", C.c_int * 3), ("eps", C.c_float)] +
                [(n, C.c_int64) for n in ("n_rows", "rows_per_batch", "unit_rows")] +
                [(n, CRopeView) for n in ("q", "q_out", "k", "k_out")])


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_23844_b200.build`")
_lib = C.CDLL(LIB_PATH)

_vp, _i, _i64, _f = C.c_void_p, C.c_int, C.c_int64, C.c_float
_Tensor = torch.Tensor
_lib.oc_status_str.restype = C.c_char_p
_lib.oc_status_str.argtypes = [_i]
_lib.oc_kernel_name.restype = C.c_char_p
_lib.oc_kernel_name.argtypes = [_i]
_lib.oc_layout_check.argtypes = [_vp]
_lib.oc_layout_counts.argtypes = [_vp, _vp, _vp, _vp]
_lib.oc_match_workspace_bytes.argtypes = [_vp, _vp]
_lib.oc_rows_from_layout.argtypes = [_vp, _i, _i, _vp]
_lib.oc_layer_cache_would_hit.argtypes = [_i, _i, _i]
_lib.oc_create.argtypes = [_vp, _i, C.c_size_t]
_lib.oc_destroy.argtypes = [_vp]
_lib.oc_device_status.argtypes = [_vp, _vp]
_lib.oc_selftest_bounded_wait.argtypes = [_vp, C.c_uint, _vp]
_lib.oc_selftest_per_device_once.argtypes = [C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int), C.POINTER(C.c_int)]
_lib.oc_profile_enable.argtypes = [_vp, _i]
_lib.oc_tc_plan_override.argtypes = [_vp, _i, _i, _i, _i, _i, _i]
_lib.oc_tc_plan_describe.argtypes = [_vp, _vp, _vp]
_lib.oc_profile_reset.argtypes = [_vp]
_lib.oc_profile_read.argtypes = [_vp, _i, _vp, _vp]
_lib.oc_profile_span_read.argtypes = [_vp, _i, _vp, _vp]
_lib.oc_profile_captured_read.argtypes = [_vp, _i, _vp, _vp]
_lib.oc_match.argtypes = [_vp] * 8
_lib.oc_match_frame_levels.argtypes = [_vp, _vp, _vp, _i, _vp, _vp, _vp, _vp, _vp, _vp]
_lib.oc_select.argtypes = [_vp, _vp, _vp, _vp, _i, _f, _i64, _i64, _vp, _vp, _vp, _vp, _vp]
_lib.oc_linear_gather_scatter.argtypes = [_vp, _vp, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _vp]
_lib.oc_joint_workspace_bytes.argtypes = [_vp, _vp]
_lib.oc_joint_groups.argtypes = [_vp] * 7
_lib.oc_match_joint.argtypes = [_vp] * 7
_lib.oc_select_joint.argtypes = [_vp, _vp, _vp, _vp, _vp, _i, _f, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp]
_lib.oc_gather.argtypes = [_vp, _vp, _vp, _vp, _i64, _vp, _vp]
_lib.oc_restore.argtypes = [_vp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _i, _vp]
_lib.oc_layer_cache_put.argtypes = [_vp, _i, _i, _vp, C.c_size_t, _vp]
_lib.oc_layer_cache_get.argtypes = [_vp, _i, _i, _i, _vp, _vp, _vp, _vp]
_lib.oc_layer_cache_clear.argtypes = [_vp]
_lib.oc_cache_step_host.argtypes = [_vp, _vp, _i, _f, _i64, _vp, _vp, _vp, _vp, _vp]
_lib.oc_schedule_propose.argtypes = [_vp, _vp, _i64, C.c_double, _vp, _vp, _vp]
_lib.oc_block_norm.argtypes = [_vp, C.POINTER(CBlockNorm)] + [_vp] * 16
_lib.oc_rope_table_size.argtypes = [_vp, _vp]
_lib.oc_rope_table.argtypes = [_vp, C.c_double, _vp]
_lib.oc_rope.argtypes = [_vp, C.POINTER(CRope)] + [_vp] * 10
_lib.oc_quantize_rows.argtypes = [_vp, _vp, _i, _i64, _i64, _vp, _i64, _i64, _vp, _vp, _vp]
_lib.oc_linear_int8.argtypes = [_vp, _vp, _vp, _i64, _i64, _vp, _vp, _i64, _vp, _vp, _i, _i64, _i64, _vp, _vp]
_lib.oc_match_frame_noalloc.argtypes = [_i, _vp, _vp, _vp, _vp, _vp, _vp]
NOALLOC_SCRATCH_BYTES = 1 << 20


def status_str(s: int) -> str:
    return _lib.oc_status_str(s).decode()


def kernel_name(k: int) -> str:
    return _lib.oc_kernel_name(k).decode()


def _chk(st: int, where: str) -> None:
    if st != OK:
        raise OmniCacheError(st, where)


_LAYOUT_CACHE: dict = {}


@dataclass
class Layout:
    kind: int
    dtype: int
    B: int
    T: int
    H: int
    W: int
    C: int
    sy: int = 2
    sx: int = 2
    oy: int = 0
    ox: int = 0
    gy: int = 1
    gx: int = 1
    self_match: int = 0
    frame_stat: int = 0
    eps: float = 1e-8

    def c(self) -> CLayout:
        key = (self.kind, self.dtype, self.B, self.T, self.H, self.W, self.C, self.sy, self.sx,
               self.oy, self.ox, self.gy, self.gx, self.self_match, self.frame_stat, self.eps)
        hit = _LAYOUT_CACHE.get(key)
        if hit is None:
            hit = _LAYOUT_CACHE[key] = CLayout(*key)
        return hit

    def check(self) -> int:
        return layout_check(self)

    def counts(self) -> tuple[int, int, int]:
        return layout_counts(self)

    @property
    def n_groups(self) -> int:
        return self.counts()[0]

    @property
    def units_per_group(self) -> int:
        return self.counts()[1]

    @property
    def reps_per_group(self) -> int:
        return self.counts()[2]

    @property
    def n_units(self) -> int:
        g, u, _ = self.counts()
        return g * u

    @property
    def elem_bytes(self) -> int:
        return 4 if self.dtype == DTYPE_F32 else 2


def layout_check(layout: Layout) -> int:
    """oc_layout_check: returns the status code (no exception), host only."""
    cl = layout.c()
    return _lib.oc_layout_check(C.byref(cl))


def layout_counts(layout: Layout) -> tuple[int, int, int]:
    cl = layout.c()
    g, u, r = C.c_int64(), C.c_int64(), C.c_int64()
    _chk(_lib.oc_layout_counts(C.byref(cl), C.byref(g), C.byref(u), C.byref(r)), "oc_layout_counts")
    return g.value, u.value, r.value


def match_workspace_bytes(layout: Layout) -> int:
    cl = layout.c()
    n = C.c_size_t()
    _chk(_lib.oc_match_workspace_bytes(C.byref(cl), C.byref(n)), "oc_match_workspace_bytes")
    return n.value


def joint_workspace_bytes(layout: Layout) -> int:
    cl = layout.c()
    n = C.c_size_t()
    _chk(_lib.oc_joint_workspace_bytes(C.byref(cl), C.byref(n)), "oc_joint_workspace_bytes")
    return n.value


def rows_from_layout(layout: Layout, channels: int, elem_bytes: int) -> CRows:
    cl, rows = layout.c(), CRows()
    _chk(_lib.oc_rows_from_layout(C.byref(cl), channels, elem_bytes, C.byref(rows)), "oc_rows_from_layout")
    return rows


def layer_cache_would_hit(stored_step: int, step: int, interval: int) -> bool:
    return bool(_lib.oc_layer_cache_would_hit(stored_step, step, interval))


def _ptr(t) -> int | None:
    if t is None:
        return None
    if type(t) is not _Tensor and isinstance(t, int):              # (the class first: isinstance takes longer to say no)
        return t
    assert t.is_contiguous(), "tensors handed to the C-ABI must be contiguous"
    return t.data_ptr()


# The current stream's handle.  torch.cuda.current_stream() builds a Stream object first (3 us on the host, as much
# as a whole launch); the handle alone takes 0.1 us.
try:
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _current_device
except ImportError:
    def _raw_stream(device: int) -> int:
        return torch.cuda.current_stream(device).cuda_stream
    _current_device = torch.cuda.current_device


def _stream(stream) -> int:
    if stream is None:
        return _raw_stream(_current_device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def _ptr_strided(t) -> int | None:
    """Pointer of a tensor whose strides the call gets on their own (a part of a larger tensor)."""
    if t is None or (type(t) is not _Tensor and isinstance(t, int)):
        return t
    return t.data_ptr()


def _rows(t, width: int, stride: int | None, name: str):
    """(pointer, elements between rows) of a matrix `width` elements wide: dense unless a stride is given or the tensor
    is a part of a larger one."""
    if t is None or (type(t) is not _Tensor and isinstance(t, int)):
        return t, width if stride is None else stride
    if t.is_contiguous():
        return t.data_ptr(), width if stride is None else stride
    if t.stride(-1) != 1:
        raise ValueError(f"the elements of a row of {name} must be contiguous")
    if stride is None:
        if t.dim() != 2 or t.shape[1] != width:
            raise ValueError(f"{name} is neither contiguous nor [rows, {width}]: its row stride must be given")
        stride = t.stride(0)
    return t.data_ptr(), stride


def _group_vectors(t, strides: tuple, desc: CBlockNorm, name: str) -> int | None:
    """Pointer of gate, scale or shift: a vector for each group, strides = (mod_stride, 1) elements apart, or one vector
    for all of them (mod_stride 0)."""
    if type(t) is _Tensor and t.stride() == strides:
        return t.data_ptr()
    if t is None or isinstance(t, int):
        return t
    apart, groups = strides[0], -(-desc.n_rows // max(desc.rows_per_group, 1))
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"the elements of a vector of {name} must be contiguous")
    vectors, last = 1, None
    for n, s in zip(t.shape[:-1], t.stride()[:-1]):
        if n == 1:
            continue
        if last is not None and last != n * s:                    # not evenly spaced from here on
            break
        vectors, last = vectors * n, s
        if s == apart and vectors >= groups:
            return t.data_ptr()
    if groups <= 1 or (last is None and apart == 0):
        return t.data_ptr()
    if last is None:                                              # one run of elements, which says nothing of the others
        end = t.storage_offset() + (groups - 1) * apart + desc.C
        if end <= t.untyped_storage().nbytes() // t.element_size():
            return t.data_ptr()
    raise ValueError(f"{name} does not hold {groups} vectors {apart} elements apart: mod_stride must be its row stride")


def block_norm_desc(n_rows: int, C_: int, dtype: int, h_dtype: int, param_dtype: int, post_norm: int = NORM_NONE,
                    pre_norm: int = NORM_NONE, post_eps: float = 1e-6, pre_eps: float = 1e-6, res_scale: float = 1.0,
                    rows_per_group: int | None = None, mod_stride: int = 0, unit_rows: int = 1,
                    dense_rows: int | None = None) -> CBlockNorm:
    """oc_block_norm_desc: made once for a layer and passed to Context.block_norm.  rows_per_group and dense_rows
    default to n_rows (one group; every row computed)."""
    return CBlockNorm(dtype, h_dtype, param_dtype, post_norm, pre_norm, post_eps, pre_eps, res_scale, n_rows, C_,
                      max(n_rows, 1) if rows_per_group is None else rows_per_group, mod_stride, unit_rows,
                      n_rows if dense_rows is None else dense_rows)


def rope_desc(n_rows: int, dtype: int, head_dim: int, axis_dims, axis_len, q_heads: int, k_heads: int = 0,
              rows_per_batch: int | None = None, unit_rows: int = 1, pairing: int = ROPE_ADJACENT, inverse: bool = False,
              eps: float = 1e-6, q=None, q_out=None, k=None, k_out=None) -> CRope:
    """oc_rope_desc, the strides taken from tensors (or from (batch, row, head) stride tuples): q, k are
    [n_rows, heads, head_dim] views, q_out, k_out [batch, heads, rows, head_dim] or [n_rows, heads, head_dim].  q and k
    may be [batch, heads, rows, head_dim] too where one stride leads from each row to the next through all the batch."""
    per_batch = rows_per_batch or max(n_rows, 1)

    def view(t, heads, rows_in_order):
        if t is None:                                                # strides that are needed are left invalid
            return CRopeView(0, -1 if n_rows > 1 else 0, -1 if heads > 1 else 0)
        if isinstance(t, tuple):
            return CRopeView(*t)
        if t.shape[-1] != head_dim or t.stride(-1) != 1:
            raise ValueError("heads must be contiguous and head_dim wide")
        if t.dim() == 4:
            if t.shape[1] != heads:
                raise ValueError("a [batch, heads, rows, head_dim] tensor has another number of heads")
            if rows_in_order and t.shape[0] > 1 and t.stride(0) != t.shape[2] * t.stride(2):
                raise ValueError("rows of q and k must follow one another at one stride: pass [rows, heads, head_dim]")
            if (t.shape[0] * t.shape[2] < n_rows if rows_in_order
                    else t.shape[2] < min(per_batch, n_rows) or t.shape[0] * per_batch < n_rows):
                raise ValueError("fewer rows than n_rows, or in a batch element of q_out or k_out than rows_per_batch")
            return CRopeView(t.stride(0), t.stride(2), t.stride(1))
        if t.dim() != 3 or t.shape[1] != heads:
            raise ValueError("expected [rows, heads, head_dim] or [batch, heads, rows, head_dim]")
        if t.shape[0] < n_rows:
            raise ValueError("fewer rows than n_rows")
        return CRopeView(t.stride(0) * per_batch, t.stride(0), t.stride(1))
    return CRope(dtype, head_dim, q_heads, k_heads, pairing, int(inverse), (C.c_int * 3)(*axis_dims), (C.c_int * 3)(*axis_len),
                 eps, n_rows, max(n_rows, 1) if rows_per_batch is None else rows_per_batch, unit_rows,
                 view(q, q_heads, True), view(q_out, q_heads, False), view(k, k_heads, True), view(k_out, k_heads, False))


def rope_table(desc: CRope, theta: float = 10000.0) -> torch.Tensor:
    """oc_rope_table: the (cos, sin) table of a rotation, as a CPU tensor.  Host only."""
    n = C.c_int64()
    _chk(_lib.oc_rope_table_size(C.byref(desc), C.byref(n)), "oc_rope_table_size")
    t = torch.empty(n.value, dtype=torch.float32)
    _chk(_lib.oc_rope_table(C.byref(desc), theta, t.data_ptr()), "oc_rope_table")
    return t


def schedule_propose(latency, quality_loss, target_speedup: float):
    """Layered Cache schedule proposal (Algorithm 1).  Returns (chosen candidate indices in the order
    taken, saved latency).  Host-side: no device work."""
    import numpy as np
    L = np.ascontiguousarray(latency, dtype=np.float64)
    Q = np.ascontiguousarray(quality_loss, dtype=np.float64)
    if L.shape != Q.shape or L.ndim != 1:
        raise ValueError("latency and quality_loss must be 1-D arrays of one length")
    chosen = np.empty(max(L.size, 1), dtype=np.int32)
    n, saved = C.c_int64(), C.c_double()
    _chk(_lib.oc_schedule_propose(L.ctypes.data_as(_vp), Q.ctypes.data_as(_vp), L.size, float(target_speedup),
                                  chosen.ctypes.data_as(_vp), C.byref(n), C.byref(saved)), "oc_schedule_propose")
    return chosen[:n.value].tolist(), saved.value


def match_frame_noalloc(device: int, layout: Layout, x, best_sim, best_idx, pair_sim=None, stream=None,
                        check: bool = True) -> int:
    """oc_match_frame_noalloc: the Frame Cache match for callers that may not allocate device memory.

    No context is involved: the partial sums go to a fixed array inside the library (at most
    NOALLOC_SCRATCH_BYTES; larger layouts come back as ERR_WORKSPACE).  Calls on one device share that
    array, so do not let two of them overlap on the GPU, and make the first call on a device outside
    of any stream capture."""
    cl = layout.c()
    st = _lib.oc_match_frame_noalloc(device, C.byref(cl), _ptr(x), _ptr(best_sim), _ptr(best_idx), _ptr(pair_sim),
                                     _stream(stream))
    if check:
        _chk(st, "oc_match_frame_noalloc")
    return st


class Context:
    """oc_create / oc_destroy and the per-context calls."""

    def __init__(self, device: int = 0, workspace_bytes: int = 0):
        self._h = C.c_void_p()
        _chk(_lib.oc_create(C.byref(self._h), device, workspace_bytes), "oc_create")
        self.device = device
        self.workspace_bytes = workspace_bytes

    def close(self) -> None:
        if self._h:
            _lib.oc_destroy(self._h)
            self._h = C.c_void_p()

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- status / profile ------------------------------------------------------------------------
    def device_status(self) -> int:
        code = C.c_int()
        _chk(_lib.oc_device_status(self._h, C.byref(code)), "oc_device_status")
        return code.value

    def selftest_bounded_wait(self, limit_us: int = 2000, stream=None) -> None:
        """Makes a bounded device-side wait run out on purpose (see oc_selftest_bounded_wait)."""
        _chk(_lib.oc_selftest_bounded_wait(self._h, limit_us, _stream(stream)), "oc_selftest_bounded_wait")

    def tc_plan_override(self, plan=None, single_accumulator: bool = False, candidates_resident: int = -1) -> None:
        """Test hook (oc_tc_plan_override): ``plan`` = (pair, tiles per CTA, pieces per row[, candidates
        resident]) forces the tensor-core matcher's work split; None returns to the planner."""
        if plan is None:
            _chk(_lib.oc_tc_plan_override(self._h, 0, 0, 1, 1, 0, -1), "oc_tc_plan_override")
        else:
            vals = [int(v) for v in plan]
            if len(vals) == 4:
                candidates_resident = vals[3]
            pair, tiles, pieces = vals[:3]
            _chk(_lib.oc_tc_plan_override(self._h, 1, pair, tiles, pieces, int(single_accumulator), int(candidates_resident)),
                 "oc_tc_plan_override")

    def tc_plan_describe(self, layout: Layout) -> dict:
        """Test hook (oc_tc_plan_describe): the tensor-core matcher's work split for this layout."""
        cl = layout.c()
        out = (C.c_int32 * 12)()
        _chk(_lib.oc_tc_plan_describe(self._h, C.byref(cl), out), "oc_tc_plan_describe")
        keys = ("pair", "tiles", "pieces_per_row", "two_acc_sets", "stages", "stage_bytes", "a_resident", "pieces",
                "walkers", "widest_cols", "kblocks")
        return dict(zip(keys, list(out)))

    def profile_enable(self, on) -> None:
        """False/0: timers off; True/1: CUDA events around every launch; 2: device-side spans of the
        tensor-core matcher (read with profile_span_read)."""
        _chk(_lib.oc_profile_enable(self._h, int(on)), "oc_profile_enable")

    def profile_reset(self) -> None:
        _chk(_lib.oc_profile_reset(self._h), "oc_profile_reset")

    def profile_read(self, kernel_id: int) -> tuple[int, float]:
        n, ms = C.c_int64(), C.c_double()
        _chk(_lib.oc_profile_read(self._h, kernel_id, C.byref(n), C.byref(ms)), "oc_profile_read")
        return n.value, ms.value

    def profile_captured_read(self, kernel_id: int) -> tuple[int, float]:
        """(brackets captured into CUDA graphs, sum of their most recent recordings in ms)."""
        n, ms = C.c_int64(), C.c_double()
        _chk(_lib.oc_profile_captured_read(self._h, kernel_id, C.byref(n), C.byref(ms)), "oc_profile_captured_read")
        return n.value, ms.value

    def profile_span_read(self, kernel_id: int) -> tuple[int, float]:
        """(launches stamped, summed first-CTA-entry -> last-CTA-exit time in ms); see profile_enable(2)."""
        n, ms = C.c_int64(), C.c_double()
        _chk(_lib.oc_profile_span_read(self._h, kernel_id, C.byref(n), C.byref(ms)), "oc_profile_span_read")
        return n.value, ms.value

    def launches(self) -> dict[str, int]:
        return {kernel_name(k): self.profile_read(k)[0] for k in range(K_COUNT)}

    # -- hot path --------------------------------------------------------------------------------
    def match(self, layout: Layout, x, best_sim, best_idx, aux_sim=None, pair_sim=None, stream=None,
              check: bool = True) -> int:
        cl = layout.c()
        st = _lib.oc_match(self._h, C.byref(cl), _ptr(x), _ptr(best_sim), _ptr(best_idx), _ptr(aux_sim),
                           _ptr(pair_sim), _stream(stream))
        if check:
            _chk(st, "oc_match")
        return st

    def linear_gather_scatter(self, a, a_rows: int, K: int, a_idx, n_rows: int, w, N: int, out, out_rows: int,
                              out_idx, stream=None, check: bool = True) -> int:
        st = _lib.oc_linear_gather_scatter(self._h, _ptr(a), a_rows, K, _ptr(a_idx), n_rows, _ptr(w), N, _ptr(out),
                                           out_rows, _ptr(out_idx), _stream(stream))
        if check:
            _chk(st, "oc_linear_gather_scatter")
        return st

    # -- the wrapped block on kept tokens ----------------------------------------------------------
    def block_norm(self, desc: CBlockNorm, x, z=None, slot_of=None, cache=None, cache_out=None, out=None, post_w=None,
                   post_b=None, gate=None, pre_w=None, pre_b=None, scale=None, shift=None, h=None, h_scale=None,
                   stream=None, check: bool = True) -> int:
        """oc_block_norm.  gate, scale and shift may be column ranges of one [groups, mod_stride] tensor."""
        apart = (desc.mod_stride, 1)
        if gate is not None:
            gate = _group_vectors(gate, apart, desc, "gate")
        if scale is not None:
            scale = _group_vectors(scale, apart, desc, "scale")
        if shift is not None:
            shift = _group_vectors(shift, apart, desc, "shift")
        st = _lib.oc_block_norm(self._h, desc, _ptr(x), _ptr(z), _ptr(slot_of), _ptr(cache), _ptr(cache_out),
                                _ptr(out), _ptr(post_w), _ptr(post_b), gate, _ptr(pre_w), _ptr(pre_b), scale, shift, _ptr(h),
                                _ptr(h_scale), _stream(stream))
        if check:
            _chk(st, "oc_block_norm")
        return st

    def rope(self, desc: CRope, table, q, q_out, k=None, k_out=None, idx=None, pos=None, q_w=None, k_w=None, stream=None,
             check: bool = True) -> int:
        """oc_rope: strides are the descriptor's, so q and k may be parts of one projection."""
        st = _lib.oc_rope(self._h, desc, _ptr(table), _ptr(idx), _ptr(pos), _ptr_strided(q), _ptr_strided(q_out),
                          _ptr(q_w), _ptr_strided(k), _ptr_strided(k_out), _ptr(k_w), _stream(stream))
        if check:
            _chk(st, "oc_rope")
        return st

    def quantize_rows(self, x, dtype: int, n_rows: int, K: int, q, scale, idx=None, x_rows: int | None = None,
                      x_stride: int | None = None, stream=None, check: bool = True) -> int:
        """oc_quantize_rows: x may be a column range of a packed projection (its stride is then the default)."""
        x, x_stride = _rows(x, K, x_stride, "x")
        st = _lib.oc_quantize_rows(self._h, x, dtype, n_rows if x_rows is None else x_rows, x_stride, _ptr(idx), n_rows, K,
                                   _ptr(q), _ptr(scale), _stream(stream))
        if check:
            _chk(st, "oc_quantize_rows")
        return st

    def linear_int8(self, a, a_scale, M: int, K: int, w, w_scale, N: int, out, out_dtype: int, bias=None,
                    out_rows: int | None = None, out_stride: int | None = None, out_idx=None, stream=None,
                    check: bool = True) -> int:
        """oc_linear_int8: out may be a column range of a packed tensor (its stride is then the default)."""
        out, out_stride = _rows(out, N, out_stride, "out")
        st = _lib.oc_linear_int8(self._h, _ptr(a), _ptr(a_scale), M, K, _ptr(w), _ptr(w_scale), N, _ptr(bias), out, out_dtype,
                                 M if out_rows is None else out_rows, out_stride, _ptr(out_idx), _stream(stream))
        if check:
            _chk(st, "oc_linear_int8")
        return st

    def joint_groups(self, layout: Layout, frame_best_sim, frame_best_idx, frame_slot_of, frames, stream=None,
                     check: bool = True) -> int:
        cl = layout.c()
        st = _lib.oc_joint_groups(self._h, C.byref(cl), _ptr(frame_best_sim), _ptr(frame_best_idx),
                                  _ptr(frame_slot_of), _ptr(frames), _stream(stream))
        if check:
            _chk(st, "oc_joint_groups")
        return st

    def match_joint(self, layout: Layout, x, frames, best_sim, best_idx, stream=None, check: bool = True) -> int:
        cl = layout.c()
        st = _lib.oc_match_joint(self._h, C.byref(cl), _ptr(x), _ptr(frames), _ptr(best_sim), _ptr(best_idx),
                                 _stream(stream))
        if check:
            _chk(st, "oc_match_joint")
        return st

    def select_joint(self, layout: Layout, frames, best_sim, best_idx, mode: int, thr: float, n_reuse_pair: int,
                     n_reuse_single: int, y_stride: int, kept_idx, kept_count, match_map, slot_of, stream=None,
                     check: bool = True) -> int:
        cl = layout.c()
        st = _lib.oc_select_joint(self._h, C.byref(cl), _ptr(frames), _ptr(best_sim), _ptr(best_idx), mode, thr,
                                  n_reuse_pair, n_reuse_single, y_stride, _ptr(kept_idx), _ptr(kept_count),
                                  _ptr(match_map), _ptr(slot_of), _stream(stream))
        if check:
            _chk(st, "oc_select_joint")
        return st

    def match_frame_levels(self, layout: Layout, x, grids, best_sim, best_idx, pos_sim=None, pair_sim=None,
                           stream=None, check: bool = True) -> int:
        """oc_match_frame_levels: ``grids`` is a sequence of (gy, gx) pairs (host side)."""
        cl = layout.c()
        flat = [int(v) for g in grids for v in g]
        arr = (C.c_int32 * max(len(flat), 1))(*flat)
        st = _lib.oc_match_frame_levels(self._h, C.byref(cl), _ptr(x), len(grids), arr, _ptr(best_sim),
                                        _ptr(best_idx), _ptr(pos_sim), _ptr(pair_sim), _stream(stream))
        if check:
            _chk(st, "oc_match_frame_levels")
        return st

    def select(self, layout: Layout, best_sim, best_idx, mode: int, thr: float, n_reuse_per_group: int,
               y_group_stride: int, kept_idx, kept_count, match_map, slot_of, stream=None,
               check: bool = True) -> int:
        cl = layout.c()
        st = _lib.oc_select(self._h, C.byref(cl), _ptr(best_sim), _ptr(best_idx), mode, thr,
                            n_reuse_per_group, y_group_stride, _ptr(kept_idx), _ptr(kept_count),
                            _ptr(match_map), _ptr(slot_of), _stream(stream))
        if check:
            _chk(st, "oc_select")
        return st

    def gather(self, rows: CRows, x, kept_idx, n_slots: int, y, stream=None, check: bool = True) -> int:
        st = _lib.oc_gather(self._h, C.byref(rows), _ptr(x), _ptr(kept_idx), n_slots, _ptr(y), _stream(stream))
        if check:
            _chk(st, "oc_gather")
        return st

    def restore(self, rows: CRows, z, cache, n_units: int, slot_of, match_map, out,
                src_mode: int = RESTORE_FROM_CACHE, stream=None, check: bool = True) -> int:
        st = _lib.oc_restore(self._h, C.byref(rows), _ptr(z), _ptr(cache), n_units, _ptr(slot_of),
                             _ptr(match_map), _ptr(out), src_mode, _stream(stream))
        if check:
            _chk(st, "oc_restore")
        return st

    def layer_cache_put(self, layer: int, step: int, src, nbytes: int | None = None, stream=None,
                        check: bool = True) -> int:
        if nbytes is None:
            nbytes = src.numel() * src.element_size()
        st = _lib.oc_layer_cache_put(self._h, layer, step, _ptr(src), nbytes, _stream(stream))
        if check:
            _chk(st, "oc_layer_cache_put")
        return st

    def layer_cache_get(self, layer: int, step: int, interval: int, dst=None, stream=None):
        """Returns (hit, view pointer, bytes).  Raises on errors other than a miss."""
        view, nbytes = C.c_void_p(), C.c_size_t()
        st = _lib.oc_layer_cache_get(self._h, layer, step, interval, _ptr(dst), C.byref(view), C.byref(nbytes),
                                     _stream(stream))
        if st == CACHE_MISS:
            return False, None, 0
        _chk(st, "oc_layer_cache_get")
        return True, view.value, nbytes.value

    def layer_cache_clear(self) -> None:
        _chk(_lib.oc_layer_cache_clear(self._h), "oc_layer_cache_clear")

    def cache_step_host(self, layout: Layout, mode: int, thr: float, n_reuse_per_group: int, x_host, cache_host,
                        out_host, kept_count_host=None, stream=None, check: bool = True) -> int:
        """Host-buffer call: tensors are CPU (ideally pinned) torch tensors."""
        cl = layout.c()
        st = _lib.oc_cache_step_host(self._h, C.byref(cl), mode, thr, n_reuse_per_group, _ptr(x_host),
                                     _ptr(cache_host), _ptr(out_host), _ptr(kept_count_host), _stream(stream))
        if check:
            _chk(st, "oc_cache_step_host")
        return st
