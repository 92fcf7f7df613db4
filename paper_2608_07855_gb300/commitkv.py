"""Python binding of the CommitKV C ABI (include/commitkv.h).

Argument marshalling only: every step of the hot path runs in the CUDA
kernels of libcommitkv.so.  Tensors are torch tensors on the GPU (torch is
used for device memory and streams); the functions carry the C names.
There is no CPU fallback: without the compiled library or a GPU every call
raises.
"""
from __future__ import annotations

import ctypes
import os
import re
from dataclasses import dataclass
from typing import Optional, Sequence

from . import build as _build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "commitkv.h")
HEADERS = [os.path.join(ROOT, "include", f) for f in ("commitkv.h", "commitkv_testing.h")]

COMMITKV_OK = 0
COMMITKV_ERR_INVALID_ARG = 1
COMMITKV_ERR_UNSUPPORTED = 2
COMMITKV_ERR_CUDA = 3
COMMITKV_ERR_TIMEOUT = 4
COMMITKV_ERR_WORKSPACE = 5
COMMITKV_ERR_DEVICE_INPUT = 6
COMMITKV_F32 = 0
COMMITKV_BF16 = 1
MAX_TRAJ = 64


class CommitKVError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Shape(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("q_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float)]


class Traj(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("stride_layer", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("stride_tok", ctypes.c_int64), ("pos", ctypes.c_void_p), ("S", ctypes.c_int32),
                ("q", ctypes.c_void_p), ("q_pos", ctypes.c_void_p), ("W", ctypes.c_int32),
                ("page_start", ctypes.c_void_p), ("page_len", ctypes.c_void_p),
                ("P", ctypes.c_int32)]


class Packed(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("stride_layer", ctypes.c_int64), ("stride_head", ctypes.c_int64), ("stride_tok", ctypes.c_int64),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("scale_layer", ctypes.c_int64), ("scale_head", ctypes.c_int64), ("scale_tok", ctypes.c_int64),
                ("pos", ctypes.c_void_p), ("S", ctypes.c_int32),
                ("q", ctypes.c_void_p), ("q_pos", ctypes.c_void_p), ("W", ctypes.c_int32),
                ("page_start", ctypes.c_void_p), ("page_len", ctypes.c_void_p), ("P", ctypes.c_int32)]


class Rows(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("stride_layer", ctypes.c_int64),
                ("stride_head", ctypes.c_int64), ("stride_tok", ctypes.c_int64), ("first", ctypes.c_int32),
                ("count", ctypes.c_int32)]


class Thresholds(ctypes.Structure):
    _fields_ = [("tau_use", ctypes.c_float), ("tau_dead", ctypes.c_float),
                ("rho_use", ctypes.c_float), ("rho_dead", ctypes.c_float)]


_lib = None


def library_path() -> str:
    return _build.LIB


def load_library(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libcommitkv.so (building it in-tree with nvcc if needed)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path) or not _build.up_to_date():
        if not build_if_missing:
            raise RuntimeError(f"CommitKV CUDA library missing: {path}")
        path = _build.build()
    lib = ctypes.CDLL(path)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    P = ctypes.POINTER
    lib.commitkv_workspace_size.argtypes = [P(Shape), i32, P(Traj)]
    lib.commitkv_workspace_size.restype = sz
    lib.commitkv_workspace_init.argtypes = [vp, sz, vp]
    lib.commitkv_workspace_status.argtypes = [vp, sz, vp, i32]
    lib.commitkv_status_string.argtypes = [ctypes.c_int]
    lib.commitkv_status_string.restype = ctypes.c_char_p
    lib.commitkv_page_effects.argtypes = [P(Shape), i32, P(Traj), vp, vp, vp, vp, vp, sz, vp]
    lib.commitkv_page_effects_from_stats.argtypes = [P(Shape), i32, P(Traj), vp, vp, vp, vp, vp, sz, vp]
    lib.commitkv_classify.argtypes = [i32, vp, vp, vp, vp, P(Thresholds), vp, vp, vp, vp, sz, vp]
    lib.commitkv_classify_variant.argtypes = [i32, vp, vp, vp, vp, P(Thresholds), ctypes.c_uint32, vp, vp, vp,
                                              vp, sz, vp]
    lib.commitkv_joint_test.argtypes = [P(Shape), i32, P(Traj), vp, vp, vp, vp, ctypes.c_float,
                                        vp, vp, vp, sz, vp]
    lib.commitkv_compact.argtypes = [P(Shape), i32, P(Traj), vp, vp, vp, vp, vp, i32, i32, i32,
                                     vp, vp, vp, vp, vp, vp, sz, vp]
    lib.commitkv_compact_in_place.argtypes = [P(Shape), i32, P(Traj), vp, vp, vp, vp, vp, i32, i32, i32,
                                              vp, vp, vp, sz, vp]
    lib.commitkv_compact_noalloc.argtypes = [P(Shape), i32, P(Traj), vp, vp, vp, vp, vp, i32, i32,
                                             i32, vp, vp, vp, vp, vp, vp, vp]
    lib.commitkv_test_barrier_timeout.argtypes = [vp, sz, i32, vp]
    lib.commitkv_test_pruned_pages.argtypes = [vp, sz, vp, vp]
    lib.commitkv_test_launches.argtypes = []
    lib.commitkv_test_launches.restype = ctypes.c_uint64
    lib.commitkv_token_scores.argtypes = [P(Shape), i32, P(Traj), vp, vp, vp, vp, sz, vp]
    lib.commitkv_attention_workspace_size.argtypes = [P(Shape), i32, P(Traj), P(Traj)]
    lib.commitkv_attention_workspace_size.restype = sz
    lib.commitkv_window_attention.argtypes = [P(Shape), i32, P(Traj), vp, i32, i32, vp, vp, vp, sz, vp]
    lib.commitkv_prefix_attention.argtypes = [P(Shape), i32, P(Traj), P(Traj), vp, i32, i32, vp, vp, vp, sz, vp]
    lib.commitkv_packed_workspace_size.argtypes = [P(Shape), i32, P(Packed)]
    lib.commitkv_packed_workspace_size.restype = sz
    lib.commitkv_packed_write.argtypes = [P(Shape), i32, P(Packed), P(Rows), vp, vp]
    lib.commitkv_packed_read.argtypes = [P(Shape), i32, P(Packed), P(Rows), vp, vp]
    lib.commitkv_packed_attention.argtypes = [P(Shape), i32, P(Packed), vp, i32, i32, vp, vp, vp, sz, vp]
    lib.commitkv_packed_compact.argtypes = [P(Shape), i32, P(Packed), vp, vp, vp, vp, vp, i32, i32, i32, vp, vp,
                                            P(Packed), vp, sz, vp]
    for f in ("commitkv_workspace_init", "commitkv_workspace_status", "commitkv_page_effects",
              "commitkv_page_effects_from_stats", "commitkv_classify", "commitkv_classify_variant",
              "commitkv_joint_test", "commitkv_compact", "commitkv_compact_in_place", "commitkv_compact_noalloc",
              "commitkv_test_barrier_timeout", "commitkv_test_pruned_pages", "commitkv_token_scores",
              "commitkv_window_attention", "commitkv_prefix_attention", "commitkv_packed_write", "commitkv_packed_read",
              "commitkv_packed_attention", "commitkv_packed_compact"):
        getattr(lib, f).restype = ctypes.c_int
    _lib = lib
    return lib


def declared_functions() -> list:
    """Names of every entry point declared in the headers under include/."""
    names = set()
    for h in HEADERS:
        with open(h) as f:
            names |= set(re.findall(r"\b(commitkv_[a-z_]+)\s*\(", f.read()))
    return sorted(names)


def status_string(status: int) -> str:
    return load_library().commitkv_status_string(int(status)).decode()


def _check(rc: int, where: str):
    if rc != COMMITKV_OK:
        raise CommitKVError(rc, where)


# ----------------------------------------------------------------------------
# marshalling helpers (torch tensors -> pointers)


_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _torch().cuda.current_stream().cuda_stream or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _current_stream(device: int) -> int:
    """The handle of torch's current stream, without the Stream object (1.7 of
    a small call's 9.6 us), where this torch offers it."""
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream(device).cuda_stream if raw is None else raw(device)


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr() if x.numel() else None


def _ptr_array(xs, n) -> Optional[ctypes.Array]:
    if xs is None:
        return None
    return (ctypes.c_void_p * n)(*map(_ptr, xs))


def _require_cuda(*ts):
    for t in ts:
        if t is not None and not isinstance(t, int) and not t.is_cuda and t.numel():
            raise ValueError("CommitKV tensors must live on the GPU (no CPU fallback)")


@dataclass
class TrajTensors:
    """One trajectory's device tensors.

    k, v: [M][H][S][d] views (any strides with contiguous d); pos [S] int32;
    q [M][Hq][W][d] contiguous; q_pos [W] int32; page_start/page_len [P]."""
    k: object
    v: object
    pos: object
    q: object = None
    q_pos: object = None
    page_start: object = None
    page_len: object = None

    def desc(self) -> Traj:
        i32 = _torch().int32
        k, v, q, ps = self.k, self.v, self.q, self.page_start
        ints = (self.pos, self.q_pos, ps, self.page_len)
        _require_cuda(k, v, q, *ints)
        strides, shape = k.stride(), k.shape
        assert len(shape) == 4 and strides == v.stride() and shape == v.shape
        assert strides[3] == 1, "head_dim must be contiguous"
        for t in ints:
            assert t is None or t.dtype == i32
        if q is not None:
            assert q.is_contiguous() and q.dtype == k.dtype
        pos, q_pos, start, length = map(_ptr, ints)
        return Traj(_ptr(k), _ptr(v), strides[0], strides[1], strides[2], pos, shape[2], _ptr(q), q_pos,
                    0 if q is None else q.shape[2], start, length, 0 if ps is None else ps.numel())


def _one_gpu(*tensors) -> int:
    devices = {x.get_device() for x in tensors if x is not None}
    if len(devices) != 1 or min(devices) < 0:
        raise ValueError("CommitKV tensors must live on one GPU (no CPU fallback)")
    return devices.pop()


def _strides(x):
    """The strides of layers, heads and rows of x [M][H][n][w].  A dimension of one entry may have any
    (torch keeps what a view leaves there, contiguous() too), so it gets that of rows side by side."""
    M, H, n, w = x.shape
    if 0 in (M, H, n):
        return 0, 0, w
    layer, head, row, _ = x.stride()
    return layer if M > 1 else 0, head if H > 1 else 0, row if n > 1 else w


def _on_current(device: int):
    if _torch().cuda.current_device() != device:
        raise ValueError("the tensors must be on the current GPU")


@dataclass(frozen=True, eq=False)
class PackedTensors:
    """One trajectory's packed cache: device tensors in 4 bits a value.  Checked and
    marshalled once, at the first call that takes it; its tensors are not exchanged.

    k, v: codes [M][H][S][d / 2] uint8 views (any strides with contiguous bytes
    of a row), k_scale, v_scale: scale bytes [M][H][S][d / 32] uint8; the rest as
    in TrajTensors (pos may be None where a call does not read positions)."""
    k: object
    v: object
    k_scale: object
    v_scale: object
    pos: object = None
    q: object = None
    q_pos: object = None
    page_start: object = None
    page_len: object = None

    def desc(self) -> Packed:
        d = self.__dict__.get("_desc")
        if d is None:
            d = self._marshal()
            object.__setattr__(self, "_desc", d)
        return d

    def device(self) -> int:
        """The GPU of all its tensors."""
        d = self.__dict__.get("_device")
        if d is None:
            d = _one_gpu(self.k, self.v, self.k_scale, self.v_scale, self.pos, self.q, self.q_pos, self.page_start,
                         self.page_len)
            object.__setattr__(self, "_device", d)
        return d

    def _marshal(self) -> Packed:
        torch = _torch()
        k, v, ks, vs, q, ps = self.k, self.v, self.k_scale, self.v_scale, self.q, self.page_start
        ints = (self.pos, self.q_pos, ps, self.page_len)
        _require_cuda(k, v, ks, vs, q, *ints)
        for x in (k, v, ks, vs):
            if x.dtype != torch.uint8 or x.dim() != 4 or (x.numel() and x.stride(3) != 1):
                raise ValueError("codes and scales must be 4-D uint8, the bytes of a row contiguous")
        shape, strides, gstrides = k.shape, _strides(k), _strides(ks)
        if v.shape != shape or vs.shape != ks.shape or ks.shape[:3] != shape[:3] or 16 * ks.shape[3] != shape[3] or \
                _strides(v) != strides or _strides(vs) != gstrides:
            raise ValueError("codes must be [M][H][S][d / 2], scales [M][H][S][d / 32], of K and V alike")
        n = shape[2]
        for x in ints:
            if x is not None and (x.dtype != torch.int32 or x.dim() != 1 or not x.is_contiguous()):
                raise ValueError("positions and pages must be contiguous int32")
        if self.pos is not None and self.pos.numel() != n:
            raise ValueError("one position per cached token")
        if (ps is None) != (self.page_len is None) or (ps is not None and ps.numel() != self.page_len.numel()):
            raise ValueError("one length per page")
        W = 0 if q is None else q.shape[2]
        if q is not None and (q.dim() != 4 or not q.is_contiguous() or
                              (W and (self.q_pos is None or self.q_pos.numel() != W))):
            raise ValueError("q must be contiguous [M][Hq][W][d] with W positions")
        pos, q_pos, start, length = map(_ptr, ints)
        return Packed(_ptr(k), _ptr(v), strides[0], strides[1], strides[2], _ptr(ks), _ptr(vs), gstrides[0], gstrides[1],
                      gstrides[2], pos, n, _ptr(q), q_pos, W, start, length, 0 if ps is None else ps.numel())


def make_shape(M, H, Hq, d, dtype, softmax_scale=0.0) -> Shape:
    torch = _torch()
    code = {torch.float32: COMMITKV_F32, torch.bfloat16: COMMITKV_BF16}[dtype] \
        if not isinstance(dtype, int) else dtype
    return Shape(M, H, Hq, d, code, softmax_scale)


def _descs(trajs: Sequence[TrajTensors]):
    n = len(trajs)
    if not 1 <= n <= MAX_TRAJ:
        raise ValueError("1 <= n_traj <= 64")
    descs = [t.desc() for t in trajs]
    kind = type(descs[0])
    if any(type(d) is not kind for d in descs):
        raise ValueError("packed caches or full-width ones, not both")
    return (kind * n)(*descs)


def _mask(layer_mask, M):
    if layer_mask is None:
        return None, None
    buf = (ctypes.c_uint8 * M)(*[1 if x else 0 for x in layer_mask])
    return buf, ctypes.cast(buf, ctypes.c_void_p)


# ----------------------------------------------------------------------------
# entry points


def commitkv_workspace_size(shape: Shape, trajs: Sequence[TrajTensors]) -> int:
    d = _descs(trajs)
    n = load_library().commitkv_workspace_size(ctypes.byref(shape), len(trajs), d)
    if n == 0:
        raise CommitKVError(COMMITKV_ERR_INVALID_ARG, "commitkv_workspace_size")
    return int(n)


def alloc_workspace(shape: Shape, trajs: Sequence[TrajTensors], device=None):
    """Allocate (with torch) and initialise a workspace for these trajectories."""
    return _alloc(commitkv_workspace_size(shape, trajs), device)


def _alloc(n: int, device):
    ws = _torch().empty(n + 256, dtype=_torch().uint8, device=device or "cuda")
    off = (-ws.data_ptr()) % 256
    ws = ws[off: off + n]
    commitkv_workspace_init(ws)
    return ws


def commitkv_workspace_init(ws, stream=None):
    _check(load_library().commitkv_workspace_init(_ptr(ws), ws.numel(), _stream(stream)),
           "commitkv_workspace_init")


def commitkv_workspace_status(ws, stream=None, clear: bool = True) -> int:
    return int(load_library().commitkv_workspace_status(_ptr(ws), ws.numel(), _stream(stream),
                                                        1 if clear else 0))


def commitkv_test_barrier_timeout(ws, blocks=2, stream=None):
    _check(load_library().commitkv_test_barrier_timeout(_ptr(ws), ws.numel(), int(blocks),
                                                        _stream(stream)),
           "commitkv_test_barrier_timeout")


def commitkv_test_pruned_pages(ws, stream=None):
    """(row tile, page) pairs that the two list passes of the last scoring
    launch scored; (0, 0) where the full page pass ran."""
    out = (ctypes.c_uint64 * 2)()
    _check(load_library().commitkv_test_pruned_pages(_ptr(ws), ws.numel(), out, _stream(stream)),
           "commitkv_test_pruned_pages")
    return out[0], out[1]


def commitkv_test_launches() -> int:
    """Kernels that this thread's calls have launched so far."""
    return load_library().commitkv_test_launches()


def commitkv_page_effects(shape: Shape, trajs, R_out, head_R_out=None, stats_out=None,
                          layer_mask=None, workspace=None, stream=None):
    n = len(trajs)
    d = _descs(trajs)
    _mbuf, mptr = _mask(layer_mask, shape.layers)
    _require_cuda(*R_out)
    rc = load_library().commitkv_page_effects(
        ctypes.byref(shape), n, d, mptr, _ptr_array(R_out, n), _ptr_array(head_R_out, n),
        _ptr_array(stats_out, n), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(rc, "commitkv_page_effects")


def commitkv_page_effects_from_stats(shape: Shape, trajs, stats_in, R_out, head_R_out=None,
                                     layer_mask=None, workspace=None, stream=None):
    n = len(trajs)
    d = _descs(trajs)
    _mbuf, mptr = _mask(layer_mask, shape.layers)
    _require_cuda(*R_out)
    rc = load_library().commitkv_page_effects_from_stats(
        ctypes.byref(shape), n, d, mptr, _ptr_array(stats_in, n), _ptr_array(R_out, n),
        _ptr_array(head_R_out, n), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(rc, "commitkv_page_effects_from_stats")


def commitkv_token_scores(shape: Shape, trajs, stats, scores_out, layer_mask=None, workspace=None, stream=None):
    """Per-token fill scores (window attention with the given row stats)."""
    n = len(trajs)
    d = _descs(trajs)
    _mbuf, mptr = _mask(layer_mask, shape.layers)
    _require_cuda(*scores_out)
    rc = load_library().commitkv_token_scores(
        ctypes.byref(shape), n, d, mptr, _ptr_array(stats, n), _ptr_array(scores_out, n), _ptr(workspace),
        workspace.numel(), _stream(stream))
    _check(rc, "commitkv_token_scores")


def commitkv_classify(P, R_pre, R_post, eligible, state_out, cand_out, n_cand_out, workspace,
                      thresholds: Optional[Thresholds] = None, stream=None):
    n = len(P)
    Parr = (ctypes.c_int32 * n)(*[int(p) for p in P])
    rc = load_library().commitkv_classify(
        n, ctypes.cast(Parr, ctypes.c_void_p), _ptr_array(R_pre, n), _ptr_array(R_post, n),
        _ptr_array(eligible, n), ctypes.byref(thresholds) if thresholds else None,
        _ptr_array(state_out, n), _ptr_array(cand_out, n), _ptr(n_cand_out), _ptr(workspace),
        workspace.numel(), _stream(stream))
    _check(rc, "commitkv_classify")


COMMITKV_CLASSIFY_NO_PRECOMMIT = 1
COMMITKV_CLASSIFY_NO_PERCENTILE = 2


def commitkv_classify_variant(P, R_pre, R_post, eligible, variant, state_out, cand_out, n_cand_out,
                              workspace, thresholds: Optional[Thresholds] = None, stream=None):
    n = len(P)
    Parr = (ctypes.c_int32 * n)(*[int(p) for p in P])
    rc = load_library().commitkv_classify_variant(
        n, ctypes.cast(Parr, ctypes.c_void_p), _ptr_array(R_pre, n), _ptr_array(R_post, n),
        _ptr_array(eligible, n), ctypes.byref(thresholds) if thresholds else None, int(variant),
        _ptr_array(state_out, n), _ptr_array(cand_out, n), _ptr(n_cand_out), _ptr(workspace),
        workspace.numel(), _stream(stream))
    _check(rc, "commitkv_classify_variant")


def commitkv_joint_test(shape: Shape, post, stats, cand, n_cand, tau_joint, accepted_out,
                        step_R_out=None, layer_mask=None, workspace=None, stream=None):
    n = len(post)
    d = _descs(post)
    _mbuf, mptr = _mask(layer_mask, shape.layers)
    rc = load_library().commitkv_joint_test(
        ctypes.byref(shape), n, d, mptr, _ptr_array(stats, n), _ptr_array(cand, n), _ptr(n_cand),
        float(tau_joint), _ptr_array(accepted_out, n), _ptr_array(step_R_out, n), _ptr(workspace),
        workspace.numel(), _stream(stream))
    _check(rc, "commitkv_joint_test")


def commitkv_compact(shape: Shape, cache, retired, pending, pending_priority, fill_score, budget_B,
                     pending_tokens_BN, pending_cap_pages, idx_out, n_idx_out, k_out=None,
                     v_out=None, pos_out=None, workspace=None, stream=None):
    n = len(cache)
    d = _descs(cache)
    npend = (ctypes.c_int32 * n)(*[0 if p is None else int(p.numel()) for p in pending])
    rc = load_library().commitkv_compact(
        ctypes.byref(shape), n, d, _ptr_array(retired, n), _ptr_array(pending, n),
        ctypes.cast(npend, ctypes.c_void_p), _ptr_array(pending_priority, n),
        _ptr_array(fill_score, n), int(budget_B), int(pending_tokens_BN), int(pending_cap_pages),
        _ptr_array(idx_out, n), _ptr(n_idx_out), _ptr_array(k_out, n), _ptr_array(v_out, n),
        _ptr_array(pos_out, n), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(rc, "commitkv_compact")


def commitkv_compact_in_place(shape: Shape, cache, retired, pending, pending_priority, fill_score, budget_B,
                              pending_tokens_BN, pending_cap_pages, idx_out, n_idx_out, workspace=None,
                              stream=None):
    """commitkv_compact with the gather inside the caches: K and V row I_j
    of every (layer, KV head) slice moves to row j of the same slice, and
    pos[j] = pos[I_j], for j < n_idx_out[t]; the caches' k, v and pos
    tensors are overwritten."""
    n = len(cache)
    d = _descs(cache)
    npend = (ctypes.c_int32 * n)(*[0 if p is None else int(p.numel()) for p in pending])
    rc = load_library().commitkv_compact_in_place(
        ctypes.byref(shape), n, d, _ptr_array(retired, n), _ptr_array(pending, n),
        ctypes.cast(npend, ctypes.c_void_p), _ptr_array(pending_priority, n),
        _ptr_array(fill_score, n), int(budget_B), int(pending_tokens_BN), int(pending_cap_pages),
        _ptr_array(idx_out, n), _ptr(n_idx_out), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(rc, "commitkv_compact_in_place")


def commitkv_compact_noalloc(shape: Shape, cache, retired, pending, pending_priority, fill_score,
                             budget_B, pending_tokens_BN, pending_cap_pages, idx_out, n_idx_out,
                             k_out=None, v_out=None, pos_out=None, status_out=None, stream=None):
    """commitkv_compact with the library's fixed device scratch instead of a
    workspace, for callers that cannot allocate device memory when they
    compact.  Calls on one device share that scratch, so calls that can
    overlap on the GPU must be serialised; status_out (device int32 [1])
    receives the call's device-side status."""
    n = len(cache)
    d = _descs(cache)
    npend = (ctypes.c_int32 * n)(*[0 if p is None else int(p.numel()) for p in pending])
    rc = load_library().commitkv_compact_noalloc(
        ctypes.byref(shape), n, d, _ptr_array(retired, n), _ptr_array(pending, n),
        ctypes.cast(npend, ctypes.c_void_p), _ptr_array(pending_priority, n),
        _ptr_array(fill_score, n), int(budget_B), int(pending_tokens_BN), int(pending_cap_pages),
        _ptr_array(idx_out, n), _ptr(n_idx_out), _ptr_array(k_out, n), _ptr_array(v_out, n),
        _ptr_array(pos_out, n), _ptr(status_out), _stream(stream))
    _check(rc, "commitkv_compact_noalloc")


def _packed_width(shape: Shape, t: PackedTensors):
    M, H, _, w = t.k.shape
    if M != shape.layers or H != shape.kv_heads or 2 * w != shape.head_dim:
        raise ValueError(f"codes must be [{shape.layers}][{shape.kv_heads}][S][{shape.head_dim // 2}] of the shape")


class AttentionBatch:
    """The arguments of an attention call, checked and marshalled once: the
    trajectories, their outputs and a shared prefix, for callers that issue
    many calls on the same buffers.  Caches that grow in place are passed as
    the whole buffers, and set_length says how many tokens they hold (the
    workspace does not depend on it, but for packed caches, which it serves up
    to the lengths it was made for).  The trajectories are TrajTensors, or all
    PackedTensors (without a prefix).  The batch keeps the tensors alive."""

    def __init__(self, shape: Shape, trajs: Sequence[TrajTensors], out, lse_out=None, prefix: TrajTensors = None):
        torch = _torch()
        n = len(trajs)
        self.shape, self.trajs, self.descs = shape, trajs, _descs(trajs)
        self.prefix = None if prefix is None else prefix.desc()
        self.tensors = (trajs, prefix, out, lse_out)
        if len(out) != n or (lse_out is not None and len(lse_out) != n):
            raise ValueError("one output per trajectory")
        M, H, Hq, d = shape.layers, shape.kv_heads, shape.q_heads, shape.head_dim
        dt = torch.bfloat16 if shape.dtype == COMMITKV_BF16 else torch.float32
        devices = set()
        self.packed = isinstance(trajs[0], PackedTensors)
        if self.packed and prefix is not None:
            raise ValueError("packed caches take no shared prefix")
        for i, t in enumerate(list(trajs) + ([prefix] if prefix is not None else [])):
            if self.packed:
                _packed_width(shape, t)
                if t.pos is None or (t.q is not None and t.q.dtype != dt):
                    raise ValueError(f"packed caches need positions, and q of {dt}")
                devices |= {t.k_scale.device, t.v_scale.device}
            elif t.k.shape[0] != M or t.k.shape[1] != H or t.k.shape[3] != d or t.k.dtype != dt or t.v.dtype != dt:
                raise ValueError(f"K and V must be [{M}][{H}][S][{d}] of {dt}")
            if t.pos.shape != (t.k.shape[2],) or not t.pos.is_contiguous():
                raise ValueError("pos must be contiguous, one position per cached token")
            devices |= {x.device for x in (t.k, t.v, t.pos)}
            if i >= n:
                continue
            W = 0 if t.q is None else t.q.shape[2]
            if W and (tuple(t.q.shape) != (M, Hq, W, d) or t.q_pos is None or t.q_pos.shape != (W,) or
                      not t.q_pos.is_contiguous()):
                raise ValueError(f"q must be [{M}][{Hq}][W][{d}] with W contiguous positions")
            lse = None if lse_out is None else lse_out[i]
            for x, want, kind, what in ((out[i], (M, Hq, W, d), dt, "out"), (lse, (M, Hq, W), torch.float32, "lse_out")):
                if x is None and (what == "lse_out" or W == 0):
                    continue
                if x is None or tuple(x.shape) != want or x.dtype != kind or not x.is_contiguous():
                    raise ValueError(f"{what} must be contiguous {want} of {kind}")
                devices.add(x.device)
            devices |= {x.device for x in (t.q, t.q_pos) if x is not None}
        if len(devices) != 1 or next(iter(devices)).type != "cuda":
            raise ValueError("CommitKV tensors must live on one GPU (no CPU fallback)")
        self.device = next(iter(devices)).index
        self._out, self._lse = _ptr_array(out, n), _ptr_array(lse_out, n)
        # what every call passes, converted once
        self._args = (ctypes.byref(shape), n, self.descs)
        self._prefix = None if prefix is None else ctypes.byref(self.prefix)

    def set_length(self, i: int, S: int):
        """Trajectory i's cache has S tokens, the first ones of its tensors."""
        if not 0 <= S <= self.trajs[i].k.shape[2]:
            raise ValueError(f"0 <= S <= {self.trajs[i].k.shape[2]}, the tokens of the tensors")
        self.descs[i].S = S


def attention_batch(shape: Shape, trajs: Sequence[TrajTensors], out, lse_out=None, prefix=None) -> AttentionBatch:
    return AttentionBatch(shape, trajs, out, lse_out, prefix)


def commitkv_attention_workspace_size(shape: Shape, trajs: Sequence[TrajTensors], prefix: TrajTensors = None) -> int:
    p = None if prefix is None else ctypes.byref(prefix.desc())
    n = load_library().commitkv_attention_workspace_size(ctypes.byref(shape), len(trajs), _descs(trajs), p)
    if n == 0:
        raise CommitKVError(COMMITKV_ERR_INVALID_ARG, "commitkv_attention_workspace_size")
    return int(n)


def alloc_attention_workspace(shape: Shape, trajs: Sequence[TrajTensors], prefix: TrajTensors = None, device=None):
    """Allocate (with torch) and initialise a workspace for the attention
    calls on these trajectories."""
    return _alloc(commitkv_attention_workspace_size(shape, trajs, prefix), device)


def _attention(name, shape, trajs, prefix, out, lse_out, window, sinks, layer_mask, workspace, stream):
    b = trajs
    if not isinstance(b, AttentionBatch):
        if not 1 <= len(trajs) <= MAX_TRAJ:
            raise ValueError("1 <= n_traj <= 64")
        b = AttentionBatch(shape, trajs, out, lse_out, prefix)
    elif out is not None or lse_out is not None or prefix is not None or \
            (b.shape is not shape and bytes(b.shape) != bytes(shape)):
        raise ValueError("the outputs, the prefix and the shape are those of the batch")
    if b.packed != (name == "commitkv_packed_attention"):
        raise ValueError("packed caches and commitkv_packed_attention go together")
    if (b._prefix is None) == (name == "commitkv_prefix_attention"):
        raise ValueError("commitkv_prefix_attention takes a prefix, commitkv_window_attention none")
    if not (-1 << 31 <= window < 1 << 31 and -1 << 31 <= sinks < 1 << 31):
        raise ValueError("window and sinks are 32-bit")
    torch = _torch()
    if workspace is None or workspace.get_device() != b.device or torch.cuda.current_device() != b.device:
        raise ValueError("the batch and the workspace must be on the current GPU")
    _mbuf, mptr = _mask(layer_mask, shape.layers)
    if stream is None:
        stream = _current_stream(b.device)
    more = () if b._prefix is None else (b._prefix,)
    rc = getattr(_lib or load_library(), name)(
        *b._args, *more, mptr, window, sinks, b._out, b._lse, workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != COMMITKV_OK:
        raise CommitKVError(rc, name)


def commitkv_window_attention(shape: Shape, trajs, out=None, lse_out=None, window: int = 0, sinks: int = 0,
                              layer_mask=None, workspace=None, stream=None):
    """Attention of every trajectory's queries over its resident cache, with a
    sliding window and sink tokens; trajs may be an AttentionBatch (then
    without out and lse_out)."""
    _attention("commitkv_window_attention", shape, trajs, None, out, lse_out, window, sinks, layer_mask, workspace,
               stream)


def commitkv_prefix_attention(shape: Shape, trajs, prefix=None, out=None, lse_out=None, window: int = 0,
                              sinks: int = 0, layer_mask=None, workspace=None, stream=None):
    """commitkv_window_attention over a shared prefix and the trajectories'
    own caches together; trajs may be an AttentionBatch with a prefix."""
    _attention("commitkv_prefix_attention", shape, trajs, prefix, out, lse_out, window, sinks, layer_mask, workspace,
               stream)


# ----------------------------------------------------------------------------
# packed caches


def commitkv_packed_attention(shape: Shape, trajs, out=None, lse_out=None, window: int = 0, sinks: int = 0,
                              layer_mask=None, workspace=None, stream=None):
    """commitkv_window_attention over packed caches (PackedTensors); trajs may
    be an AttentionBatch of them."""
    _attention("commitkv_packed_attention", shape, trajs, None, out, lse_out, window, sinks, layer_mask, workspace,
               stream)


def alloc_packed_cache(shape: Shape, capacity: int, device="cuda") -> PackedTensors:
    """An empty packed cache with room for `capacity` tokens."""
    torch = _torch()
    M, H, d = shape.layers, shape.kv_heads, shape.head_dim

    def zeros(width):
        return torch.zeros(M, H, capacity, width, dtype=torch.uint8, device=device)

    return PackedTensors(zeros(d // 2), zeros(d // 2), zeros(d // 32), zeros(d // 32),
                         torch.zeros(capacity, dtype=torch.int32, device=device))


def commitkv_packed_workspace_size(shape: Shape, trajs: Sequence[PackedTensors]) -> int:
    n = load_library().commitkv_packed_workspace_size(ctypes.byref(shape), len(trajs), _descs(trajs))
    if n == 0:
        raise CommitKVError(COMMITKV_ERR_INVALID_ARG, "commitkv_packed_workspace_size")
    return int(n)


def alloc_packed_workspace(shape: Shape, trajs: Sequence[PackedTensors], device=None):
    """Allocate (with torch) and initialise a workspace for the attention and
    the checkpoints of these packed caches."""
    return _alloc(commitkv_packed_workspace_size(shape, trajs), device)


class PackedRows:
    """The arguments of a write or a read, checked and marshalled once: packed
    caches, the full-width rows k, v [M][H][n][d] of each (any strides with
    contiguous d) and the token at which they begin.  Keeps the tensors alive."""

    def __init__(self, shape: Shape, caches: Sequence[PackedTensors], k, v, first: Sequence[int]):
        torch = _torch()
        n = len(caches)
        if not 1 <= n <= MAX_TRAJ or len(k) != n or len(v) != n or len(first) != n:
            raise ValueError("1 <= n_traj <= 64, rows and a first token for each")
        if not all(isinstance(c, PackedTensors) for c in caches):
            raise ValueError("caches must be PackedTensors")
        self.shape, self.tensors = shape, (caches, k, v)
        self.descs = _descs(caches)
        M, H, d = shape.layers, shape.kv_heads, shape.head_dim
        dt = torch.bfloat16 if shape.dtype == COMMITKV_BF16 else torch.float32
        self.rows = (Rows * n)()
        for i, (c, x, y) in enumerate(zip(caches, k, v)):
            _packed_width(shape, c)
            if x.dim() != 4 or tuple(x.shape) != (M, H, x.shape[2], d) or y.shape != x.shape or x.dtype != dt or \
                    y.dtype != dt or (x.numel() and (_strides(x) != _strides(y) or x.stride(3) != 1 or y.stride(3) != 1)):
                raise ValueError(f"rows must be [{M}][{H}][n][{d}] of {dt} with contiguous channels, K and V alike")
            self.rows[i] = Rows(_ptr(x), _ptr(y), *_strides(x), 0, 0)
        # once, and not in every call
        self.device = _one_gpu(*[t for c in caches for t in (c.k, c.v, c.k_scale, c.v_scale)], *k, *v)
        _on_current(self.device)
        for i, f in enumerate(first):
            self.set_rows(i, f)

    def set_rows(self, i: int, first: int, count: int = None):
        """Trajectory i's rows, or the first `count` of them, stand at tokens first .. of its cache."""
        caches, k, _ = self.tensors
        count = k[i].shape[2] if count is None else count
        if not (0 <= count <= k[i].shape[2] and 0 <= first <= caches[i].k.shape[2] - count):
            raise ValueError("rows outside the cache")
        self.rows[i].first, self.rows[i].count = first, count


def packed_rows(shape: Shape, caches: Sequence[PackedTensors], k, v, first) -> PackedRows:
    return PackedRows(shape, caches, k, v, first)


def _packed_copy(name, shape, caches, k, v, first, layer_mask, stream):
    r = caches
    if not isinstance(r, PackedRows):
        r = PackedRows(shape, caches, k, v, first)
    elif k is not None or v is not None or first is not None or \
            (r.shape is not shape and bytes(r.shape) != bytes(shape)):
        raise ValueError("the rows and the shape are those of the PackedRows")
    _on_current(r.device)
    _mbuf, mptr = _mask(layer_mask, shape.layers)
    if stream is None:
        stream = _current_stream(r.device)
    rc = getattr(_lib or load_library(), name)(ctypes.byref(r.shape), len(r.rows), r.descs, r.rows, mptr, _stream(stream))
    _check(rc, name)


def commitkv_packed_write(shape: Shape, caches, k=None, v=None, first=None, layer_mask=None, stream=None):
    """New tokens' rows into their places of packed caches; caches may be
    PackedRows (then without k, v and first)."""
    _packed_copy("commitkv_packed_write", shape, caches, k, v, first, layer_mask, stream)


def commitkv_packed_read(shape: Shape, caches, k=None, v=None, first=None, layer_mask=None, stream=None):
    """Rows of packed caches as full-width values, into k and v; caches may be
    PackedRows (then without k, v and first)."""
    _packed_copy("commitkv_packed_read", shape, caches, k, v, first, layer_mask, stream)


def commitkv_packed_compact(shape: Shape, cache, retired, pending, pending_priority, fill_score, budget_B,
                            pending_tokens_BN, pending_cap_pages, idx_out, n_idx_out, dst=None, workspace=None,
                            stream=None):
    """commitkv_compact for packed caches, into the caches `dst`; without them in
    place, as commitkv_compact_in_place."""
    torch = _torch()
    n = len(cache)
    if dst is not None and len(dst) != n:
        raise ValueError("one destination per cache")
    if workspace is None:
        raise ValueError("a workspace is needed")
    for xs, what in ((retired, "retired"), (pending, "pending"), (pending_priority, "pending_priority"),
                     (fill_score, "fill_score"), (idx_out, "idx_out")):
        if len(xs) != n:
            raise ValueError(f"{what}: one for each cache")
    device = workspace.get_device()
    for c in (cache if dst is None else [*cache, *dst]):
        if not isinstance(c, PackedTensors):
            raise ValueError("caches must be PackedTensors")
        _packed_width(shape, c)
        if c.device() != device:
            raise ValueError("CommitKV tensors must live on one GPU (no CPU fallback)")
    descs, to = _descs(cache), None if dst is None else _descs(dst)

    def pointer(x, dt, least, what):
        m = 0 if x is None else x.numel()
        if m < least:
            raise ValueError("scores for every token, marks and priorities for every page, budget_B indices, a count per cache")
        if x is None:
            return None
        if x.dtype is not dt or not x.is_contiguous():
            raise ValueError(f"{what} must be contiguous {dt}")
        if x.get_device() != device:
            raise ValueError("CommitKV tensors must live on one GPU (no CPU fallback)")
        return x.data_ptr() if m else None

    u8, i32, f32 = torch.uint8, torch.int32, torch.float32
    array = ctypes.c_void_p * n
    marks, some, prio, fill, idx = array(), array(), array(), array(), array()
    npend = (ctypes.c_int32 * n)()
    for i, (c, x) in enumerate(zip(descs, pending)):
        P, m = c.P, 0 if x is None else x.numel()
        npend[i] = m
        marks[i] = pointer(retired[i], u8, P, "retired")
        some[i] = pointer(x, i32, 0, "pending")
        prio[i] = pointer(pending_priority[i], f32, P if m else 0, "pending_priority")
        fill[i] = pointer(fill_score[i], f32, c.S, "fill_score")
        idx[i] = pointer(idx_out[i], i32, budget_B, "idx_out")
    counts = pointer(n_idx_out, i32, n, "n_idx_out")
    _on_current(device)
    rc = (_lib or load_library()).commitkv_packed_compact(
        ctypes.byref(shape), n, descs, marks, some, ctypes.byref(npend), prio, fill, int(budget_B), int(pending_tokens_BN),
        int(pending_cap_pages), idx, counts, to, workspace.data_ptr(), workspace.numel(),
        _stream(_current_stream(device) if stream is None else stream))
    _check(rc, "commitkv_packed_compact")
