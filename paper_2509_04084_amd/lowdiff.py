"""ctypes binding of the LowDiff C ABI (include/lowdiff.h): argument marshalling only.

Every function takes torch tensors that already live on the GPU, hands their
device addresses and the current HIP stream to the library, and returns.  All
arithmetic happens in the HIP kernels; there is no fallback - if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import importlib
import math
import os
from typing import List, NamedTuple, Optional, Sequence, Tuple

import numpy as np
import torch

from . import _build

LD_OK = 0
LD_MERGE_AUTO, LD_MERGE_SWEEP, LD_MERGE_SCATTER = 0, 1, 2
LD_COMPRESS_AUTO, LD_COMPRESS_FULL = 0, 1
LD_MAX_WINDOW = 4096
LD_MAX_ADAM_WINDOW = 64

_lib = None
_gather = None  # _marshal.gather (csrc/ld_marshal.cpp), or _gather_tensors


class LowDiffError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn}: {status_string(status)} ({status})")


def library_path() -> str:
    return _build.LIB


def _gather_tensors(tensors, dtype, pinned):
    """_marshal.gather in Python: the same answers, a few microseconds per tensor more."""
    tensors = list(tensors)
    if not isinstance(dtype, torch.dtype):
        raise TypeError("gather: a torch.dtype expected")
    ptr, sizes, device, bad = np.zeros(len(tensors), np.uint64), np.zeros(len(tensors), np.int64), -2, -1
    for i, t in enumerate(tensors):
        if not isinstance(t, torch.Tensor):
            raise TypeError("a torch tensor expected")
        at = t.get_device() if t.is_cuda else -1
        device = at if i == 0 or device == at else -2
        if t.dtype == dtype and t.is_contiguous() and (t.is_cuda or (pinned and t.is_pinned())):
            ptr[i] = t.data_ptr()
        elif bad < 0:
            bad = i
        sizes[i] = t.numel()
    return ptr.tobytes(), sizes.tobytes(), device, bad


def _load_gather():
    """The compiled gather. It holds only for the torch and the Python that it was built with: one that does not load
    is built anew, and where that cannot be done (no compiler, no headers) Python does its work."""
    for build in (False, True):
        try:
            if build or not os.path.exists(_build.MARSHAL):
                _build.build_marshal(force=True)
            importlib.invalidate_caches()
            return importlib.import_module("._marshal", __package__).gather
        except (ImportError, OSError, RuntimeError, AttributeError):
            pass  # also: a torch that does not tell how it was built
    return _gather_tensors


def load() -> ctypes.CDLL:
    """Loads liblowdiff.so (building it only if no built library is present)."""
    global _lib, _gather
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build_library(force=True)
    if _gather is None:
        _gather = _load_gather()
    lib = ctypes.CDLL(_build.LIB)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    lib.ld_status_string.argtypes = [i32]
    lib.ld_status_string.restype = ctypes.c_char_p
    lib.ld_compress_topk_workspace.argtypes = [i32, vp]
    lib.ld_compress_topk_workspace.restype = sz
    lib.ld_merge_sparse_from_host_staging.argtypes = [vp, i32, i32]
    lib.ld_merge_sparse_from_host_staging.restype = sz
    lib.ld_merge_sparse_from_host.argtypes = [vp, i64, vp, vp, vp, i32, f32, i32, vp, sz, vp, sz, vp, vp]
    lib.ld_merge_sparse_from_host.restype = i32
    lib.ld_merge_sparse_from_host_events.argtypes = [vp, i64, vp, vp, vp, i32, f32, i32, vp, sz, vp, sz, vp, vp, vp]
    lib.ld_merge_sparse_from_host_events.restype = i32
    lib.ld_check_diff.argtypes = [vp, vp, i64, i64, vp, vp]
    lib.ld_check_diff.restype = i32
    lib.ld_compress_topk_workspace_for.argtypes = [i32, vp, vp]
    lib.ld_compress_topk_workspace_for.restype = sz
    lib.ld_compress_topk.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.ld_compress_topk.restype = i32
    lib.ld_compress_topk_strategy.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, sz, vp, i32]
    lib.ld_compress_topk_strategy.restype = i32
    lib.ld_compress_topk_paths.argtypes = [vp, sz, i32, vp, vp, vp, vp]
    lib.ld_compress_topk_paths.restype = i32
    lib.ld_snapshot_layer.argtypes = [vp, vp, i64, vp]
    lib.ld_snapshot_layer.restype = i32
    lib.ld_snapshot_layers.argtypes = [vp, vp, vp, i32, vp]
    lib.ld_snapshot_layers.restype = i32
    lib.ld_merge_sparse_workspace.argtypes = [i64, i32, vp]
    lib.ld_merge_sparse_workspace.restype = sz
    lib.ld_merge_sparse.argtypes = [vp, i64, vp, vp, vp, i32, f32, vp, sz, vp]
    lib.ld_merge_sparse.restype = i32
    lib.ld_merge_sparse_strategy.argtypes = [vp, i64, vp, vp, vp, i32, f32, vp, sz, vp, i32]
    lib.ld_merge_sparse_strategy.restype = i32
    lib.ld_merge_sparse_static_limit.argtypes = []
    lib.ld_merge_sparse_static_limit.restype = sz
    lib.ld_merge_sparse_static.argtypes = [vp, i64, vp, vp, vp, i32, f32, vp]
    lib.ld_merge_sparse_static.restype = i32
    lib.ld_merge_dense_adam.argtypes = [vp, vp, vp, i64, vp, i32, i64, f32, f32, f32, f32, vp]
    lib.ld_merge_dense_adam.restype = i32
    lib.ld_merge_sparse_adam_workspace.argtypes = [i64, i32, vp]
    lib.ld_merge_sparse_adam_workspace.restype = sz
    lib.ld_merge_sparse_adam.argtypes = [vp, vp, vp, i64, vp, vp, vp, i32, i64, f32, f32, f32, f32, vp, sz, vp]
    lib.ld_merge_sparse_adam.restype = i32
    lib.ld_combine_sparse_workspace.argtypes = [i64, i32]
    lib.ld_combine_sparse_workspace.restype = sz
    lib.ld_combine_sparse.argtypes = [vp, vp, vp, i32, i64, f32, vp, vp, i64, vp, vp, sz, vp]
    lib.ld_combine_sparse.restype = i32
    lib.ld_combine_sparse_strategy.argtypes = lib.ld_combine_sparse.argtypes + [i32]
    lib.ld_combine_sparse_strategy.restype = i32
    lib.ld_grad_norm_workspace.argtypes = [i32]
    lib.ld_grad_norm_workspace.restype = sz
    lib.ld_clip_grad_norm_workspace.argtypes = [i32, vp]
    lib.ld_clip_grad_norm_workspace.restype = sz
    lib.ld_grad_norm.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.ld_grad_norm.restype = i32
    lib.ld_clip_grads.argtypes = [vp, vp, vp, i32, i32, i32, vp, f32, vp]
    lib.ld_clip_grads.restype = i32
    lib.ld_clip_grad_norm.argtypes = [vp, vp, vp, i32, i32, i32, f32, vp, vp, sz, vp]
    lib.ld_clip_grad_norm.restype = i32
    lib.ld_embed_lookup.argtypes = [vp, i64, i64, vp, i64, i64, i32, vp, vp, i32, i64, i32, f32, vp, i64, i32, vp]
    lib.ld_embed_lookup.restype = i32
    lib.ld_embed_grad_workspace.argtypes = [i64, i64, i32]
    lib.ld_embed_grad_workspace.restype = sz
    lib.ld_embed_grad.argtypes = [vp, i64, i32, vp, i32, i64, i32, f32, vp, i64, i64, i32, i32, vp, sz, vp]
    lib.ld_embed_grad.restype = i32
    lib.ld_token_logprob_workspace.argtypes = [i64, i32, i32]
    lib.ld_token_logprob_workspace.restype = sz
    lib.ld_token_logprob.argtypes = [vp, i64, i32, i64, i32, vp, i32, f32, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.ld_token_logprob.restype = i32
    lib.ld_token_logprob_grad.argtypes = [vp, i64, i32, i64, i32, vp, i32, f32, vp, vp, i64, vp, vp, i64, vp, i64, i32, vp]
    lib.ld_token_logprob_grad.restype = i32
    lib.ld_orthogonalize_workspace.argtypes = [vp, vp, i32]
    lib.ld_orthogonalize_workspace.restype = sz
    lib.ld_orthogonalize.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, f32, vp, sz, vp]
    lib.ld_orthogonalize.restype = i32
    lib.ld_merge_dense_muon_workspace.argtypes = [vp, vp, i32, i32]
    lib.ld_merge_dense_muon_workspace.restype = sz
    lib.ld_merge_dense_muon.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, f32, f32, i32, f32, vp, i32, vp, f32, vp, sz, vp]
    lib.ld_merge_dense_muon.restype = i32
    dbl = ctypes.c_double
    lib.ld_config_wasted_time.argtypes = [vp, dbl, dbl, dbl, dbl]
    lib.ld_config_wasted_time.restype = dbl
    lib.ld_config_critical_interval.argtypes = [vp, dbl, dbl, dbl]
    lib.ld_config_critical_interval.restype = dbl
    lib.ld_config_select.argtypes = [vp, i32, vp, vp, vp, vp, vp]
    lib.ld_config_select.restype = i32
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().ld_status_string(int(status)).decode()


def _check(fn: str, status: int) -> None:
    if status != LD_OK:
        raise LowDiffError(fn, status)


# the current stream's handle without an object around it, where torch has that (0.3 us of a call instead of 2.9)
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> ctypes.c_void_p:
    if stream is not None:
        return ctypes.c_void_p(stream.cuda_stream)
    if _current_raw_stream is not None:
        return ctypes.c_void_p(_current_raw_stream(torch.cuda.current_device()))
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(t: Optional[torch.Tensor], dtype, name: str) -> ctypes.c_void_p:
    if t is None:
        return ctypes.c_void_p(0)
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous {dtype} tensor on the GPU")
    return ctypes.c_void_p(t.data_ptr())


def _same_device(*tensors) -> None:
    devs = {t.device for t in tensors if t is not None}
    if len(devs) > 1:
        raise ValueError(f"tensors lie on different devices: {sorted(map(str, devs))}")


class _Table:
    """Addresses, sizes and device of a list of tensors, for a call that takes host arrays of pointers."""

    def __init__(self, tensors: Sequence[torch.Tensor], dtype, pinned: bool = False):
        self.tensors, self.dtype, self.pinned = tensors, dtype, pinned
        self.ptr, self.sizes, self.device, self.bad = _gather(tensors, dtype, pinned)

    def numel(self) -> np.ndarray:
        return np.frombuffer(self.sizes, dtype=np.int64) if self.sizes else np.zeros(0, np.int64)

    def checked(self, name: str) -> bytes:
        """The addresses; raises if a tensor cannot be handed to the library."""
        if self.bad >= 0:
            (_dev_or_pinned if self.pinned else _dev)(self.tensors[self.bad], self.dtype, name)
            raise TypeError(f"{name}: expected a contiguous {self.dtype} tensor on the GPU")
        return self.ptr


def _one_device(first: torch.Tensor, others: Sequence, *tables: _Table) -> None:
    """_same_device over single tensors and the tensors of tables."""
    at = first.get_device()
    if at >= 0:
        for t in others:
            if t is not None and t.get_device() != at:
                break
        else:
            for b in tables:
                if b.sizes and b.device != at:
                    break
            else:
                return
    _same_device(first, *others, *(t for b in tables for t in b.tensors))


def _allocates_for(stream, device) -> bool:
    """Whether memory that torch's allocator gives now is that of `stream` (None: the current one), or no stream's."""
    return stream is None or torch.device(device).type != "cuda" or \
        (_current_raw_stream is not None and _current_raw_stream(stream.device_index) == stream.cuda_stream)


def _empty(dtype, device, stream, *shape) -> torch.Tensor:
    """An uninitialised tensor out of the memory that torch's allocator keeps for `stream`. What it keeps for another stream may be a
    block that was just given back and that kernels of that stream, still to run, use."""
    if _allocates_for(stream, device):
        return torch.empty(*shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(*shape, dtype=dtype, device=device)


def _record(t: torch.Tensor, *streams) -> torch.Tensor:
    """Marks a tensor the binding allocated as in use on these streams (None: the current one) besides the one it belongs to."""
    if t.is_cuda:
        for st in streams:
            t.record_stream(torch.cuda.current_stream() if st is None else st)
    return t


def _output(dtype, device, stream, *shape) -> torch.Tensor:
    """A tensor that a call writes on `stream` and returns. What reads it is taken to run there or on the current stream; once it is
    dropped, its memory is not handed out again before both have passed that point."""
    if stream is None or _allocates_for(stream, device):
        return torch.empty(*shape, dtype=dtype, device=device)
    return _record(_empty(dtype, device, stream, *shape), None)


def _scratch(nbytes: int, device, stream, *others) -> torch.Tensor:
    """A temporary the binding allocates itself and drops when the call returns, first written on `stream`. The block belongs to
    that stream, and is marked as in use on the other streams of the call: it is handed out again only behind the call's kernels,
    and holds nothing that others before them still use."""
    return _record(_empty(torch.uint8, device, stream, max(1, int(nbytes))), *others)


def _host(a, dtype) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=dtype)


def _hp(a: np.ndarray) -> ctypes.c_void_p:
    return ctypes.c_void_p(a.ctypes.data)


def ld_compress_topk_workspace(seg_off, seg_k=None) -> int:
    """Workspace bytes: the minimum, or with `seg_k` the size that keeps calls of that density fast."""
    seg_off = _host(seg_off, np.int64)
    if seg_k is None:
        return int(load().ld_compress_topk_workspace(seg_off.shape[0] - 1, _hp(seg_off)))
    seg_k = _host(seg_k, np.int32)
    if seg_k.shape[0] != seg_off.shape[0] - 1:
        raise ValueError("seg_k must have one entry per segment")
    return int(load().ld_compress_topk_workspace_for(seg_off.shape[0] - 1, _hp(seg_off), _hp(seg_k)))


def ld_compress_topk(grad: torch.Tensor, residual: torch.Tensor, seg_off, seg_k,
                     out_idx: Optional[torch.Tensor] = None, out_val: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, stream=None,
                     strategy: int = LD_COMPRESS_AUTO) -> Tuple[torch.Tensor, torch.Tensor]:
    """Per-segment top-k with error feedback; `residual` is updated in place.
    Returns (out_idx int32[K], out_val float32[K])."""
    lib = load()
    seg_off = _host(seg_off, np.int64)
    seg_k = _host(seg_k, np.int32)
    n_seg = int(seg_k.shape[0])
    if seg_off.shape[0] != n_seg + 1:
        raise ValueError("seg_off must have n_seg + 1 entries")
    if int(seg_off[-1]) != grad.numel() or grad.numel() != residual.numel():
        raise ValueError(f"segment table covers {int(seg_off[-1])} elements, grad has {grad.numel()}, "
                         f"residual has {residual.numel()}")
    _same_device(grad, residual, out_idx, out_val, workspace)
    K = int(seg_k.astype(np.int64).sum())
    if out_idx is None:
        out_idx = _output(torch.int32, grad.device, stream, K)
    if out_val is None:
        out_val = _output(torch.float32, grad.device, stream, K)
    if out_idx.numel() < K or out_val.numel() < K:
        raise ValueError("output buffers smaller than sum(seg_k)")
    if workspace is None:
        workspace = _scratch(lib.ld_compress_topk_workspace_for(n_seg, _hp(seg_off), _hp(seg_k)), grad.device, stream)
    st = lib.ld_compress_topk_strategy(
        _dev(grad, torch.float32, "grad"), _dev(residual, torch.float32, "residual"),
        _hp(seg_off), _hp(seg_k), n_seg,
        _dev(out_idx, torch.int32, "out_idx"), _dev(out_val, torch.float32, "out_val"),
        _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream), int(strategy))
    _check("ld_compress_topk", st)
    return out_idx, out_val


LD_PATH_CANDIDATES, LD_PATH_FULL, LD_PATH_TIES = 0, 1, 2


def ld_compress_topk_paths(workspace: torch.Tensor, seg_off, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(paths, overflowed_tiles), int32 device tensors of one entry per segment: which way the last
    ld_compress_topk call that used `workspace` took for each segment (see lowdiff.h)."""
    seg_off = _host(seg_off, np.int64)
    n_seg = int(seg_off.shape[0]) - 1
    paths = _output(torch.int32, workspace.device, stream, max(n_seg, 1))
    over = _output(torch.int32, workspace.device, stream, max(n_seg, 1))
    st = load().ld_compress_topk_paths(_dev(workspace, torch.uint8, "workspace"), workspace.numel(), n_seg,
                                       _hp(seg_off), _dev(paths, torch.int32, "paths"),
                                       _dev(over, torch.int32, "overflowed_tiles"), _stream(stream))
    _check("ld_compress_topk_paths", st)
    return paths[:n_seg], over[:n_seg]


def _dev_or_pinned(t: torch.Tensor, dtype, name: str) -> ctypes.c_void_p:
    """Device tensor, or a pinned host tensor (page-locked memory is mapped into the GPU's address space)."""
    if not t.is_cuda:
        if not t.is_pinned() or t.dtype != dtype or not t.is_contiguous():
            raise TypeError(f"{name}: expected a contiguous {dtype} tensor on the GPU or in pinned host memory")
        return ctypes.c_void_p(t.data_ptr())
    return _dev(t, dtype, name)


def ld_snapshot_layer(grad_bf16: torch.Tensor, snap_bf16: torch.Tensor, stream=None) -> None:
    """Copies one layer's gradient into `snap_bf16`: a device tensor, or a pinned host tensor (the
    paper's device-to-host snapshot; the copy then runs at the host link's speed)."""
    if grad_bf16.numel() != snap_bf16.numel():
        raise ValueError("snapshot source and destination differ in size")
    st = load().ld_snapshot_layer(_dev(grad_bf16, torch.bfloat16, "grad_bf16"),
                                  _dev_or_pinned(snap_bf16, torch.bfloat16, "snap_bf16"),
                                  grad_bf16.numel(), _stream(stream))
    _check("ld_snapshot_layer", st)


def ld_snapshot_layers(srcs: Sequence[torch.Tensor], dsts: Sequence[torch.Tensor], stream=None) -> None:
    lib = load()
    n = len(srcs)
    if len(dsts) != n:
        raise ValueError("srcs and dsts differ in length")
    s, d = _Table(srcs, torch.bfloat16), _Table(dsts, torch.bfloat16, pinned=True)
    sp, dp = s.checked("src"), d.checked("dst")
    if s.sizes != d.sizes:
        raise ValueError("snapshot source and destination differ in size")
    st = lib.ld_snapshot_layers(sp, dp, s.sizes, n, _stream(stream))
    _check("ld_snapshot_layers", st)


def ld_merge_sparse_workspace(n: int, K: Sequence[int]) -> int:
    K = _host(K, np.int64)
    return int(load().ld_merge_sparse_workspace(int(n), int(K.shape[0]), _hp(K)))


def ld_merge_sparse(w: torch.Tensor, idx: Sequence[torch.Tensor], val: Sequence[torch.Tensor], lr: float,
                    workspace: Optional[torch.Tensor] = None, stream=None,
                    strategy: int = LD_MERGE_AUTO) -> None:
    """Replays the diffs (idx[t], val[t]) onto `w` in list order, in place."""
    lib = load()
    W = len(idx)
    if len(val) != W:
        raise ValueError("idx and val differ in length")
    gi, gv = _Table(idx, torch.int32), _Table(val, torch.float32)
    if gi.sizes != gv.sizes:
        raise ValueError("idx[t] and val[t] differ in size")
    K = gi.numel()
    _one_device(w, (workspace,), gi, gv)
    ip, vp = gi.checked("idx"), gv.checked("val")
    if workspace is None:
        workspace = _scratch(lib.ld_merge_sparse_workspace(w.numel(), W, _hp(K)), w.device, stream)
    st = lib.ld_merge_sparse_strategy(_dev(w, torch.float32, "w"), w.numel(), ip, vp, _hp(K), W,
                                      ctypes.c_float(lr), _dev(workspace, torch.uint8, "workspace"),
                                      workspace.numel(), _stream(stream), int(strategy))
    _check("ld_merge_sparse", st)


def ld_merge_sparse_static_limit() -> int:
    return int(load().ld_merge_sparse_static_limit())


def ld_merge_sparse_static(w: torch.Tensor, idx: Sequence[torch.Tensor], val: Sequence[torch.Tensor], lr: float,
                           stream=None) -> None:
    """ld_merge_sparse without a workspace and without any allocation (its table lies in a
    device array of the library); refuses windows beyond ld_merge_sparse_static_limit()."""
    lib = load()
    W = len(idx)
    if len(val) != W:
        raise ValueError("idx and val differ in length")
    gi, gv = _Table(idx, torch.int32), _Table(val, torch.float32)
    if gi.sizes != gv.sizes:
        raise ValueError("idx[t] and val[t] differ in size")
    K = gi.numel()
    ip, vp = gi.checked("idx"), gv.checked("val")
    st = lib.ld_merge_sparse_static(_dev(w, torch.float32, "w"), w.numel(), ip, vp, _hp(K), W,
                                       ctypes.c_float(lr), _stream(stream))
    _check("ld_merge_sparse_static", st)


def ld_merge_dense_adam(w: torch.Tensor, m: torch.Tensor, v: torch.Tensor, grads_bf16: Sequence[torch.Tensor],
                        step0: int, lr: float, beta1: float, beta2: float, eps: float, stream=None) -> None:
    """Replays the bf16 gradients as Adam steps step0+1.. onto (w, m, v), in place."""
    lib = load()
    W = len(grads_bf16)
    if m.numel() != w.numel() or v.numel() != w.numel():
        raise ValueError("w, m, v differ in size")
    g = _Table(grads_bf16, torch.bfloat16)
    if np.any(g.numel() != w.numel()):
        raise ValueError("gradient and parameter sizes differ")
    _one_device(w, (m, v), g)
    gp = g.checked("grad")
    st = lib.ld_merge_dense_adam(_dev(w, torch.float32, "w"), _dev(m, torch.float32, "m"),
                                    _dev(v, torch.float32, "v"), w.numel(), gp, W, int(step0),
                                    ctypes.c_float(lr), ctypes.c_float(beta1), ctypes.c_float(beta2),
                                    ctypes.c_float(eps), _stream(stream))
    _check("ld_merge_dense_adam", st)


def ld_merge_sparse_from_host(w: torch.Tensor, idx: Sequence[torch.Tensor], val: Sequence[torch.Tensor], lr: float,
                              group: int = 4, staging: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, copy_stream=None,
                              merge_stream=None, events: Optional[Sequence[int]] = None) -> None:
    """ld_merge_sparse for diffs in (pinned) host tensors: groups of `group` diffs are copied on
    `copy_stream` while the previous group is merged on `merge_stream` (default: the current stream
    for both, i.e. no overlap). The host tensors must stay alive until the copies are done.
    `events`: four hipEvent_t handles of the caller's (then the call creates none of its own)."""
    lib = load()
    W = len(idx)
    if len(val) != W:
        raise ValueError("idx and val differ in length")
    for i, v in zip(idx, val):
        if i.is_cuda or v.is_cuda or i.dtype != torch.int32 or v.dtype != torch.float32 \
                or not i.is_contiguous() or not v.is_contiguous() or i.numel() != v.numel():
            raise TypeError("host diffs: contiguous CPU int32 / float32 tensors of equal length expected")
    K = np.array([t.numel() for t in idx], dtype=np.int64)
    n = w.numel()
    group = max(1, min(int(group), 64))
    if staging is None:
        staging = _scratch(max(256, int(lib.ld_merge_sparse_from_host_staging(_hp(K), W, group))), w.device,
                           copy_stream, merge_stream)
    if workspace is None:
        workspace = _scratch(max(256, int(lib.ld_merge_sparse_workspace(n, min(group, max(W, 1)), _hp(K)))),
                             w.device, merge_stream)
    ip = (ctypes.c_void_p * max(W, 1))(*[t.data_ptr() for t in idx])
    vp = (ctypes.c_void_p * max(W, 1))(*[t.data_ptr() for t in val])
    ev = None
    if events is not None:
        if len(events) != 4:
            raise ValueError("events: four hipEvent_t handles expected")
        ev = (ctypes.c_void_p * 4)(*[int(e) for e in events])
    st = lib.ld_merge_sparse_from_host_events(_dev(w, torch.float32, "w"), n, ip, vp, _hp(K), W, ctypes.c_float(lr),
                                              group, _dev(staging, torch.uint8, "staging"), staging.numel(),
                                              _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
                                              _stream(copy_stream), _stream(merge_stream), ev)
    _check("ld_merge_sparse_from_host", st)


def ld_check_diff(idx: torch.Tensor, val: Optional[torch.Tensor], n: int,
                  counts: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Counts (indices out of range, records not strictly ascending, NaN values) of one diff.
    Returns the 3-element int64 device tensor `counts`; all zero means the diff can be merged."""
    if val is not None and val.numel() != idx.numel():
        raise ValueError("idx and val differ in length")
    if counts is None:
        counts = _output(torch.int64, idx.device, stream, 3)
    if counts.numel() < 3:
        raise ValueError("counts needs 3 elements")
    st = load().ld_check_diff(_dev(idx, torch.int32, "idx"), _dev(val, torch.float32, "val"),
                              int(idx.numel()), int(n), _dev(counts, torch.int64, "counts"), _stream(stream))
    _check("ld_check_diff", st)
    return counts


def ld_merge_sparse_adam_workspace(n: int, K: Sequence[int]) -> int:
    K = _host(K, np.int64)
    return int(load().ld_merge_sparse_adam_workspace(int(n), int(K.shape[0]), _hp(K)))


def ld_merge_sparse_adam(w: torch.Tensor, m: torch.Tensor, v: torch.Tensor, idx: Sequence[torch.Tensor],
                         val: Sequence[torch.Tensor], step0: int, lr: float, beta1: float, beta2: float,
                         eps: float, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Replays the sparse diffs (idx[t], val[t]) as Adam steps step0+1.. onto (w, m, v), in place."""
    lib = load()
    W = len(idx)
    if len(val) != W:
        raise ValueError("idx and val differ in length")
    if m.numel() != w.numel() or v.numel() != w.numel():
        raise ValueError("w, m, v differ in size")
    gi, gv = _Table(idx, torch.int32), _Table(val, torch.float32)
    if gi.sizes != gv.sizes:
        raise ValueError("idx[t] and val[t] differ in size")
    K = gi.numel()
    _one_device(w, (m, v, workspace), gi, gv)
    ip, vp = gi.checked("idx"), gv.checked("val")
    if workspace is None:
        workspace = _scratch(lib.ld_merge_sparse_adam_workspace(w.numel(), W, _hp(K)), w.device, stream)
    st = lib.ld_merge_sparse_adam(_dev(w, torch.float32, "w"), _dev(m, torch.float32, "m"),
                                  _dev(v, torch.float32, "v"), w.numel(), ip, vp, _hp(K), W, int(step0),
                                  ctypes.c_float(lr), ctypes.c_float(beta1), ctypes.c_float(beta2),
                                  ctypes.c_float(eps), _dev(workspace, torch.uint8, "workspace"),
                                  workspace.numel(), _stream(stream))
    _check("ld_merge_sparse_adam", st)


def ld_combine_sparse(idx: Sequence[torch.Tensor], val: Sequence[torch.Tensor], n: int, scale: float = 1.0,
                      out_idx: Optional[torch.Tensor] = None, out_val: Optional[torch.Tensor] = None,
                      out_count: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Combines N per-worker record lists (values at equal indices added in list order).

    Returns (out_idx, out_val, out_count): the buffers (capacity sum K unless given) and a one-element
    int64 device tensor with the number of records; nothing is synchronized."""
    lib = load()
    N = len(idx)
    if len(val) != N:
        raise ValueError("idx and val differ in length")
    gi, gv = _Table(idx, torch.int32), _Table(val, torch.float32)
    if gi.sizes != gv.sizes:
        raise ValueError("idx[r] and val[r] differ in size")
    K = gi.numel()
    dev = idx[0].device if N else torch.device("cuda", torch.cuda.current_device())
    total = int(K.sum())
    if out_idx is None:
        out_idx = _output(torch.int32, dev, stream, total)
    if out_val is None:
        out_val = _output(torch.float32, dev, stream, total)
    if out_count is None:
        out_count = _output(torch.int64, dev, stream, 1)
    cap = min(out_idx.numel(), out_val.numel())
    _one_device(out_idx, (out_val, out_count, workspace), gi, gv)
    ip, vp = gi.checked("idx"), gv.checked("val")
    if workspace is None:
        workspace = _scratch(lib.ld_combine_sparse_workspace(int(n), N), dev, stream)
    st = lib.ld_combine_sparse(ip, vp, _hp(K), N, int(n), ctypes.c_float(scale),
                               _dev(out_idx, torch.int32, "out_idx"), _dev(out_val, torch.float32, "out_val"),
                               cap, _dev(out_count, torch.int64, "out_count"),
                               _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream))
    _check("ld_combine_sparse", st)
    return out_idx, out_val, out_count


def ld_combine_sparse_workspace(n: int, N: int) -> int:
    return int(load().ld_combine_sparse_workspace(int(n), int(N)))


_ELEM = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # LD_F32, LD_BF16, LD_F16
_ID = {torch.int32: 0, torch.int64: 1}                           # LD_I32, LD_I64


def _elem(t: torch.Tensor, name: str) -> int:
    code = _ELEM.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: expected float32, bfloat16 or float16, got {t.dtype}")
    return code


def _lists(grads: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]]):
    """Tables and element types of a step's gradients and of where they go (the same, in place); None where the list is empty."""
    if outs is not None and len(outs) != len(grads):
        raise ValueError("grads and outs differ in length")
    if not len(grads):
        return None
    g, gt = _Table(grads, grads[0].dtype), _elem(grads[0], "grads")
    if outs is None:
        return g, g, gt, gt
    o, ot = _Table(outs, outs[0].dtype), _elem(outs[0], "outs")
    if g.sizes != o.sizes:
        raise ValueError("grads[t] and outs[t] differ in size")
    return g, o, gt, ot


def ld_grad_norm(grads: Sequence[torch.Tensor], sumsq: Optional[torch.Tensor] = None, norm: Optional[torch.Tensor] = None,
                 accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(sumsq float64[1], norm float32[1]) over all elements of the tensors, which share one of the types float32,
    bfloat16 and float16. With `accumulate` the squares are added to what `sumsq` holds."""
    lib = load()
    if accumulate and sumsq is None:
        raise ValueError("accumulate needs the sumsq to add to")
    got = _lists(grads, None)
    dev = grads[0].device if got else sumsq.device if sumsq is not None else torch.device("cuda", torch.cuda.current_device())
    if sumsq is None:
        sumsq = _output(torch.float64, dev, stream, 1)
    if norm is None:
        norm = _output(torch.float32, dev, stream, 1)
    _one_device(sumsq, (norm, workspace), *(got[:1] if got else ()))
    gp, sizes, gt = (got[0].checked("grads"), got[0].sizes, got[2]) if got else (None, None, 0)
    if sumsq.numel() < 1 or norm.numel() < 1:
        raise ValueError("sumsq and norm need an element each")
    if workspace is None:
        workspace = _scratch(lib.ld_grad_norm_workspace(len(grads)), dev, stream)
    st = lib.ld_grad_norm(gp, sizes, len(grads), gt, int(accumulate), _dev(sumsq, torch.float64, "sumsq"),
                          _dev(norm, torch.float32, "norm"), _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
                          _stream(stream))
    _check("ld_grad_norm", st)
    return sumsq, norm


def ld_clip_grads(grads: Sequence[torch.Tensor], sumsq: torch.Tensor, max_norm: float,
                  outs: Optional[Sequence[torch.Tensor]] = None, stream=None) -> None:
    """Scales the tensors by max_norm / sqrt(sumsq) where that root is larger than max_norm (by the quotient itself:
    torch.nn.utils.clip_grad_norm_ adds 1e-6 to the norm and so scales a little further): in place, or into
    `outs` (of one type, which may be another; copied unscaled where the root is not larger, or not finite)."""
    got = _lists(grads, outs)
    if sumsq.numel() < 1:
        raise ValueError("sumsq needs an element")
    if got is None:
        return
    g, o, gt, ot = got
    _one_device(sumsq, (), g, o)
    st = load().ld_clip_grads(g.checked("grads"), o.checked("outs"), g.sizes, len(grads), gt, ot,
                              _dev(sumsq, torch.float64, "sumsq"), max_norm, _stream(stream))
    _check("ld_clip_grads", st)


def ld_clip_grad_norm(grads: Sequence[torch.Tensor], max_norm: float, outs: Optional[Sequence[torch.Tensor]] = None,
                      norm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """ld_grad_norm and ld_clip_grads in one call. Returns the norm before clipping, a float32[1] on the device. A step whose
    sum of squares is not finite (an infinity or NaN among the gradients) is left unscaled, and the norm tells the caller. The sum
    is 64 bits wide: finite gradients whose norm is only too large for 32 bits are clipped, though the norm reads infinite."""
    lib = load()
    got = _lists(grads, outs)
    dev = grads[0].device if got else norm.device if norm is not None else torch.device("cuda", torch.cuda.current_device())
    if norm is None:
        norm = _output(torch.float32, dev, stream, 1)
    _one_device(norm, (workspace,), *(got[:2] if got else ()))
    gp, op, sizes, gt, ot = (got[0].checked("grads"), got[1].checked("outs"), got[0].sizes, got[2], got[3]) if got else (None, None, None, 0, 0)
    if norm.numel() < 1:
        raise ValueError("norm needs an element")
    if workspace is None and (need := lib.ld_clip_grad_norm_workspace(len(grads), sizes)) > 0:
        workspace = _scratch(need, dev, stream)
    st = lib.ld_clip_grad_norm(gp, op, sizes, len(grads), gt, ot, max_norm, _dev(norm, torch.float32, "norm"),
                               _dev(workspace, torch.uint8, "workspace"), workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("ld_clip_grad_norm", st)
    return norm


def _rows(t: torch.Tensor, name: str, dims: Optional[int] = 2, written: bool = False) -> Tuple[int, int, int]:
    """Address, rows and row stride of a tensor on the GPU, taken as rows of its last dimension: one that is contiguous (of any
    number of dimensions with dims = None), or of two dimensions with rows that are, and that do not overlap where they are written."""
    shape = t.shape
    if not t.is_cuda or not shape or (dims is not None and len(shape) != dims):
        raise TypeError(f"{name}: expected a{' 2-D' if dims == 2 else ''} tensor on the GPU")
    width = shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), shape[0] if len(shape) == 2 else math.prod(shape[:-1]), width
    if len(shape) != 2 or (width > 1 and t.stride(1) != 1):
        raise TypeError(f"{name}: expected contiguous rows")
    stride = t.stride(0)
    if written and shape[0] > 1 and stride < width:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), shape[0], stride


def _ids(t: torch.Tensor, name: str) -> int:
    code = _ID.get(t.dtype)
    if code is None or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name}: expected a contiguous int32 or int64 tensor on the GPU")
    return code


def ld_embed_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, pos_table: Optional[torch.Tensor] = None,
                    positions: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                    out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """scale * table[ids] (+ pos_table[positions]) in `out` or a new tensor of shape ids.shape + (d,) and type
    `out_dtype` (the table's unless given). Rows outside their table count as zeros. The tables, and an `out` of two
    dimensions, may have any row stride; `out` overlaps none of the inputs. Autograd records nothing, whatever the table's
    requires_grad: the table's gradient is ld_embed_grad's to make."""
    if (pos_table is None) != (positions is None):
        raise ValueError("pos_table and positions go together")
    try:
        d, T = table.shape[-1], ids.numel()
        if pos_table is not None:
            if positions.numel() != T or positions.dtype != ids.dtype:
                raise ValueError("positions must be as many as ids, and of their type")
            if pos_table.shape[-1] != d or pos_table.dtype != table.dtype:
                raise ValueError("table and pos_table differ in width or type")
    except IndexError:
        raise TypeError("table, pos_table: expected a 2-D tensor on the GPU") from None
    _one_device(table, (ids, pos_table, positions, out))
    code, it = _elem(table, "table"), _ids(ids, "ids")
    tp, V, ts = _rows(table, "table")
    pp, P, ps, at = None, 0, 0, None
    if pos_table is not None:
        pp, P, ps = _rows(pos_table, "pos_table")
        _ids(positions, "positions")
        at = positions.data_ptr()
    if out is None:
        out = _output(out_dtype or table.dtype, table.device, stream, *ids.shape, d)
    elif out.numel() != T * d or out.shape[-1:] != (d,) or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError("out differs in shape or type from what the lookup gives")
    op, _, os_ = _rows(out, "out", None, written=True)
    st = load().ld_embed_lookup(tp, V, ts, pp, P, ps, code, ids.data_ptr(), at, it, T, d, scale, op, os_, _elem(out, "out"),
                                _stream(stream))
    _check("ld_embed_lookup", st)
    return out


def ld_embed_grad_workspace(T: int, V: int, d: int) -> int:
    return int(load().ld_embed_grad_workspace(int(T), int(V), int(d)))


def ld_embed_grad(dout: torch.Tensor, ids: torch.Tensor, grad: torch.Tensor, scale: float = 1.0, accumulate: bool = False,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """The gradient of ld_embed_lookup by its table from that of its output, `dout` (ids.shape + (d,), or [T, d] with any
    row stride): written to `grad` [V, d], or with `accumulate` added to it. Deterministic. A workspace that is not given is
    allocated for the call: ld_embed_grad_workspace bytes, for a small batch about as many as its `dout` has in 16 bits."""
    lib = load()
    try:
        T, d = ids.numel(), grad.shape[-1]
        if dout.shape[-1] != d or dout.numel() != T * d:
            raise ValueError("dout must have a row of grad's width for every id")
    except IndexError:
        raise TypeError("dout, grad: expected rows") from None
    _one_device(grad, (dout, ids, workspace))
    it, dt, gt = _ids(ids, "ids"), _elem(dout, "dout"), _elem(grad, "grad")
    dp, _, ds = _rows(dout, "dout", None)
    gp, V, gs = _rows(grad, "grad", written=True)
    if workspace is None and (need := lib.ld_embed_grad_workspace(T, V, d)) > 0:
        workspace = _scratch(need, grad.device, stream)
    st = lib.ld_embed_grad(dp, ds, dt, ids.data_ptr(), it, T, d, scale, gp, V, gs, gt, int(accumulate),
                           _dev(workspace, torch.uint8, "workspace"), workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("ld_embed_grad", st)


class TokenLogprob(NamedTuple):
    """What ld_token_logprob gives; None where it was not asked for."""
    logprob: Optional[torch.Tensor]      # float32, of the ids' shape
    entropy: Optional[torch.Tensor]      # float32, the same
    stats: torch.Tensor                  # float32 [..., 2]: the largest logit M, and log sum exp(scale (logit - M))
    top_ids: Optional[torch.Tensor]      # int32 [..., top]
    top_logprob: Optional[torch.Tensor]  # float32 [..., top]


def _on_device_of(stream, t: torch.Tensor) -> None:
    """A call runs on the device of its stream: the given one's, or the current device."""
    at = torch.cuda.current_device() if stream is None else stream.device_index
    if t.get_device() != at:
        raise ValueError(f"tensors lie on {t.device}, the call's stream belongs to cuda:{at}")


def _vocabulary_rows(logits: torch.Tensor, ids: Optional[torch.Tensor]) -> Tuple[Tuple[int, ...], int, int]:
    """(shape of the rows, their number, vocabulary)."""
    if logits.dim() < 1:
        raise TypeError("logits: expected rows over a vocabulary")
    rows = tuple(logits.shape[:-1])
    if ids is not None and tuple(ids.shape) != rows:
        raise ValueError("ids must name one token for every row of logits")
    return rows, math.prod(rows), logits.shape[-1]


def ld_token_logprob_workspace(T: int, V: int, top: int = 0) -> int:
    return int(load().ld_token_logprob_workspace(int(T), int(V), int(top)))


def ld_token_logprob(logits: torch.Tensor, ids: Optional[torch.Tensor] = None, scale: float = 1.0, entropy: bool = False, top: int = 0,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> TokenLogprob:
    """Log probabilities of the tokens `ids` under softmax(scale * logits) (0 where an id names no token, as -1 for padding), the
    rows' entropies, and their `top` most probable tokens (ties: the lower id first) with log probabilities. logits: [..., V], or
    [T, V] with any row stride; masked tokens are -inf. A row that is masked entirely has entropy 0 and log probabilities of -inf.
    Autograd records nothing: the gradient is ld_token_logprob_grad's, which takes the stats (and entropy) given here."""
    lib = load()
    rows, T, V = _vocabulary_rows(logits, ids)
    _one_device(logits, (ids, workspace))
    code, it = _elem(logits, "logits"), _ids(ids, "ids") if ids is not None else 0
    lp, _, stride = _rows(logits, "logits", None)
    _on_device_of(stream, logits)
    if not 0 <= top <= max(V, 0):
        raise ValueError("top: more alternatives than tokens")
    dev = logits.device
    # each of its own memory: what is kept for the gradient keeps no alternatives, and is not changed where another is (views of one
    # allocation would take 2 us less of the host)
    logprob = _output(torch.float32, dev, stream, rows) if ids is not None else None
    ent = _output(torch.float32, dev, stream, rows) if entropy else None
    stats = _output(torch.float32, dev, stream, *rows, 2)
    top_ids = _output(torch.int32, dev, stream, *rows, top) if top else None
    top_logprob = _output(torch.float32, dev, stream, *rows, top) if top else None
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    if workspace is None and (need := lib.ld_token_logprob_workspace(T, V, top)) > 0:
        workspace = _scratch(need, dev, stream)
    st = lib.ld_token_logprob(lp, T, V, stride, code, at(ids), it, scale, at(logprob), at(ent), stats.data_ptr(), top, at(top_ids),
                              at(top_logprob), _dev(workspace, torch.uint8, "workspace"), workspace.numel() if workspace is not None else 0,
                              _stream(stream))
    _check("ld_token_logprob", st)
    return TokenLogprob(logprob, ent, stats, top_ids, top_logprob)


def _per_row(t: torch.Tensor, rows: Tuple[int, ...], name: str) -> Tuple[int, int]:
    """Address and stride of a float32 for every row: contiguous, [T] with any stride, or one for all (expanded)."""
    if t.dtype != torch.float32 or not t.is_cuda:
        raise TypeError(f"{name}: expected a float32 tensor on the GPU")
    if tuple(t.shape) != rows:
        raise ValueError(f"{name}: expected one value for every row of logits")
    if t.is_contiguous():
        return t.data_ptr(), 1
    if not any(t.stride()):
        return t.data_ptr(), 0
    if t.dim() != 1:
        raise TypeError(f"{name}: expected a contiguous tensor, a strided one of one dimension, or one value expanded")
    return t.data_ptr(), t.stride(0)


def ld_token_logprob_grad(logits: torch.Tensor, stats: torch.Tensor, ids: Optional[torch.Tensor] = None,
                          d_logprob: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                          d_entropy: Optional[torch.Tensor] = None, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                          out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """The gradient of ld_token_logprob by its logits, from that of its log probabilities (with the ids) and that of its
    entropies (with them): in `out`, which may be the logits themselves, or a new tensor of the logits' shape and type `out_dtype`
    (theirs unless given). `stats` and `entropy` are what the call gave for the same logits and scale."""
    rows, T, V = _vocabulary_rows(logits, ids)
    if (ids is None) != (d_logprob is None):
        raise ValueError("ids and d_logprob go together")
    if (entropy is None) != (d_entropy is None):
        raise ValueError("entropy and d_entropy go together")
    if tuple(stats.shape) != rows + (2,):
        raise ValueError("stats must have two values for every row of logits")
    if entropy is not None and tuple(entropy.shape) != rows:
        raise ValueError("entropy must have one value for every row of logits")
    _one_device(logits, (stats, ids, d_logprob, entropy, d_entropy, out))
    code, it = _elem(logits, "logits"), _ids(ids, "ids") if ids is not None else 0
    lp, _, stride = _rows(logits, "logits", None)
    _on_device_of(stream, logits)
    gp, gs = _per_row(d_logprob, rows, "d_logprob") if d_logprob is not None else (None, 0)
    hp, hs = _per_row(d_entropy, rows, "d_entropy") if d_entropy is not None else (None, 0)
    if out is None:
        out = _output(out_dtype or logits.dtype, logits.device, stream, *logits.shape)
    elif out.shape != logits.shape or (out_dtype is not None and out.dtype != out_dtype):
        raise ValueError("out differs in shape or type from what the gradient has")
    op, _, os_ = _rows(out, "out", None, written=True)
    st = load().ld_token_logprob_grad(lp, T, V, stride, code, None if ids is None else ids.data_ptr(), it, scale,
                                      _dev(stats, torch.float32, "stats"), gp, gs, _dev(entropy, torch.float32, "entropy"), hp, hs, op, os_,
                                      _elem(out, "out"), _stream(stream))
    _check("ld_token_logprob_grad", st)
    return out


def _sides(mats: Sequence[torch.Tensor], name: str) -> Tuple[np.ndarray, np.ndarray]:
    """Rows and columns of a list of matrices."""
    shapes = [tuple(t.shape) for t in mats]
    if any(len(s) != 2 for s in shapes):
        raise TypeError(f"{name}: expected 2-D tensors")
    both = np.array(shapes, dtype=np.int64).reshape(-1, 2)
    return np.ascontiguousarray(both[:, 0]), np.ascontiguousarray(both[:, 1])


def _apart(name: str, written: Sequence[int], read: Sequence[int]) -> None:
    """Refuses tensors, by their addresses, of which one is written for two matrices, or written for one and read for another."""
    once = set(written)
    if len(once) < len(written) or not once.isdisjoint(read):
        raise ValueError(f"{name}: a tensor stands for two matrices")


def _coefficients(coeffs, steps: int) -> Optional[np.ndarray]:
    """Three a step: from None (the usual ones), three for all steps, or three for each."""
    if coeffs is None:
        return None
    c = np.asarray(coeffs, dtype=np.float32)
    if c.shape == (3,):
        c = np.broadcast_to(c, (max(int(steps), 0), 3))
    if c.shape != (steps, 3):
        raise ValueError("coeffs: three numbers, or three for every step")
    return np.ascontiguousarray(c)


def ld_orthogonalize_workspace(shapes: Sequence[Tuple[int, int]]) -> int:
    both = np.array([tuple(s) for s in shapes], dtype=np.int64).reshape(-1, 2)
    rows, cols = np.ascontiguousarray(both[:, 0]), np.ascontiguousarray(both[:, 1])
    return int(load().ld_orthogonalize_workspace(_hp(rows), _hp(cols), len(both)))


def ld_orthogonalize(mats: Sequence[torch.Tensor], outs: Optional[Sequence[torch.Tensor]] = None, steps: int = 5, coeffs=None,
                     eps: float = 1e-7, out_dtype: Optional[torch.dtype] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> List[torch.Tensor]:
    """Every matrix's nearest orthogonal one, about: `steps` Newton-Schulz steps of X <- (a I + b X X^T + c (X X^T)^2) X from
    X = U / (|U|_F + eps), about as precise as products in float32. Into `outs` (which may be the matrices themselves) or new tensors
    of type `out_dtype` (theirs unless given). Matrices of one call share a type, their shapes are any, and rows may have any stride.
    A matrix's result does not depend on the others of the call. `coeffs`: (a, b, c), or three for every step; those that
    let singular values grow too far are refused."""
    lib, n = load(), len(mats)
    if outs is not None and len(outs) != n:
        raise ValueError("mats and outs differ in length")
    if not n:
        return []
    rows, cols = _sides(mats, "mats")
    code, first = _elem(mats[0], "mats"), mats[0]
    if any(t.dtype != first.dtype for t in mats):
        raise TypeError("mats: expected tensors of one type")
    coeff = _coefficients(coeffs, steps)
    _one_device(first, (workspace, *mats[1:], *(outs or ())))
    sp, ss = np.empty(n, np.uint64), np.empty(n, np.int64)
    for i, t in enumerate(mats):
        sp[i], _, ss[i] = _rows(t, "mats")
    _on_device_of(stream, first)
    if outs is None:
        outs = [_output(out_dtype or first.dtype, first.device, stream, *t.shape) for t in mats]
    elif any(a.shape != b.shape for a, b in zip(mats, outs)) or any(o.dtype != (out_dtype or outs[0].dtype) for o in outs):
        raise ValueError("outs differ in shape from mats, or in type from one another or from out_dtype")
    dp, ds = np.empty(n, np.uint64), np.empty(n, np.int64)
    for i, t in enumerate(outs):
        dp[i], _, ds[i] = _rows(t, "outs", written=True)
        if dp[i] == sp[i] and t.numel() and (t.dtype != first.dtype or ds[i] != ss[i]):
            raise ValueError("outs: in place a matrix keeps its type and stride")
    kept = [i for i, t in enumerate(mats) if t.numel()]
    _apart("outs", [int(dp[i]) for i in kept], [int(sp[i]) for i in kept if sp[i] != dp[i]])
    if workspace is None and (need := lib.ld_orthogonalize_workspace(_hp(rows), _hp(cols), n)) > 0:
        workspace = _scratch(need, first.device, stream)
    st = lib.ld_orthogonalize(_hp(sp), _hp(ss), _hp(dp), _hp(ds), _hp(rows), _hp(cols), n, code, _elem(outs[0], "outs"), int(steps),
                              None if coeff is None else _hp(coeff), eps, _dev(workspace, torch.uint8, "workspace"),
                              workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("ld_orthogonalize", st)
    return list(outs)


def ld_merge_dense_muon_workspace(shapes: Sequence[Tuple[int, int]], W: int = 1) -> int:
    both = np.array([tuple(s) for s in shapes], dtype=np.int64).reshape(-1, 2)
    rows, cols = np.ascontiguousarray(both[:, 0]), np.ascontiguousarray(both[:, 1])
    return int(load().ld_merge_dense_muon_workspace(_hp(rows), _hp(cols), len(both), int(W)))


def ld_merge_dense_muon(ws: Sequence[torch.Tensor], ms: Sequence[torch.Tensor], grads: Sequence[Sequence[torch.Tensor]], lr: float,
                        momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, scale=None, steps: int = 5,
                        coeffs=None, eps: float = 1e-7, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Replays dense gradients, grads[t][i] of matrix i, as steps of the optimizer that orthogonalises its updates, onto the
    weights ws and momenta ms (float32), in place; with one t it is a training step. Per step: m = momentum * m + g, u = g + momentum * m
    with nesterov, else m, w = (1 - lr * weight_decay) * w - lr * scale[i] * orthogonalize(u). A trainer that keeps
    momentum * m + (1 - momentum) * g has (1 - momentum) times this m, and the same updates up to eps. scale: one number, one for every
    matrix, or None: sqrt(max(1, rows / cols)). Gradients share one of the types float32, bfloat16 and float16. Any cut of the
    gradients into calls gives the same bits."""
    lib, n, W = load(), len(ws), len(grads)
    if len(ms) != n or any(len(g) != n for g in grads):
        raise ValueError("ws, ms and every step's grads differ in length")
    if not n:
        return
    rows, cols = _sides(ws, "ws")
    shapes = [t.shape for t in ws]
    if any(m.shape != s for m, s in zip(ms, shapes)) or any(g.shape != s for step in grads for g, s in zip(step, shapes)):
        raise ValueError("a weight, its momentum and its gradients differ in shape")
    flat = [g for step in grads for g in step]
    dtype = flat[0].dtype if flat else torch.float32
    code = _ELEM.get(dtype)
    if code is None:
        raise TypeError(f"grads: expected float32, bfloat16 or float16, got {dtype}")
    coeff = _coefficients(coeffs, steps)
    w, m, g = _Table(ws, torch.float32), _Table(ms, torch.float32), _Table(flat, dtype)
    _one_device(ws[0], (workspace,), w, m, g)
    wp, mp, gp = w.checked("ws"), m.checked("ms"), g.checked("grads")
    _on_device_of(stream, ws[0])
    kept = [i for i, k in enumerate(w.numel().tolist()) if k]
    at = [np.frombuffer(p, np.uint64).reshape(-1, n)[:, kept].ravel().tolist() for p in (wp, mp, gp)]
    _apart("ws, ms", at[0] + at[1], at[2])
    factor = None
    if scale is not None:
        factor = np.ascontiguousarray(np.broadcast_to(np.asarray(scale, dtype=np.float32), (n,)))
    if workspace is None and (need := lib.ld_merge_dense_muon_workspace(_hp(rows), _hp(cols), n, W)) > 0:
        workspace = _scratch(need, ws[0].device, stream)
    st = lib.ld_merge_dense_muon(wp, mp, gp, _hp(rows), _hp(cols), n, W, code, lr, momentum, int(nesterov), weight_decay,
                                 None if factor is None else _hp(factor), int(steps), None if coeff is None else _hp(coeff), eps,
                                 _dev(workspace, torch.uint8, "workspace"), workspace.numel() if workspace is not None else 0, _stream(stream))
    _check("ld_merge_dense_muon", st)


class ConfigParams(ctypes.Structure):
    """ld_config_params of lowdiff.h (Sec. V-C): N, T, M, tau, R_F, C_F."""
    _fields_ = [(k, ctypes.c_double) for k in ("N", "T", "M", "tau", "R_F", "C_F")]


def ld_config_wasted_time(p: ConfigParams, f: float, b: float, R_B: float, C_B: float) -> float:
    return float(load().ld_config_wasted_time(ctypes.byref(p), f, b, R_B, C_B))


def ld_config_critical_interval(p: ConfigParams, b: float, R_B: float, C_B: float) -> float:
    return float(load().ld_config_critical_interval(ctypes.byref(p), b, R_B, C_B))


def ld_config_select(p: ConfigParams, f: Sequence[int], b: Sequence[int], R_B: Sequence[float],
                     C_B: Sequence[float]) -> Tuple[int, np.ndarray]:
    """Index of the candidate (f[i], b[i]) with the smallest wasted time, and every T_w."""
    fa, ba = _host(f, np.int32), _host(b, np.int32)
    ra, ca = _host(R_B, np.float64), _host(C_B, np.float64)
    if not (len(fa) == len(ba) == len(ra) == len(ca)):
        raise ValueError("candidate arrays differ in length")
    out = np.empty(len(fa), np.float64)
    i = load().ld_config_select(ctypes.byref(p), len(fa), _hp(fa), _hp(ba), _hp(ra), _hp(ca), _hp(out))
    return int(i), out
