"""Thin Python binding over the C ABI (include/augtree.h).

Argument marshalling only: every step of the computation runs in the HIP
kernels of libaugtree.so. torch provides device memory (outputs and
workspace are allocated with torch when the caller passes none) and the
current HIP stream. Function names and argument order follow the C entry
points without the ``augtree_`` prefix.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence

import numpy as np
import torch
from torch.autograd import forward_ad

from . import _lib
from ._lib import (REPLAY_FUSED, REPLAY_SPLIT, REPLAY_AUTO, OP_PREFILL_FWD, OP_REPLAY_FWD,  # noqa: F401
                   OP_PREFILL_BWD, OP_REPLAY_BWD, OP_TREE_FWD, OP_TREE_BWD, ACT_NONE, ACT_SILU)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _need(t: torch.Tensor, name: str, dtype, shape):
    if t.dtype != dtype:
        raise TypeError(f"{name}: dtype {t.dtype}, expected {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a device tensor")


def _offsets(cu) -> np.ndarray:
    """A batch's own copy: a caller may refill its arrays for the next batch before the backward of this one reads them."""
    a = np.array(cu, dtype=np.int32, order="C")
    a.flags.writeable = False
    return a


class GroupBatch:
    """A batch of replay trees (struct augtree_groups) with its host offsets, which are copied and stay as they are."""

    def __init__(self, cu_prompt, cu_branch, cu_resp, num_q_heads: int, num_kv_heads: int, head_dim: int,
                 softmax_scale: Optional[float] = None):
        self.cu_prompt, self.cu_branch, self.cu_resp = _offsets(cu_prompt), _offsets(cu_branch), _offsets(cu_resp)
        self.num_groups = len(self.cu_prompt) - 1
        self.num_branches = len(self.cu_resp) - 1
        self.hq, self.hkv, self.d = int(num_q_heads), int(num_kv_heads), int(head_dim)
        self.scale = float(softmax_scale if softmax_scale is not None else 1.0 / math.sqrt(head_dim))
        self.tp = int(self.cu_prompt[-1])
        self.tr = int(self.cu_resp[-1])
        i32p = ctypes.POINTER(ctypes.c_int32)
        self.struct = _lib.Groups(self.num_groups, self.num_branches, self.hq, self.hkv, self.d, self.scale,
                                  self.cu_prompt.ctypes.data_as(i32p), self.cu_branch.ctypes.data_as(i32p),
                                  self.cu_resp.ctypes.data_as(i32p))

    @classmethod
    def from_shape(cls, shape) -> "GroupBatch":
        return cls(shape.cu_prompt, shape.cu_branch, shape.cu_resp, shape.num_q_heads, shape.num_kv_heads,
                   shape.head_dim, shape.scale)

    @property
    def ref(self):
        return ctypes.byref(self.struct)

    def workspace_size(self, op: int, arg: int = 0) -> int:
        lib = _lib.load()
        n = lib.augtree_workspace_size(self.ref, op, arg)
        if n == 0:
            raise _lib.AugtreeError(_lib.AUGTREE_ERR_INVALID_ARGUMENT, "workspace_size",
                                    lib.augtree_last_error().decode())
        return int(n)

    def workspace(self, op: int, arg: int = 0, device=None) -> torch.Tensor:
        return torch.empty(self.workspace_size(op, arg), dtype=torch.uint8, device=device or "cuda")


def _ws(b: GroupBatch, ws, op, arg, device):
    if ws is None:
        ws = b.workspace(op, arg, device)
    return ws, ctypes.c_size_t(ws.numel())


def prefill_fwd(b: GroupBatch, q_p, k_p, v_p, o_p=None, lse_p=None, ws=None, stream=None):
    _need(q_p, "q_p", torch.bfloat16, (b.tp, b.hq, b.d))
    _need(k_p, "k_p", torch.bfloat16, (b.tp, b.hkv, b.d))
    _need(v_p, "v_p", torch.bfloat16, (b.tp, b.hkv, b.d))
    o_p = torch.empty_like(q_p) if o_p is None else o_p
    lse_p = torch.empty((b.hq, b.tp), dtype=torch.float32, device=q_p.device) if lse_p is None else lse_p
    _need(o_p, "o_p", torch.bfloat16, q_p.shape)
    _need(lse_p, "lse_p", torch.float32, (b.hq, b.tp))
    ws, nws = _ws(b, ws, OP_PREFILL_FWD, 0, q_p.device)
    _lib.check(_lib.load().augtree_prefill_fwd(b.ref, _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(o_p), _ptr(lse_p),
                                               _ptr(ws), nws, _stream(stream)), "prefill_fwd")
    return o_p, lse_p


def replay_fwd(b: GroupBatch, q_r, k_r, v_r, k_p, v_p, mode: int = REPLAY_FUSED, o_r=None, lse_r=None,
               o_part=None, lse_part=None, ws=None, stream=None):
    _need(q_r, "q_r", torch.bfloat16, (b.tr, b.hq, b.d))
    _need(k_r, "k_r", torch.bfloat16, (b.tr, b.hkv, b.d))
    _need(v_r, "v_r", torch.bfloat16, (b.tr, b.hkv, b.d))
    _need(k_p, "k_p", torch.bfloat16, (b.tp, b.hkv, b.d))
    _need(v_p, "v_p", torch.bfloat16, (b.tp, b.hkv, b.d))
    dev = q_r.device
    o_r = torch.empty_like(q_r) if o_r is None else o_r
    lse_r = torch.empty((b.hq, b.tr), dtype=torch.float32, device=dev) if lse_r is None else lse_r
    if mode != REPLAY_FUSED:
        o_part = torch.empty((2, b.tr, b.hq, b.d), dtype=torch.float32, device=dev) if o_part is None else o_part
        lse_part = torch.empty((2, b.hq, b.tr), dtype=torch.float32, device=dev) if lse_part is None else lse_part
    ws, nws = _ws(b, ws, OP_REPLAY_FWD, mode, dev)
    _lib.check(_lib.load().augtree_replay_fwd(b.ref, mode, _ptr(q_r), _ptr(k_r), _ptr(v_r), _ptr(k_p), _ptr(v_p),
                                              _ptr(o_r), _ptr(lse_r), _ptr(o_part), _ptr(lse_part), _ptr(ws), nws,
                                              _stream(stream)), "replay_fwd")
    return o_r, lse_r, o_part, lse_part


def replay_split_groups(b: GroupBatch) -> np.ndarray:
    """Per group, 1 if AUGTREE_REPLAY_AUTO runs it SPLIT, 0 if FUSED."""
    out = np.zeros(b.num_groups, dtype=np.int32)
    _lib.check(_lib.load().augtree_replay_split_groups(b.ref, out.ctypes.data_as(ctypes.c_void_p)),
               "replay_split_groups")
    return out


def set_tree_chunk_blocks(blocks: int) -> None:
    """Most query blocks (64 rows x one query head) a prompt-key tile of the
    tree backward sweeps over a group's branch rows before the sweep is cut
    into chunks (0 restores the default). Process-wide; workspaces sized
    afterwards follow it."""
    _lib.check(_lib.load().augtree_set_tree_chunk_blocks(int(blocks)), "set_tree_chunk_blocks")


def tree_chunk_blocks() -> int:
    return int(_lib.load().augtree_tree_chunk_blocks())


def lse_merge(o_parts, lse_parts, o=None, o_f32=None, lse=None, want_bf16=True, stream=None):
    n, rows, heads, d = o_parts.shape
    _need(o_parts, "o_parts", torch.float32, (n, rows, heads, d))
    _need(lse_parts, "lse_parts", torch.float32, (n, heads, rows))
    dev = o_parts.device
    if o is None and o_f32 is None:
        if want_bf16:
            o = torch.empty((rows, heads, d), dtype=torch.bfloat16, device=dev)
        else:
            o_f32 = torch.empty((rows, heads, d), dtype=torch.float32, device=dev)
    lse = torch.empty((heads, rows), dtype=torch.float32, device=dev) if lse is None else lse
    _lib.check(_lib.load().augtree_lse_merge(rows, heads, d, n, _ptr(o_parts), _ptr(lse_parts), _ptr(o),
                                             _ptr(o_f32), _ptr(lse), _stream(stream)), "lse_merge")
    return o, o_f32, lse


def replay_bwd(b: GroupBatch, q_r, k_r, v_r, k_p, v_p, o_r, lse_r, do_r, n_seed: int = 1, dq_r=None, dk_r=None,
               dv_r=None, dkv_p_seed=None, ws=None, stream=None):
    for t, nm, h in ((q_r, "q_r", b.hq), (o_r, "o_r", b.hq), (do_r, "do_r", b.hq), (k_r, "k_r", b.hkv),
                     (v_r, "v_r", b.hkv)):
        _need(t, nm, torch.bfloat16, (b.tr, h, b.d))
    _need(k_p, "k_p", torch.bfloat16, (b.tp, b.hkv, b.d))
    _need(v_p, "v_p", torch.bfloat16, (b.tp, b.hkv, b.d))
    _need(lse_r, "lse_r", torch.float32, (b.hq, b.tr))
    dev = q_r.device
    dq_r = torch.empty_like(q_r) if dq_r is None else dq_r
    dk_r = torch.empty_like(k_r) if dk_r is None else dk_r
    dv_r = torch.empty_like(v_r) if dv_r is None else dv_r
    if dkv_p_seed is None:
        dkv_p_seed = torch.empty((n_seed, 2, b.tp, b.hkv, b.d), dtype=torch.float32, device=dev)
    _need(dkv_p_seed, "dkv_p_seed", torch.float32, (n_seed, 2, b.tp, b.hkv, b.d))
    ws, nws = _ws(b, ws, OP_REPLAY_BWD, n_seed, dev)
    _lib.check(_lib.load().augtree_replay_bwd(b.ref, _ptr(q_r), _ptr(k_r), _ptr(v_r), _ptr(k_p), _ptr(v_p),
                                              _ptr(o_r), _ptr(lse_r), _ptr(do_r), _ptr(dq_r), _ptr(dk_r),
                                              _ptr(dv_r), n_seed, _ptr(dkv_p_seed), _ptr(ws), nws,
                                              _stream(stream)), "replay_bwd")
    return dq_r, dk_r, dv_r, dkv_p_seed


def prefill_bwd(b: GroupBatch, q_p, k_p, v_p, o_p, lse_p, do_p, dq_p=None, dq_p_f32=None, dkv_p_self=None,
                want_bf16=True, ws=None, stream=None):
    for t, nm, h in ((q_p, "q_p", b.hq), (o_p, "o_p", b.hq), (do_p, "do_p", b.hq), (k_p, "k_p", b.hkv),
                     (v_p, "v_p", b.hkv)):
        _need(t, nm, torch.bfloat16, (b.tp, h, b.d))
    _need(lse_p, "lse_p", torch.float32, (b.hq, b.tp))
    dev = q_p.device
    if dq_p is None and dq_p_f32 is None:
        if want_bf16:
            dq_p = torch.empty_like(q_p)
        else:
            dq_p_f32 = torch.empty(q_p.shape, dtype=torch.float32, device=dev)
    if dkv_p_self is None:
        dkv_p_self = torch.empty((2, b.tp, b.hkv, b.d), dtype=torch.float32, device=dev)
    _need(dkv_p_self, "dkv_p_self", torch.float32, (2, b.tp, b.hkv, b.d))
    ws, nws = _ws(b, ws, OP_PREFILL_BWD, 0, dev)
    _lib.check(_lib.load().augtree_prefill_bwd(b.ref, _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(o_p), _ptr(lse_p),
                                               _ptr(do_p), _ptr(dq_p), _ptr(dq_p_f32), _ptr(dkv_p_self), _ptr(ws),
                                               nws, _stream(stream)), "prefill_bwd")
    return dq_p, dq_p_f32, dkv_p_self


def prompt_grad_reduce(parts, self_part=None, row_map=None, rows: Optional[int] = None, out=None, out_f32=None,
                       want_bf16=True, shared_slab: bool = False, n_parts: Optional[int] = None, stream=None):
    """Eq. 2 sum. ``parts`` is [n_parts, n_tensors, part_rows, heads, d] fp32
    (one slab per term), or, with ``shared_slab=True``, a single slab
    [n_tensors, part_rows, heads, d] that every one of the ``n_parts`` terms
    reads through ``row_map`` [n_parts, rows] (int32, -1 = no row).
    Returns (out bf16 [n_tensors, rows, heads, d] or None, out_f32 or None)."""
    if shared_slab:
        n_tensors, part_rows, heads, d = parts.shape
        if row_map is None or n_parts is None:
            raise ValueError("shared_slab needs row_map and n_parts")
        part_stride = 0
    else:
        n_parts, n_tensors, part_rows, heads, d = parts.shape
        part_stride = n_tensors * part_rows * heads * d
    _need(parts, "parts", torch.float32, parts.shape)
    rows = part_rows if rows is None else int(rows)
    if self_part is not None:
        _need(self_part, "self", torch.float32, (n_tensors, rows, heads, d))
    if row_map is not None:
        _need(row_map, "row_map", torch.int32, (n_parts, rows))
    dev = parts.device
    if out is None and out_f32 is None:
        if want_bf16:
            out = torch.empty((n_tensors, rows, heads, d), dtype=torch.bfloat16, device=dev)
        else:
            out_f32 = torch.empty((n_tensors, rows, heads, d), dtype=torch.float32, device=dev)
    _lib.check(_lib.load().augtree_prompt_grad_reduce(n_tensors, rows, heads, d, _ptr(self_part), n_parts, part_rows,
                                                      part_stride, _ptr(parts), _ptr(row_map), _ptr(out),
                                                      _ptr(out_f32), _stream(stream)), "prompt_grad_reduce")
    return out, out_f32


def tree_fwd(b: GroupBatch, q_p, k_p, v_p, q_r, k_r, v_r, mode: int = REPLAY_FUSED, o_p=None, lse_p=None, o_r=None,
             lse_r=None, o_part=None, lse_part=None, ws=None, stream=None):
    """Prefill + replay forward of every tree in one call (augtree_tree_fwd).
    Returns (o_p, lse_p, o_r, lse_r, o_part, lse_part)."""
    for t, nm, rows, h in ((q_p, "q_p", b.tp, b.hq), (k_p, "k_p", b.tp, b.hkv), (v_p, "v_p", b.tp, b.hkv),
                           (q_r, "q_r", b.tr, b.hq), (k_r, "k_r", b.tr, b.hkv), (v_r, "v_r", b.tr, b.hkv)):
        _need(t, nm, torch.bfloat16, (rows, h, b.d))
    dev = q_p.device
    o_p = torch.empty_like(q_p) if o_p is None else o_p
    o_r = torch.empty_like(q_r) if o_r is None else o_r
    lse_p = torch.empty((b.hq, b.tp), dtype=torch.float32, device=dev) if lse_p is None else lse_p
    lse_r = torch.empty((b.hq, b.tr), dtype=torch.float32, device=dev) if lse_r is None else lse_r
    _need(o_p, "o_p", torch.bfloat16, q_p.shape)
    _need(o_r, "o_r", torch.bfloat16, q_r.shape)
    _need(lse_p, "lse_p", torch.float32, (b.hq, b.tp))
    _need(lse_r, "lse_r", torch.float32, (b.hq, b.tr))
    if mode != REPLAY_FUSED:
        o_part = torch.empty((2, b.tr, b.hq, b.d), dtype=torch.float32, device=dev) if o_part is None else o_part
        lse_part = torch.empty((2, b.hq, b.tr), dtype=torch.float32, device=dev) if lse_part is None else lse_part
    ws, nws = _ws(b, ws, OP_TREE_FWD, mode, dev)
    _lib.check(_lib.load().augtree_tree_fwd(b.ref, mode, _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(q_r), _ptr(k_r),
                                            _ptr(v_r), _ptr(o_p), _ptr(lse_p), _ptr(o_r), _ptr(lse_r), _ptr(o_part),
                                            _ptr(lse_part), _ptr(ws), nws, _stream(stream)), "tree_fwd")
    return o_p, lse_p, o_r, lse_r, o_part, lse_part


def tree_bwd(b: GroupBatch, q_p, k_p, v_p, o_p, lse_p, do_p, q_r, k_r, v_r, o_r, lse_r, do_r, dq_p=None, dk_p=None,
             dv_p=None, dkv_p_f32=None, dq_r=None, dk_r=None, dv_r=None, want_f32=False, ws=None, stream=None):
    """Gradients of every tree in one call (augtree_tree_bwd): the Eq. 2 sum of
    the prompt-key gradient is formed in registers. Returns
    (dq_p, dk_p, dv_p, dq_r, dk_r, dv_r, dkv_p_f32 or None)."""
    for t, nm, rows, h in ((q_p, "q_p", b.tp, b.hq), (k_p, "k_p", b.tp, b.hkv), (v_p, "v_p", b.tp, b.hkv),
                           (o_p, "o_p", b.tp, b.hq), (do_p, "do_p", b.tp, b.hq),
                           (q_r, "q_r", b.tr, b.hq), (k_r, "k_r", b.tr, b.hkv), (v_r, "v_r", b.tr, b.hkv),
                           (o_r, "o_r", b.tr, b.hq), (do_r, "do_r", b.tr, b.hq)):
        _need(t, nm, torch.bfloat16, (rows, h, b.d))
    _need(lse_p, "lse_p", torch.float32, (b.hq, b.tp))
    _need(lse_r, "lse_r", torch.float32, (b.hq, b.tr))
    dev = q_p.device
    dq_p = torch.empty_like(q_p) if dq_p is None else dq_p
    dk_p = torch.empty_like(k_p) if dk_p is None else dk_p
    dv_p = torch.empty_like(v_p) if dv_p is None else dv_p
    dq_r = torch.empty_like(q_r) if dq_r is None else dq_r
    dk_r = torch.empty_like(k_r) if dk_r is None else dk_r
    dv_r = torch.empty_like(v_r) if dv_r is None else dv_r
    for t, nm, ref in ((dq_p, "dq_p", q_p), (dk_p, "dk_p", k_p), (dv_p, "dv_p", v_p), (dq_r, "dq_r", q_r),
                       (dk_r, "dk_r", k_r), (dv_r, "dv_r", v_r)):
        _need(t, nm, torch.bfloat16, ref.shape)
    if dkv_p_f32 is None and want_f32:
        dkv_p_f32 = torch.empty((2, b.tp, b.hkv, b.d), dtype=torch.float32, device=dev)
    if dkv_p_f32 is not None:
        _need(dkv_p_f32, "dkv_p_f32", torch.float32, (2, b.tp, b.hkv, b.d))
    ws, nws = _ws(b, ws, OP_TREE_BWD, 0, dev)
    _lib.check(_lib.load().augtree_tree_bwd(b.ref, _ptr(q_p), _ptr(k_p), _ptr(v_p), _ptr(o_p), _ptr(lse_p),
                                            _ptr(do_p), _ptr(q_r), _ptr(k_r), _ptr(v_r), _ptr(o_r), _ptr(lse_r),
                                            _ptr(do_r), _ptr(dq_p), _ptr(dk_p), _ptr(dv_p), _ptr(dkv_p_f32),
                                            _ptr(dq_r), _ptr(dk_r), _ptr(dv_r), _ptr(ws), nws, _stream(stream)),
               "tree_bwd")
    return dq_p, dk_p, dv_p, dq_r, dk_r, dv_r, dkv_p_f32


# ---------------------------------------------------------------------------- linear attention layer

# What torch.cuda.current_device() and current_stream().cuda_stream end in, without their 3 us (the tensors are on a GPU:
# torch.cuda is initialised).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)


class _On:
    """The device of a call's tensors made current, with the stream it runs on there. Every tensor has to be on that
    device (a stream given by the caller too)."""

    __slots__ = ("device", "stream", "guard")

    def __init__(self, tensors, stream=None):
        dev = None
        for name, t in tensors:
            if t is None:
                continue
            d = t.device
            if dev is None:
                if d.type != "cuda":
                    raise ValueError(f"{name} must be a GPU tensor (the op has no CPU path)")
                dev = d
            elif d != dev:
                raise ValueError(f"{name} is on {d}, other tensors on {dev}")
        if stream is not None and stream.device != dev:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {dev}")
        self.device, self.stream, self.guard = dev, stream, None

    def __enter__(self):
        if self.stream is not None:  # what is allocated inside belongs to that stream
            self.guard = torch.cuda.stream(self.stream)
        elif self.device.index != _current_device():
            self.guard = torch.cuda.device(self.device)
        if self.guard is not None:
            self.guard.__enter__()
        return _raw_stream(self.device.index)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _addr(t):
    return None if t is None else t.data_ptr()


def _want(t: torch.Tensor, name: str, dtype, shape):
    """_need for tensors that _On has seen, quick where there is nothing to say."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _need(t, name, dtype, shape)


def _tangent(tensors) -> bool:
    """Whether one of them is a dual tensor: forward-mode derivatives are taken of nothing here. (Outside a dual level,
    where the ops are called, that is one comparison.)"""
    return (getattr(forward_ad, "_current_level", 0) >= 0
            and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors))


def _decay(decay, heads: int) -> np.ndarray:
    """Host array [heads] of fp32 decays (a sequence, a numpy array or a CPU tensor; one number for all heads)."""
    if type(decay) is np.ndarray and decay.dtype == np.float32 and decay.shape == (heads,) and decay.flags.c_contiguous:
        return decay
    if isinstance(decay, torch.Tensor):
        if decay.device.type != "cpu":
            raise ValueError("decay must be on the host")
        if (decay.requires_grad and torch.is_grad_enabled()) or _tangent((decay,)):
            raise ValueError("decay is a constant of the layer: no gradient is formed for it")
        decay = decay.detach().numpy()
    a = np.asarray(decay, dtype=np.float32)
    a = np.ascontiguousarray(np.broadcast_to(a, (heads,)) if a.ndim == 0 else a)
    if a.shape != (heads,):
        raise ValueError(f"decay: shape {a.shape}, expected {(heads,)}")
    return a


def _out(t, name, dtype, shape, device):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _want(t, name, dtype, shape)
    return t


def _written(given):
    """Counts a call's writes to the caller's own tensors as torch's in-place operations count theirs, so that a backward
    which saved one of them notices."""
    given = [t for t in given if t is not None]
    if given:
        torch.autograd.graph.increment_version(given)


def _check_batch(b: GroupBatch):
    """The offsets' counts, which the library takes from the batch's struct."""
    if b.num_branches and len(b.cu_branch) != b.num_groups + 1:
        raise ValueError(f"cu_branch: {len(b.cu_branch)} offsets for {b.num_groups} prompts")


def linear_workspace_size(b: GroupBatch, backward: bool = False, from_fwd_ws: bool = False) -> int:
    """Bytes of workspace of linear_fwd, or of linear_bwd, which needs less where it is given the forward's."""
    lib = _lib.load()
    _check_batch(b)
    n = lib.augtree_linear_workspace_size(b.ref, 0 if not backward else 2 if from_fwd_ws else 1)
    if n == 0:
        raise _lib.AugtreeError(_lib.AUGTREE_ERR_INVALID_ARGUMENT, "linear_workspace_size",
                                lib.augtree_last_error().decode())
    return int(n)


def _want_ws(ws, name: str):
    if ws is not None and (ws.dtype is not torch.uint8 or not ws.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous uint8 tensor")


def _linear_ws(b, backward, ws, device, from_fwd_ws=False):
    if ws is None:
        ws = torch.empty(linear_workspace_size(b, backward, from_fwd_ws), dtype=torch.uint8, device=device)
    _want_ws(ws, "ws")
    return ws


def _linear_inputs(b: GroupBatch, named):
    _check_batch(b)
    for n, t in named:
        rows = b.tp if n.endswith("_p") else b.tr
        _want(t, n, torch.bfloat16, (rows, b.hkv if n[0] in "kv" else b.hq, b.d))


def linear_fwd(b: GroupBatch, decay, q_p, k_p, v_p, q_r, k_r, v_r, state=None, o_p=None, o_r=None, state_p=None,
               state_r=None, want_states: bool = False, ws=None, stream=None):
    """Linear attention of every tree (augtree_linear_fwd). `decay`: host values, one per KV head. A batch without
    branches (cu_branch all 0, cu_resp [0]) takes response tensors of no rows. Returns (o_p, o_r, state_p, state_r);
    the states are None unless asked for."""
    dec = _decay(decay, b.hkv)
    named = (("q_p", q_p), ("k_p", k_p), ("v_p", v_p), ("q_r", q_r), ("k_r", k_r), ("v_r", v_r))
    on = _On(named + (("state", state), ("o_p", o_p), ("o_r", o_r), ("state_p", state_p), ("state_r", state_r),
                      ("ws", ws)), stream)
    _linear_inputs(b, named)
    dev, f32, given = on.device, torch.float32, (o_p, o_r, state_p, state_r, ws)
    if state is not None:
        _want(state, "state", f32, (b.num_groups, b.hkv, b.d, b.d))
    with on as st:
        o_p = _out(o_p, "o_p", torch.bfloat16, q_p.shape, dev)
        o_r = _out(o_r, "o_r", torch.bfloat16, q_r.shape, dev)
        if want_states or state_p is not None:
            state_p = _out(state_p, "state_p", f32, (b.num_groups, b.hkv, b.d, b.d), dev)
        if want_states or state_r is not None:
            state_r = _out(state_r, "state_r", f32, (b.num_branches, b.hkv, b.d, b.d), dev)
        ws = _linear_ws(b, False, ws, dev)
        _lib.check(_lib.load().augtree_linear_fwd(
            b.ref, dec.ctypes.data, _addr(q_p), _addr(k_p), _addr(v_p), _addr(q_r), _addr(k_r), _addr(v_r), _addr(state),
            _addr(o_p), _addr(o_r), _addr(state_p), _addr(state_r) if b.num_branches else None, _addr(ws), ws.numel(),
            st), "linear_fwd")
    _written(given)
    return o_p, o_r, state_p, state_r


def linear_bwd(b: GroupBatch, decay, q_p, k_p, v_p, do_p, q_r, k_r, v_r, do_r, state=None, dq_p=None, dk_p=None,
               dv_p=None, dq_r=None, dk_r=None, dv_r=None, fwd_ws=None, ws=None, stream=None):
    """Gradients of linear_fwd's outputs (augtree_linear_bwd). `fwd_ws`: the workspace that linear_fwd was given for the
    same inputs, not written since (saves forming its states again; `state` is not read then). Returns
    (dq_p, dk_p, dv_p, dq_r, dk_r, dv_r)."""
    dec = _decay(decay, b.hkv)
    named = (("q_p", q_p), ("k_p", k_p), ("v_p", v_p), ("do_p", do_p), ("q_r", q_r), ("k_r", k_r), ("v_r", v_r),
             ("do_r", do_r))
    on = _On(named + (("state", state), ("dq_p", dq_p), ("dk_p", dk_p), ("dv_p", dv_p), ("dq_r", dq_r),
                      ("dk_r", dk_r), ("dv_r", dv_r), ("fwd_ws", fwd_ws), ("ws", ws)), stream)
    _linear_inputs(b, named)
    dev, given = on.device, (dq_p, dk_p, dv_p, dq_r, dk_r, dv_r, ws)
    _want_ws(fwd_ws, "fwd_ws")
    if state is not None:
        _want(state, "state", torch.float32, (b.num_groups, b.hkv, b.d, b.d))
    with on as st:
        outs = [_out(t, n, torch.bfloat16, like.shape, dev)
                for t, n, like in ((dq_p, "dq_p", q_p), (dk_p, "dk_p", k_p), (dv_p, "dv_p", v_p),
                                   (dq_r, "dq_r", q_r), (dk_r, "dk_r", k_r), (dv_r, "dv_r", v_r))]
        _linear_bwd(b, dec, (q_p, k_p, v_p, do_p, q_r, k_r, v_r, do_r, state, *outs), fwd_ws,
                    _linear_ws(b, True, ws, dev, fwd_ws is not None), st)
    _written(given)
    return tuple(outs)


def _linear_bwd(b: GroupBatch, dec, tensors, fwd_ws, ws, stream):
    """The call of linear_bwd behind its checks: inputs, state and outputs in the order of augtree_linear_bwd."""
    _lib.check(_lib.load().augtree_linear_bwd(b.ref, dec.ctypes.data, *(_addr(t) for t in tensors), _addr(fwd_ws),
                                              0 if fwd_ws is None else fwd_ws.numel(), _addr(ws), ws.numel(), stream),
               "linear_bwd")


def linear_step(q, k, v, decay, state, src=None, state_out=None, o=None, scale: Optional[float] = None, stream=None):
    """One token of linear attention for every row (augtree_linear_step): q [rows, Hq, d], k, v [rows, Hkv, d] bf16,
    state [n, Hkv, d, d] fp32. `src` [rows] int32 on the GPU names the state each row goes on from (the branches of a
    prompt share one; outside [0, n): from zero). Writes the new states to `state_out` (a new tensor if None; `state`
    itself only without src) and returns (o, state_out). Decode only: tensors that ask for a gradient are refused while
    gradients are enabled."""
    on = _On((("q", q), ("k", k), ("v", v), ("state", state), ("src", src), ("state_out", state_out), ("o", o)), stream)
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad or state.requires_grad or
                                    (state_out is not None and state_out.requires_grad) or
                                    (o is not None and o.requires_grad)):
        raise ValueError("linear_step forms no gradient: call it under torch.no_grad(), or with detached tensors")
    if _tangent((q, k, v, state, state_out, o)):
        raise ValueError("linear_step takes no dual tensors: a tangent would get lost")
    if q.dim() != 3 or k.dim() != 3 or state.dim() != 4:
        raise ValueError("q and k must be [rows, heads, head_dim], state [n, heads, head_dim, head_dim]")
    rows, hq, d = q.shape
    hkv, n = k.shape[1], state.shape[0]
    _want(q, "q", torch.bfloat16, (rows, hq, d))
    _want(k, "k", torch.bfloat16, (rows, hkv, d))
    _want(v, "v", torch.bfloat16, (rows, hkv, d))
    _want(state, "state", torch.float32, (n, hkv, d, d))
    if src is not None:
        _want(src, "src", torch.int32, (rows,))
    dec, given = _decay(decay, hkv), (state_out, o)
    with on as st:
        state_out = _out(state_out, "state_out", torch.float32, (rows, hkv, d, d), on.device)
        o = _out(o, "o", torch.bfloat16, q.shape, on.device)
        _lib.check(_lib.load().augtree_linear_step(
            rows, hq, hkv, d, 1.0 / math.sqrt(d) if scale is None else float(scale),
            dec.ctypes.data, _addr(q), _addr(k), _addr(v), n, _addr(state), _addr(src),
            _addr(state_out), _addr(o), st), "linear_step")
    _written(given)
    return o, state_out


def _norm_inputs(x, gate, weight, bias):
    if x.dim() != 3:
        raise ValueError("x must be [rows, heads, head_dim]")
    _want(x, "x", torch.bfloat16, x.shape)
    if gate is not None:
        _want(gate, "gate", torch.bfloat16, x.shape)
    for n, t in (("weight", weight), ("bias", bias)):
        if t is not None:
            _want(t, n, torch.float32, x.shape[1:])


def head_norm_fwd(x, weight=None, bias=None, gate=None, activation: int = ACT_NONE, eps: float = 1e-5, y=None,
                  stream=None):
    """Norm over each head with an activation or a gate (augtree_head_norm_fwd)."""
    on = _On((("x", x), ("weight", weight), ("bias", bias), ("gate", gate), ("y", y)), stream)
    _norm_inputs(x, gate, weight, bias)
    rows, heads, d = x.shape
    given = (y,)
    with on as st:
        y = _out(y, "y", torch.bfloat16, x.shape, on.device)
        _lib.check(_lib.load().augtree_head_norm_fwd(rows, heads, d, int(activation), float(eps), _addr(x), _addr(gate),
                                                     _addr(weight), _addr(bias), _addr(y), st), "head_norm_fwd")
    _written(given)
    return y


def head_norm_bwd(x, dy, weight=None, bias=None, gate=None, activation: int = ACT_NONE, eps: float = 1e-5, dx=None,
                  dgate=None, dweight=None, dbias=None, want_dweight: bool = False, want_dbias: bool = False, ws=None,
                  stream=None):
    """Its gradients (augtree_head_norm_bwd). Returns (dx, dgate, dweight, dbias); dgate is None without a gate, the
    last two unless asked for."""
    on = _On((("x", x), ("dy", dy), ("weight", weight), ("bias", bias), ("gate", gate), ("dx", dx), ("dgate", dgate),
              ("dweight", dweight), ("dbias", dbias), ("ws", ws)), stream)
    _norm_inputs(x, gate, weight, bias)
    _want(dy, "dy", torch.bfloat16, x.shape)
    rows, heads, d = x.shape
    dev, f32, given = on.device, torch.float32, (dx, dgate, dweight, dbias, ws)
    with on as st:
        dx = _out(dx, "dx", torch.bfloat16, x.shape, dev)
        if gate is not None:
            dgate = _out(dgate, "dgate", torch.bfloat16, x.shape, dev)
        if want_dweight or dweight is not None:
            dweight = _out(dweight, "dweight", f32, (heads, d), dev)
        if want_dbias or dbias is not None:
            dbias = _out(dbias, "dbias", f32, (heads, d), dev)
        _want_ws(ws, "ws")
        _head_norm_bwd(x, dy, weight, bias, gate, int(activation), float(eps), dx, dgate, dweight, dbias, ws, st)
    _written(given)
    return dx, dgate, dweight, dbias


def _head_norm_bwd(x, dy, weight, bias, gate, activation, eps, dx, dgate, dweight, dbias, ws, stream):
    """The call of head_norm_bwd behind its checks."""
    rows, heads, d = x.shape
    lib, n = _lib.load(), 0
    if dweight is not None or dbias is not None:
        if ws is None:
            ws = torch.empty(lib.augtree_head_norm_workspace_size(rows, heads, d), dtype=torch.uint8, device=x.device)
        n = ws.numel()
    _lib.check(lib.augtree_head_norm_bwd(rows, heads, d, activation, eps, _addr(x), _addr(gate), _addr(weight),
                                         _addr(bias), _addr(dy), _addr(dx), _addr(dgate), _addr(dweight), _addr(dbias),
                                         _addr(ws), n, stream), "head_norm_bwd")


# ---------------------------------------------------------------------------- paged KV cache

class PageTable:
    """The tables of a paged KV cache (struct augtree_pages), int32 tensors on one GPU that stay the caller's: `table`
    [seqs, max_pages], `length` [seqs] cached tokens, `parent` [seqs] (< 0, or no tensor: none), `free_pages` [pages] a
    ring of free pages, `free_state` [2] its first free entry and their number. One PageTable serves all layers of a
    model; the caches of a layer are tensors [pages, Hkv, page_size, d]. PageTable.empty makes an unused one. The tensors
    are written to, not exchanged for others."""

    __slots__ = ("device", "table", "length", "parent", "free_pages", "free_state", "num_seqs", "max_pages", "num_pages",
                 "page_size", "struct", "ref", "_sizes")

    def __setattr__(self, name, value):
        if hasattr(self, "_sizes"):  # the library has the tensors' addresses
            raise AttributeError(f"PageTable.{name} stays what it was made with: write into it")
        object.__setattr__(self, name, value)

    def __init__(self, table, length, parent, free_pages, free_state, page_size: int):
        on = _On((("table", table), ("length", length), ("parent", parent), ("free_pages", free_pages),
                  ("free_state", free_state)))
        if table.dim() != 2 or free_pages.dim() != 1:
            raise ValueError("table must be [seqs, max_pages], free_pages [pages]")
        seqs, i32 = table.shape[0], torch.int32
        _want(table, "table", i32, table.shape)
        _want(length, "length", i32, (seqs,))
        if parent is not None:
            _want(parent, "parent", i32, (seqs,))
        _want(free_pages, "free_pages", i32, free_pages.shape)
        _want(free_state, "free_state", i32, (2,))
        self.device = on.device
        self.table, self.length, self.parent = table, length, parent
        self.free_pages, self.free_state = free_pages, free_state
        self.num_seqs, self.max_pages, self.num_pages = seqs, table.shape[1], free_pages.shape[0]
        self.page_size = int(page_size)
        self.struct = _lib.Pages(seqs, self.max_pages, self.num_pages, self.page_size, _addr(table), _addr(length),
                                 _addr(parent), _addr(free_pages), _addr(free_state))
        self.ref = ctypes.byref(self.struct)
        self._sizes = {}

    def _plan_sizes(self, rows: int, hq: int, hkv: int):
        """Words of a plan, offsets of its fields, and a dict of the workspaces of its attention; kept for the last few
        sizes."""
        found = self._sizes.get((rows, hq, hkv))
        if found is None:
            lib = _lib.load()
            n = lib.augtree_page_plan_size(self.ref, rows, hq, hkv)
            if n == 0:
                raise _lib.AugtreeError(_lib.AUGTREE_ERR_INVALID_ARGUMENT, "page_plan_size",
                                        lib.augtree_last_error().decode())
            if len(self._sizes) >= 64:
                self._sizes.clear()
            at = tuple(lib.augtree_page_plan_offset(self.ref, rows, hq, hkv, f) for f in range(4))
            found = self._sizes[rows, hq, hkv] = n // 4, at, {}
        return found

    @classmethod
    def empty(cls, num_seqs: int, max_pages: int, num_pages: int, page_size: int, device="cuda") -> "PageTable":
        """Tables of `num_seqs` sequences without tokens or parents, all pages free."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.zeros(num_seqs, max_pages, **i32), torch.zeros(num_seqs, **i32),
                   torch.full((num_seqs,), -1, **i32), torch.arange(num_pages, **i32),
                   torch.tensor([0, num_pages], **i32), page_size)


class PagePlan:
    """A step's plan (page_plan): `cu_rows` [seqs + 1], `slots` and `positions` [rows] and `status` [1] are views of it
    on the GPU."""

    def __init__(self, pages: PageTable, rows: int, num_q_heads: int, num_kv_heads: int):
        self.pages, self.rows, self.hq, self.hkv = pages, int(rows), int(num_q_heads), int(num_kv_heads)
        self._words, self._at, self._ws_bytes = pages._plan_sizes(self.rows, self.hq, self.hkv)
        self.data = torch.empty(self._words, dtype=torch.int32, device=pages.device)

    def _field(self, field: int, count: int) -> torch.Tensor:
        return self.data[self._at[field]:self._at[field] + count]

    @property
    def status(self) -> torch.Tensor:
        return self._field(_lib.PLAN_STATUS, 1)

    @property
    def cu_rows(self) -> torch.Tensor:
        return self._field(_lib.PLAN_CU_ROWS, self.pages.num_seqs + 1)

    @property
    def slots(self) -> torch.Tensor:
        return self._field(_lib.PLAN_SLOTS, self.rows)

    @property
    def positions(self) -> torch.Tensor:
        return self._field(_lib.PLAN_POSITIONS, self.rows)

    def check(self) -> None:
        """Raises if the tables could not take the step (waits for the GPU, all of its streams)."""
        torch.cuda.synchronize(self.pages.device)
        bits = int(self.status)
        if bits:
            raise RuntimeError("page_plan: " + "; ".join(text for bit, text in PAGES_STATUS.items() if bits & bit))

    def workspace_size(self, head_dim: int) -> int:
        """Bytes of workspace of paged_fwd with this plan: room for the most partial results that any plan of its sizes
        can have (135 MB for one token at 32 / 8 heads, d = 128; 1.08 GB for 4096 branches). One serves all layers, one
        after the other."""
        n = self._ws_bytes.get(head_dim)
        if n is None:
            lib = _lib.load()
            n = int(lib.augtree_paged_workspace_size(self.pages.ref, self.rows, self.hq, self.hkv, head_dim))
            if n == 0:
                raise _lib.AugtreeError(_lib.AUGTREE_ERR_UNSUPPORTED, "paged_workspace_size",
                                        lib.augtree_last_error().decode())
            self._ws_bytes[head_dim] = n
        return n


PAGES_STATUS = {
    _lib.PAGES_SHORT: "fewer free pages than the new tokens need",
    _lib.PAGES_LONG: "a sequence outgrows its row of the table",
    _lib.PAGES_ROWS: "more new tokens than the plan has rows",
    _lib.PAGES_LENGTH: "a length or the free list's state is out of range",
    _lib.PAGES_PARENT: "a parent is no sequence, the sequence itself, has a parent or ends in this step",
    _lib.PAGES_PAGE: "a page of the new tokens is outside the pool",
}


def page_plan(pages: PageTable, new_rows, rows: int, num_q_heads: int, num_kv_heads: int, length_out=None,
              free_state_out=None, plan: Optional[PagePlan] = None, stream=None) -> PagePlan:
    """Plans a step of a paged cache (augtree_page_plan): `new_rows` [seqs] int32 on the GPU are the new tokens of every
    sequence (< 0: it has ended and gives its pages back), `rows` at least their sum. Takes pages from the ring into the
    tables, advances the lengths and the ring's state (in place, unless length_out and free_state_out are given) and
    returns the plan that cache_write and paged_fwd of all layers take; `plan`: one of an earlier step of the same sizes,
    written over. What does not fit leaves everything as it was: PagePlan.check tells."""
    on = _On((("table", pages.table), ("new_rows", new_rows), ("length_out", length_out),
              ("free_state_out", free_state_out)), stream)
    _want(new_rows, "new_rows", torch.int32, (pages.num_seqs,))
    length = pages.length if length_out is None else length_out
    state = pages.free_state if free_state_out is None else free_state_out
    _want(length, "length_out", torch.int32, (pages.num_seqs,))
    _want(state, "free_state_out", torch.int32, (2,))
    with on as st:
        if plan is None:
            plan = PagePlan(pages, rows, num_q_heads, num_kv_heads)
        elif plan.pages is not pages or (plan.rows, plan.hq, plan.hkv) != (rows, num_q_heads, num_kv_heads):
            raise ValueError("the plan was made for other tables, rows or heads")
        _lib.check(_lib.load().augtree_page_plan(pages.ref, _addr(new_rows), plan.rows, plan.hq, plan.hkv, _addr(length),
                                                 _addr(state), _addr(plan.data), 4 * plan.data.numel(), st), "page_plan")
    _written((pages.table, pages.free_pages, length, state, plan.data))
    return plan


def _no_grad(what: str, tensors):
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError(f"{what} forms no gradient: call it under torch.no_grad(), or with detached tensors")
    if _tangent(tensors):
        raise ValueError(f"{what} takes no dual tensors: a tangent would get lost")


def _cache(t, name: str, plan: PagePlan, d: int):
    """A cache's type and the bytes between its pages: [pages, Hkv, page_size, d], dense but for the first dimension."""
    pages = plan.pages
    if t.dtype is torch.bfloat16:
        kind, size = _lib.CACHE_BF16, 2
    elif t.dtype is torch.float8_e4m3fn:
        kind, size = _lib.CACHE_E4M3, 1
    else:
        raise TypeError(f"{name}: dtype {t.dtype}, expected torch.bfloat16 or torch.float8_e4m3fn")
    shape = (pages.num_pages, plan.hkv, pages.page_size, d)
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    if t.is_contiguous():
        return kind, plan.hkv * pages.page_size * d * size
    stride, page = t.stride(), pages.page_size * d
    if stride[3] != 1 or stride[2] != d or (stride[1] != page and plan.hkv > 1):
        raise ValueError(f"{name} must be contiguous but for its first dimension")
    return kind, (stride[0] if pages.num_pages > 1 else plan.hkv * page) * size


def _caches(k_cache, v_cache, k_scale, v_scale, plan: PagePlan, d: int):
    kind, k_stride = _cache(k_cache, "k_cache", plan, d)
    if v_cache.dtype is not k_cache.dtype:
        raise TypeError(f"k_cache is {k_cache.dtype}, v_cache {v_cache.dtype}")
    like_k = v_cache.shape == k_cache.shape and v_cache.stride() == k_cache.stride()
    v_stride = k_stride if like_k else _cache(v_cache, "v_cache", plan, d)[1]
    if kind == _lib.CACHE_BF16 and k_scale is None and v_scale is None:
        return kind, k_stride, v_stride
    for n, t in (("k_scale", k_scale), ("v_scale", v_scale)):
        if (t is not None) != (kind == _lib.CACHE_E4M3):
            raise ValueError(f"{n} goes with a cache in 8 bits" + (", which needs it" if t is None else ""))
        if t is not None:
            _want(t, n, torch.float32, (plan.hkv,))
    return kind, k_stride, v_stride


def cache_write(k, v, k_cache, v_cache, plan: PagePlan, k_scale=None, v_scale=None, stream=None) -> None:
    """Writes the keys and values of a step's new tokens, k, v [rows, Hkv, d] bf16, into their slots of the caches
    [pages, Hkv, page_size, d] (augtree_cache_write): bf16, or float8_e4m3fn holding value / scale with fp32 scales [Hkv]
    on the GPU. The caches may be views with any stride between pages (two halves of one tensor). Tensors that ask for a
    gradient, the scales among them, are refused while gradients are enabled, dual tensors always."""
    on = _On((("plan", plan.data), ("k", k), ("v", v), ("k_cache", k_cache), ("v_cache", v_cache), ("k_scale", k_scale),
              ("v_scale", v_scale)), stream)
    _no_grad("cache_write", (k, v, k_cache, v_cache, k_scale, v_scale))
    if k.dim() != 3:
        raise ValueError("k must be [rows, heads, head_dim]")
    d = k.shape[2]
    _want(k, "k", torch.bfloat16, (plan.rows, plan.hkv, d))
    _want(v, "v", torch.bfloat16, (plan.rows, plan.hkv, d))
    kind, k_stride, v_stride = _caches(k_cache, v_cache, k_scale, v_scale, plan, d)
    with on as st:
        _lib.check(_lib.load().augtree_cache_write(plan.pages.ref, _addr(plan.data), plan.rows, plan.hq, plan.hkv, d,
                                                   _addr(k), _addr(v), kind, _addr(k_cache), k_stride, _addr(v_cache),
                                                   v_stride, _addr(k_scale), _addr(v_scale), st), "cache_write")
    _written((k_cache, v_cache))


def paged_fwd(q, k_cache, v_cache, plan: PagePlan, k_scale=None, v_scale=None, o=None, lse=None,
              scale: Optional[float] = None, want_lse: bool = False, ws=None, stream=None):
    """Attention of a step's new tokens, q [rows, Hq, d] bf16, over the cached tokens of their sequences' parents and
    their own up to themselves (augtree_paged_fwd). Returns (o, lse): o like q, lse [Hq, rows] fp32 or None unless asked
    for; rows behind the plan's last one are not written. Decode only: tensors that ask for a gradient, the scales and
    outputs among them, are refused while gradients are enabled, dual tensors always."""
    on = _On((("plan", plan.data), ("q", q), ("k_cache", k_cache), ("v_cache", v_cache), ("k_scale", k_scale),
              ("v_scale", v_scale), ("o", o), ("lse", lse), ("ws", ws)), stream)
    _no_grad("paged_fwd", (q, k_cache, v_cache, k_scale, v_scale, o, lse))
    if q.dim() != 3:
        raise ValueError("q must be [rows, heads, head_dim]")
    d = q.shape[2]
    _want(q, "q", torch.bfloat16, (plan.rows, plan.hq, d))
    kind, k_stride, v_stride = _caches(k_cache, v_cache, k_scale, v_scale, plan, d)
    given = (o, lse, ws)
    _want_ws(ws, "ws")
    with on as st:
        if o is None:
            o = torch.empty_like(q)
        else:
            _want(o, "o", torch.bfloat16, q.shape)
        if want_lse or lse is not None:
            lse = _out(lse, "lse", torch.float32, (plan.hq, plan.rows), on.device)
        n = plan.workspace_size(d) if ws is None else ws.numel()
        if ws is None:
            ws = plan.data.new_empty(n // 4)
        _lib.check(_lib.load().augtree_paged_fwd(
            plan.pages.ref, _addr(plan.data), plan.rows, plan.hq, plan.hkv, d,
            1.0 / math.sqrt(d) if scale is None else float(scale), _addr(q), kind, _addr(k_cache), k_stride,
            _addr(v_cache), v_stride, _addr(k_scale), _addr(v_scale), _addr(o), _addr(lse), _addr(ws), n, st), "paged_fwd")
    _written(given)
    return o, lse
