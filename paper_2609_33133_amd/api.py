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
        elif self.device.index != torch.cuda.current_device():
            self.guard = torch.cuda.device(self.device)
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream().cuda_stream

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
    for t in given:
        if t is not None:
            torch.autograd.graph.increment_version(t)


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
