"""Operators of a population that fine-tunes adapters on shared blocks: gradient clipping and block norms.

Thin wrappers over the pbt_clip_* and pbt_block_norm_* calls of the C ABI: argument checks, result allocation and
marshalling; every computation runs in the library's CUDA kernels.  Each call only enqueues work, on `stream` (a torch
stream) or the current stream of the tensors' device; results are allocated for that stream.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence

import torch

from .binding import PbtBlockNormDesc, PbtClipTensor, PbtError, load_library

_TYPES = {torch.float32: 0, torch.bfloat16: 1}


def _check(rc: int) -> None:
    if rc:
        raise PbtError(rc, load_library().pbt_last_error(None).decode())


def _require(ok, message: str) -> None:
    if not ok:
        raise ValueError(message)


class _On:
    """Makes `device` and `stream` current for a call; inputs that live on another stream are kept until it is done."""

    def __init__(self, device, stream, inputs=()):
        self.handle = None
        current = torch.cuda.current_stream(device)
        if stream is None or stream == current:
            self.stream, self.scope = current, (None if torch.cuda.current_device() == device.index else torch.cuda.device(device))
        else:
            _require(stream.device == device, "the stream belongs to another device than the tensors")
            self.stream, self.scope = stream, torch.cuda.stream(stream)
            for t in inputs:
                if t is not None:
                    t.record_stream(stream)

    def __enter__(self):
        if self.scope is not None:
            self.scope.__enter__()
        return self.stream.cuda_stream

    def __exit__(self, *exc):
        if self.scope is not None:
            self.scope.__exit__(*exc)


def _workspace(nbytes: int, device) -> torch.Tensor:
    """At least nbytes, 256-byte aligned (the allocator's blocks are 512-byte aligned)."""
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


# --- gradient clipping ---------------------------------------------------------------------------------------------------


class GradientClip:
    """Global gradient norm per group, and clipping, over many tensors (pbt_clip_*).

    grads: CUDA tensors, contiguous, float32 or bfloat16, where the gradients live; groups: the group (population member)
    of each tensor (default: one group for all); out: tensors that receive the clipped gradients (default: in place).
    Every run() reads the tensors' current contents."""

    def __init__(self, grads: Sequence[torch.Tensor], groups: Optional[Sequence[int]] = None,
                 out: Optional[Sequence[torch.Tensor]] = None, n_groups: Optional[int] = None):
        grads = list(grads)
        out = grads if out is None else list(out)
        groups = [0] * len(grads) if groups is None else [int(g) for g in groups]
        _require(grads, "no gradient tensors")
        _require(len(groups) == len(grads) and len(out) == len(grads), "grads, groups and out differ in length")
        self.n_groups = max(groups) + 1 if n_groups is None else int(n_groups)
        self.device = grads[0].device
        table = (PbtClipTensor * len(grads))()
        for e, g, o, k in zip(table, grads, out, groups):
            _require(g.is_cuda and g.device == self.device and o.device == self.device, "gradients live on one CUDA device")
            _require(g.dtype in _TYPES and o.dtype == g.dtype, "gradients are float32 or bfloat16, out has their type")
            _require(g.is_contiguous() and o.is_contiguous() and o.numel() == g.numel(), "gradients and out are contiguous and of equal size")
            e.src, e.dst, e.numel, e.dtype, e.group = g.data_ptr() or None, o.data_ptr() or None, g.numel(), _TYPES[g.dtype], k
        self.lib = load_library()
        self._keep = (grads, out)
        nbytes = C.c_size_t(0)
        _check(self.lib.pbt_clip_query_workspace(table, len(grads), self.n_groups, C.byref(nbytes)))
        self._handle = C.c_void_p(None)
        with _On(self.device, None) as s:
            self._ws = _workspace(nbytes.value, self.device)
            _check(self.lib.pbt_clip_create(C.byref(self._handle), table, len(grads), self.n_groups, self._ws.data_ptr(),
                                            nbytes.value, s))

    def run(self, max_norm, stream=None) -> torch.Tensor:
        """Clip every group to max_norm (a number, or a float32 tensor [n_groups] on the device); returns the norms
        before clipping, float32 [n_groups]."""
        limits, limit = None, 0.0
        if isinstance(max_norm, torch.Tensor):
            _require(max_norm.dtype == torch.float32 and max_norm.device == self.device and max_norm.is_contiguous()
                     and max_norm.numel() == self.n_groups, "max_norm is a number or a contiguous float32 tensor [n_groups] on the gradients' device")
            limits = max_norm.data_ptr()
        else:
            limit = float(max_norm)
        with _On(self.device, stream, (max_norm,) if limits else ()) as s:
            norms = torch.empty(self.n_groups, dtype=torch.float32, device=self.device)
            _check(self.lib.pbt_clip_run(self._handle, limit, limits, norms.data_ptr(), s))
        return norms

    def __del__(self):
        if getattr(self, "_handle", None):
            self.lib.pbt_clip_destroy(self._handle)
            self._handle = None


# --- block norms -----------------------------------------------------------------------------------------------------------


class BlockNormOut(NamedTuple):
    y: torch.Tensor                      # residual stream behind the block (x itself without a block)
    u: Optional[torch.Tensor]            # normalised input of the next block
    rstd_block: Optional[torch.Tensor]   # reciprocal roots for the backward pass, float32 [members, rows]
    rstd_next: Optional[torch.Tensor]


class BlockNormGrads(NamedTuple):
    dx: torch.Tensor
    dblock: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dpost_weight: Optional[torch.Tensor]
    dnext_weight: Optional[torch.Tensor]
    dscale: Optional[torch.Tensor]


def _norm_desc(x, block, post_weight, gate, scale, next_weight):
    """The description of the inputs that both directions share; x stands for y in the backward pass."""
    _require(x.is_cuda and x.dim() == 3 and x.dtype in _TYPES, "activations are CUDA tensors [members, rows, width], float32 or bfloat16")
    m, rows, width = x.shape
    d = PbtBlockNormDesc()
    d.members, d.rows, d.width, d.dtype = m, rows, width, _TYPES[x.dtype]
    d.x, d.x_member, d.x_row = _activation(x, x, "x")
    if block is not None:
        _require(post_weight is not None, "a block output needs post_weight")
        d.block, d.block_member, d.block_row = _activation(block, x, "block")
        d.post_weight = _weight(post_weight, x, (m, width), "post_weight")
        if gate is not None:
            if gate.dim() == 2:
                _require(gate.shape == (m, width) and gate.dtype == x.dtype and gate.device == x.device and gate.stride(1) == 1,
                         "a gate vector is [members, width] of the activations' type")
                d.gate, d.gate_member, d.gate_vector = gate.data_ptr(), gate.stride(0), 1
            else:
                d.gate, d.gate_member, d.gate_row = _activation(gate, x, "gate")
        if scale is not None:
            d.scale = _weight(scale, x, (m,), "scale")
    else:
        _require(post_weight is None and gate is None and scale is None, "post_weight, gate and scale belong to a block output")
    if next_weight is not None:
        d.next_weight = _weight(next_weight, x, (m, width), "next_weight")
    return d


def _activation(t, like, name):
    _require(t.shape == like.shape and t.dtype == like.dtype and t.device == like.device and (t.stride(2) == 1 or t.shape[2] == 1),
             f"{name} has to have the activations' shape, type and device, with contiguous columns")
    return t.data_ptr(), t.stride(0), t.stride(1)


def _weight(t, like, shape, name):
    _require(t.dtype == torch.float32 and t.shape == shape and t.device == like.device and t.is_contiguous(),
             f"{name} has to be a contiguous float32 tensor {list(shape)} on the activations' device")
    return t.data_ptr()


def block_norm_forward(x, block=None, *, post_weight=None, gate=None, scale=None, next_weight=None, eps: float = 1e-6,
                       stream=None) -> BlockNormOut:
    """Norms before and after a residual block with its gate and residual scale (pbt_block_norm_forward):
    y = x + scale sigmoid(gate) rms(block) post_weight, u = rms(y) next_weight.

    x, block: [members, rows, width]; post_weight, next_weight: float32 [members, width]; gate: logits, one per element or
    [members, width], or None; scale: float32 [members] or None.  Without `block`, only u from x; without `next_weight`,
    only y."""
    _require(block is not None or next_weight is not None, "nothing to compute: neither a block output nor a next norm")
    d = _norm_desc(x, block, post_weight, gate, scale, next_weight)
    d.eps = eps
    m, rows, width = x.shape
    y, u, rb, rn = x, None, None, None
    with _On(x.device, stream, (x, block, post_weight, gate, scale, next_weight)) as s:
        if block is not None:
            y = torch.empty((m, rows, width), dtype=x.dtype, device=x.device)
            rb = torch.empty((m, rows), dtype=torch.float32, device=x.device)
            d.y, d.rstd_block = y.data_ptr(), rb.data_ptr()
        if next_weight is not None:
            u = torch.empty((m, rows, width), dtype=x.dtype, device=x.device)
            rn = torch.empty((m, rows), dtype=torch.float32, device=x.device)
            d.u, d.rstd_next = u.data_ptr(), rn.data_ptr()
        if rows:                        # (tensors without elements have no address to hand over)
            _check(load_library().pbt_block_norm_forward(C.byref(d), s))
    return BlockNormOut(y, u, rb, rn)


def block_norm_backward(dy, du, y, block=None, *, post_weight=None, gate=None, scale=None, next_weight=None,
                        rstd_block=None, rstd_next=None, stream=None) -> BlockNormGrads:
    """Gradients of block_norm_forward from dy (the residual stream's, or None) and du (None without a next norm), with
    the forward pass's y and reciprocal roots."""
    _require(du is not None or block is not None, "nothing to differentiate: neither du nor a block output")
    _require((du is None) == (next_weight is None), "du and next_weight belong together")
    d = _norm_desc(y, block, post_weight, gate, scale, next_weight)
    m, rows, width = y.shape
    if dy is not None:
        d.dy, d.dy_member, d.dy_row = _activation(dy, y, "dy")
    if du is not None:
        d.du, d.du_member, d.du_row = _activation(du, y, "du")
        _require(rstd_next is not None, "rstd_next is what the forward pass returned")
        d.rstd_next = _weight(rstd_next, y, (m, rows), "rstd_next")
    if block is not None:
        _require(rstd_block is not None, "rstd_block is what the forward pass returned")
        d.rstd_block = _weight(rstd_block, y, (m, rows), "rstd_block")
    lib = load_library()
    nbytes = C.c_size_t(0)
    dblock = dgate = dpost = dnext = dscale = None
    inputs = (dy, du, y, block, post_weight, gate, scale, next_weight, rstd_block, rstd_next)
    with _On(y.device, stream, inputs) as s:
        dx = torch.empty((m, rows, width), dtype=y.dtype, device=y.device)
        d.dx = dx.data_ptr()
        if block is not None:
            dblock = torch.empty((m, rows, width), dtype=y.dtype, device=y.device)
            dpost = torch.empty((m, width), dtype=torch.float32, device=y.device)
            dscale = torch.empty((m,), dtype=torch.float32, device=y.device)
            d.dblock, d.dpost_weight, d.dscale = dblock.data_ptr(), dpost.data_ptr(), dscale.data_ptr()
            if gate is not None:
                dgate = torch.empty(gate.shape, dtype=y.dtype, device=y.device)
                d.dgate = dgate.data_ptr()
        if du is not None:
            dnext = torch.empty((m, width), dtype=torch.float32, device=y.device)
            d.dnext_weight = dnext.data_ptr()
        if rows:
            _check(lib.pbt_block_norm_query_workspace(C.byref(d), C.byref(nbytes)))
            ws = _workspace(nbytes.value, y.device)
            _check(lib.pbt_block_norm_backward(C.byref(d), ws.data_ptr(), nbytes.value, s))
        else:                           # no row contributes: the sums over rows are zero
            for t in (dpost, dscale, dnext, dgate):
                if t is not None:
                    t.zero_()
    return BlockNormGrads(dx, dblock, dgate, dpost, dnext, dscale if scale is not None else None)
