"""Operators of a population that fine-tunes adapters on shared blocks: low-rank adapters beside a shared projection,
block norms, gradient clipping.

Thin wrappers over the pbt_adapter_*, pbt_block_norm_* and pbt_clip_* calls of the C ABI: argument checks, result allocation and
marshalling; every computation runs in the library's CUDA kernels.  Each call only enqueues work, on `stream` (a torch
stream) or the current stream of the tensors' device; results are allocated for that stream.

The calls build no autograd graph: their backward passes are calls of the caller's, and inputs that require a gradient are
taken as plain numbers.  To put an operator into a graph, call the pair from a torch.autograd.Function.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence

import torch

from .binding import PbtAdapterDesc, PbtBlockNormDesc, PbtClipTensor, PbtError, load_library

_TYPES = {torch.float32: 0, torch.bfloat16: 1}
_MOST = 0x7FFFFFFF      # what the library's 32-bit sizes hold; ctypes would cut a larger one without a word


def _check(rc: int) -> None:
    if rc:
        raise PbtError(rc, load_library().pbt_last_error(None).decode())


def _require(ok, message: str) -> None:
    if not ok:
        raise ValueError(message)


# What torch.cuda.current_stream, current_device and caching_allocator_alloc / _delete rest on, without the Python objects
# around them: those cost a small call more than all of its checks (a workspace as a tensor 1.5 to 2.4 us, like this 0.5).  Bound at the first
# call, which has CUDA tensors: a torch build without CUDA lacks them.
_current_device = _allocate = _release = None


def _current_stream(index):
    global _current_stream, _current_device, _allocate, _release
    _current_device = torch._C._cuda_getDevice
    _allocate, _release = torch._C._cuda_cudaCachingAllocator_raw_alloc, torch._C._cuda_cudaCachingAllocator_raw_delete
    _current_stream = torch._C._cuda_getCurrentRawStream
    return _current_stream(index)


def _on(device, stream, inputs, work, *args):
    """work(stream handle, *args) with `device` and `stream` current, so that what it allocates belongs to the stream.
    When that is not the current stream, the memory of the inputs is kept until it is done with them."""
    index = device.index
    current = _current_stream(index)
    if stream is None or (stream.cuda_stream == current and stream.device == device):
        if _current_device() == index:
            return work(current, *args)
        with torch.cuda.device(device):
            return work(current, *args)
    _require(stream.device == device, "the stream belongs to another device than the tensors")
    for t in inputs:
        if t is not None:
            t.record_stream(stream)
    with torch.cuda.stream(stream):
        return work(stream.cuda_stream, *args)


def _like(x) -> torch.Tensor:
    """A contiguous tensor of x's shape and type."""
    return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _with_workspace(call, desc, nbytes: int, s) -> int:
    """call(desc, workspace, bytes, stream) with a workspace of the current device's allocator (its blocks are 512-byte
    aligned), which may go to the stream's next work as soon as the call has been enqueued."""
    ws = _allocate(max(nbytes, 1), s)
    try:
        return call(desc, ws, nbytes, s)
    finally:
        _release(ws)


# --- gradient clipping ---------------------------------------------------------------------------------------------------


class GradientClip:
    """Global gradient norm per group, and clipping, over many tensors (pbt_clip_*).

    grads: CUDA tensors, contiguous, float32 or bfloat16, where the gradients live; groups: the group (population member)
    of each tensor (default: one group for all); out: tensors that receive the clipped gradients (default: in place).
    Every run() reads the tensors' current contents.

    For gradients that stay where they are, like the slabs of a population: making the object sorts and checks the
    tensors, uploads their table and waits for it (0.3 ms for 96 tensors, 2 ms for 640), which run() then saves.  A loop that
    allocates its gradients anew (autograd's default after set_to_none) should keep them in place, or pays for that every
    step.  An object serves one run at a time: runs on several streams have to be ordered."""

    def __init__(self, grads: Sequence[torch.Tensor], groups: Optional[Sequence[int]] = None,
                 out: Optional[Sequence[torch.Tensor]] = None, n_groups: Optional[int] = None):
        grads = list(grads)
        out = grads if out is None else list(out)
        groups = [0] * len(grads) if groups is None else [int(g) for g in groups]
        _require(grads, "no gradient tensors")
        _require(len(groups) == len(grads) and len(out) == len(grads), "grads, groups and out differ in length")
        self.n_groups = max(groups) + 1 if n_groups is None else int(n_groups)
        _require(max(groups) < _MOST and -_MOST <= min(groups) and abs(self.n_groups) <= _MOST, "groups are 32-bit numbers")
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

        def create(s):
            self._ws, self._home = torch.empty(nbytes.value, dtype=torch.uint8, device=self.device), s
            _check(self.lib.pbt_clip_create(C.byref(self._handle), table, len(grads), self.n_groups, self._ws.data_ptr(),
                                            nbytes.value, s))
        _on(self.device, None, (), create)

    def run(self, max_norm, stream=None) -> torch.Tensor:
        """Clip every group to max_norm (a number, or a float32 tensor [n_groups] on the device); returns the norms
        before clipping, float32 [n_groups]."""
        limits, limit = None, 0.0
        if isinstance(max_norm, torch.Tensor):
            _require(max_norm.dtype is torch.float32 and max_norm.device == self.device and max_norm.is_contiguous()
                     and max_norm.numel() == self.n_groups, "max_norm is a number or a contiguous float32 tensor [n_groups] on the gradients' device")
            limits = max_norm.data_ptr()
        else:
            limit = float(max_norm)
        inputs = () if stream is None else (max_norm if limits else None, *self._keep[0], *self._keep[1])
        return _on(self.device, stream, inputs, self._run, limit, limits)

    def _run(self, s, limit, limits):
        if s != self._home:      # keeps the workspace until the run is done, should the object go first
            self._ws.record_stream(torch.cuda.current_stream(self.device))
        norms = torch.empty(self.n_groups, dtype=torch.float32, device=self.device)
        rc = self.lib.pbt_clip_run(self._handle, limit, limits, norms.data_ptr(), s)
        if rc:
            _check(rc)
        return norms

    def __del__(self):
        if getattr(self, "_handle", None):
            self.lib.pbt_clip_destroy(self._handle)
            self._handle = None


# --- block norms -----------------------------------------------------------------------------------------------------------


class BlockNormOut(NamedTuple):
    y: torch.Tensor                      # residual stream behind the block (x itself without a block)
    u: Optional[torch.Tensor]            # normalised input of the next block
    rstd_block: Optional[torch.Tensor]   # with keep: reciprocal roots for the backward pass, float32 [members, rows]
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
    shape, dtype, device = kind = x.shape, x.dtype, x.device
    if not (x.is_cuda and len(shape) == 3 and dtype in _TYPES):
        raise ValueError("activations are CUDA tensors [members, rows, width], float32 or bfloat16")
    m, rows, width = shape
    if m > _MOST or rows > _MOST or width > _MOST:
        raise ValueError("activations have at most 2^31 - 1 members, rows and columns")
    d = PbtBlockNormDesc()
    d.members, d.rows, d.width, d.dtype = m, rows, width, _TYPES[dtype]
    d.x, d.x_member, d.x_row = _activation(x, kind, "x")
    if block is not None:
        if post_weight is None:
            raise ValueError("a block output needs post_weight")
        d.block, d.block_member, d.block_row = _activation(block, kind, "block")
        d.post_weight = _weight(post_weight, (m, width), device, "post_weight")
        if gate is not None:
            if gate.dim() == 2:
                _require(gate.shape == (m, width) and gate.dtype == dtype and gate.device == device
                         and (gate.stride(1) == 1 or width == 1), "a gate vector is [members, width] of the activations' type")
                d.gate, d.gate_member, d.gate_vector = gate.data_ptr(), gate.stride(0), 1
            else:
                d.gate, d.gate_member, d.gate_row = _activation(gate, kind, "gate")
        if scale is not None:
            d.scale = _weight(scale, (m,), device, "scale")
    else:
        _require(post_weight is None and gate is None and scale is None, "post_weight, gate and scale belong to a block output")
    if next_weight is not None:
        d.next_weight = _weight(next_weight, (m, width), device, "next_weight")
    return d, kind


def _activation(t, kind, name):
    shape, dtype, device = kind
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} has to have the activations' shape, type and device")
    member, row, column = t.stride()
    if column != 1 and shape[2] != 1:
        raise ValueError(f"{name} has to have contiguous columns")
    return t.data_ptr(), member, row


def _weight(t, shape, device, name):
    if t.shape != shape or t.dtype is not torch.float32 or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} has to be a contiguous float32 tensor {list(shape)} on the activations' device")
    return t.data_ptr()


def block_norm_forward(x, block=None, *, post_weight=None, gate=None, scale=None, next_weight=None, eps: float = 1e-6,
                       keep: bool = False, stream=None) -> BlockNormOut:
    """Norms before and after a residual block with its gate and residual scale (pbt_block_norm_forward):
    y = x + scale sigmoid(gate) rms(block) post_weight, u = rms(y) next_weight.

    x, block: [members, rows, width]; post_weight, next_weight: float32 [members, width]; gate: logits, one per element or
    [members, width], or None; scale: float32 [members] or None.  Without `block`, only u from x; without `next_weight`,
    only y.  With `keep`, also the reciprocal roots that the backward pass takes."""
    if block is None and next_weight is None:
        raise ValueError("nothing to compute: neither a block output nor a next norm")
    d, kind = _norm_desc(x, block, post_weight, gate, scale, next_weight)
    d.eps = eps
    return _on(kind[2], stream, (x, block, post_weight, gate, scale, next_weight), _norm_forward, d, kind[0], x, block is not None,
               next_weight is not None, keep)


def _norm_forward(s, d, shape, x, block, nxt, keep):
    y, u, rb, rn = x, None, None, None
    if block:
        y = _like(x)
        d.y = y.data_ptr()
        if keep:
            rb = torch.empty(shape[:2], dtype=torch.float32, device=x.device)
            d.rstd_block = rb.data_ptr()
    if nxt:
        u = _like(x)
        d.u = u.data_ptr()
        if keep:
            rn = torch.empty(shape[:2], dtype=torch.float32, device=x.device)
            d.rstd_next = rn.data_ptr()
    if d.rows:                              # (tensors without elements have no address to hand over)
        rc = load_library().pbt_block_norm_forward(C.byref(d), s)
        if rc:
            _check(rc)
    return BlockNormOut(y, u, rb, rn)


def block_norm_backward(dy, du, y, block=None, *, post_weight=None, gate=None, scale=None, next_weight=None,
                        rstd_block=None, rstd_next=None, stream=None) -> BlockNormGrads:
    """Gradients of block_norm_forward from dy (the residual stream's, or None) and du (None without a next norm), with
    the y and the reciprocal roots of a forward pass that kept them."""
    _require(du is not None or block is not None, "nothing to differentiate: neither du nor a block output")
    _require((du is None) == (next_weight is None), "du and next_weight belong together")
    d, kind = _norm_desc(y, block, post_weight, gate, scale, next_weight)
    if dy is not None:
        d.dy, d.dy_member, d.dy_row = _activation(dy, kind, "dy")
    if du is not None:
        d.du, d.du_member, d.du_row = _activation(du, kind, "du")
        _require(rstd_next is not None, "rstd_next is what the forward pass kept")
        d.rstd_next = _weight(rstd_next, kind[0][:2], kind[2], "rstd_next")
    if block is not None:
        _require(rstd_block is not None, "rstd_block is what the forward pass kept")
        d.rstd_block = _weight(rstd_block, kind[0][:2], kind[2], "rstd_block")
    inputs = (dy, du, y, block, post_weight, gate, scale, next_weight, rstd_block, rstd_next)
    return _on(kind[2], stream, inputs, _norm_backward, d, y, gate, post_weight, scale, next_weight)


def _norm_backward(s, d, y, gate, post_weight, scale, next_weight):
    lib = load_library()
    dblock = dgate = dpost = dnext = dscale = None
    dx = _like(y)
    d.dx = dx.data_ptr()
    if post_weight is not None:
        dblock = _like(y)
        dpost = torch.empty_like(post_weight)
        d.dblock, d.dpost_weight = dblock.data_ptr(), dpost.data_ptr()
        if scale is not None:
            dscale = torch.empty_like(scale)
            d.dscale = dscale.data_ptr()
        if gate is not None:
            dgate = _like(gate)
            d.dgate = dgate.data_ptr()
    if next_weight is not None:
        dnext = torch.empty_like(next_weight)
        d.dnext_weight = dnext.data_ptr()
    if d.rows:
        nbytes = C.c_size_t(0)
        _check(lib.pbt_block_norm_query_workspace(C.byref(d), C.byref(nbytes)))
        _check(_with_workspace(lib.pbt_block_norm_backward, C.byref(d), nbytes.value, s))
    else:                                   # no row contributes: the sums over rows are zero
        for t in (dpost, dscale, dnext, dgate):
            if t is not None:
                t.zero_()
    return BlockNormGrads(dx, dblock, dgate, dpost, dnext, dscale)


# --- adapters --------------------------------------------------------------------------------------------------------------


def _row_stride(t, name):
    row, column = t.stride()
    columns = t.shape[1]
    if column != 1 and columns != 1:
        raise ValueError(f"{name} has to have contiguous columns")
    return row if t.shape[0] > 1 else max(row, columns)      # (a single row may carry any stride)


class AdapterProjection:
    """One shared frozen projection with a low-rank adapter per request or member (pbt_adapter_*).

    weight [outputs, inputs] (contiguous columns), A [adapters, rank, inputs], B [adapters, outputs, rank] (contiguous),
    all float32 or all bfloat16; scale float32 [adapters] (say alpha / rank, a hyperparameter of every member); bias
    float32 [outputs] or None.  The tensors are used where they lie: update A, B and scale in place between calls.

    Rows come in segments: segment j holds rows [row_offsets[j], row_offsets[j + 1]) and uses adapter adapter_ids[j]
    (outside [0, adapters): none); both int32 on the device.  One token per request is a batch of segments of length 1."""

    def __init__(self, weight, A, B, scale, bias=None):
        _require(weight.is_cuda and weight.dim() == 2 and weight.dtype in _TYPES and (weight.stride(1) == 1 or weight.shape[1] == 1),
                 "weight is a CUDA tensor [outputs, inputs], float32 or bfloat16, with contiguous columns")
        n, k = weight.shape
        _require(A.dim() == 3 and A.shape[2] == k and A.dtype == weight.dtype and A.device == weight.device and A.is_contiguous(),
                 "A is a contiguous [adapters, rank, inputs] of the weight's type and device")
        count, rank = A.shape[0], A.shape[1]
        _require(max(n, k, count, rank) <= _MOST, "inputs, outputs, adapters and rank are at most 2^31 - 1")
        _require(B.shape == (count, n, rank) and B.dtype == weight.dtype and B.device == weight.device and B.is_contiguous(),
                 "B is a contiguous [adapters, outputs, rank] of the weight's type and device")
        for t, shape, name in ((scale, (count,), "scale"), (bias, (n,), "bias")):
            _require(t is None or (t.dtype == torch.float32 and t.shape == shape and t.device == weight.device and t.is_contiguous()),
                     f"{name} is a contiguous float32 tensor {list(shape)} on the weight's device")
        self.weight, self.A, self.B, self.scale, self.bias = weight, A, B, scale, bias
        self.lib = load_library()
        d = self._desc = PbtAdapterDesc()
        d.inputs, d.outputs, d.rank, d.n_adapters, d.dtype = k, n, rank, count, _TYPES[weight.dtype]
        d.weight, d.ld_weight, d.A, d.B, d.scale = weight.data_ptr(), _row_stride(weight, "weight"), A.data_ptr(), B.data_ptr(), scale.data_ptr()
        d.bias = bias.data_ptr() if bias is not None else None
        self._status = torch.zeros(8, dtype=torch.int32, device=weight.device)
        self._home = _current_stream(weight.device.index)
        torch.cuda.current_stream(weight.device).synchronize()      # the calls may be on any stream
        d.status_device = self._status.data_ptr()
        d.row_offsets = d.adapter_ids = weight.data_ptr()
        _check(self.lib.pbt_adapter_query_workspace(C.byref(d), 0, C.byref(C.c_size_t(0))))

    def _call(self, x, row_offsets, adapter_ids):
        """The description of a call on these rows (a copy: calls from several threads do not share it)."""
        w = self.weight
        device = w.device
        if not (x.dim() == 2 and x.shape[1] == self._desc.inputs and x.dtype == w.dtype and x.device == device):
            raise ValueError("x is [rows, inputs] of the weight's type and device")
        n = adapter_ids.numel()
        if not (row_offsets.dtype is torch.int32 and adapter_ids.dtype is torch.int32 and row_offsets.numel() == n + 1 and row_offsets.device == device
                and adapter_ids.device == device and row_offsets.is_contiguous() and adapter_ids.is_contiguous()):
            raise ValueError("row_offsets [segments + 1] and adapter_ids [segments] are contiguous int32 tensors on the weight's device")
        if x.shape[0] > _MOST or n > _MOST:
            raise ValueError("a call has at most 2^31 - 1 rows and segments")
        d = PbtAdapterDesc.from_buffer_copy(self._desc)
        d.rows, d.n_segments = x.shape[0], n
        d.row_offsets, d.adapter_ids = row_offsets.data_ptr(), adapter_ids.data_ptr()
        d.x, d.ld_x = x.data_ptr(), _row_stride(x, "x")
        return d

    def forward(self, x, row_offsets, adapter_ids, keep: bool = False, stream=None):
        """y = x W^T + bias + scale_a (x A_a^T) B_a^T; with keep, also S = x A_a^T (float32 [rows, rank], defined for the
        rows that have an adapter), which the backward pass takes."""
        d, w = self._call(x, row_offsets, adapter_ids), self.weight
        return _on(w.device, stream, (x, row_offsets, adapter_ids, w, self.A, self.B, self.scale, self.bias), self._forward, d, keep)

    def _forward(self, s, d, keep):
        w = self.weight
        y = w.new_empty((d.rows, d.outputs))
        d.y, d.ld_y = y.data_ptr(), d.outputs
        kept = None
        if keep:
            kept = torch.empty((d.rows, d.rank), dtype=torch.float32, device=w.device)
            d.s = kept.data_ptr()
        if d.rows:
            self._run(d, 0, self.lib.pbt_adapter_forward, s)
        return (y, kept) if keep else y

    def backward(self, dy, x, kept, row_offsets, adapter_ids, stream=None):
        """(dx, dA, dB) from dy [rows, outputs], the forward pass's x and what it kept; dA and dB are float32."""
        d, w = self._call(x, row_offsets, adapter_ids), self.weight
        _require(dy.shape == (d.rows, d.outputs) and dy.dtype == w.dtype and dy.device == w.device, "dy is [rows, outputs] of the weight's type and device")
        _require(kept.shape == (d.rows, d.rank) and kept.dtype is torch.float32 and kept.device == w.device and kept.is_contiguous(),
                 "kept is what forward(keep=True) returned")
        d.dy, d.ld_dy, d.s = dy.data_ptr(), _row_stride(dy, "dy"), kept.data_ptr()
        return _on(w.device, stream, (x, dy, kept, row_offsets, adapter_ids, w, self.A, self.B, self.scale), self._backward, d)

    def _backward(self, s, d):
        w = self.weight
        dx = w.new_empty((d.rows, d.inputs))
        d_a = torch.empty((d.n_adapters, d.rank, d.inputs), dtype=torch.float32, device=w.device)
        d_b = torch.empty((d.n_adapters, d.outputs, d.rank), dtype=torch.float32, device=w.device)
        d.dx, d.ld_dx, d.dA, d.dB = dx.data_ptr(), d.inputs, d_a.data_ptr(), d_b.data_ptr()
        self._run(d, 1, self.lib.pbt_adapter_backward, s)
        return dx, d_a, d_b

    def check(self):
        """Waits for the enqueued calls and raises if one of the kernels' bounded waits ran out (PBT_ERR_TIMEOUT)."""
        torch.cuda.synchronize(self.weight.device)
        code = int(self._status[4].item())
        if code:
            raise PbtError(code, "a bounded wait inside an adapter kernel ran out")

    def _run(self, d, backward, call, s):
        if s != self._home:      # keeps the status words until the call is done, should the object go first
            self._status.record_stream(torch.cuda.current_stream(self.weight.device))
        nbytes, at = C.c_size_t(0), C.byref(d)
        rc = self.lib.pbt_adapter_query_workspace(at, backward, C.byref(nbytes))
        if not rc:
            rc = _with_workspace(call, at, nbytes.value, s)
        if rc:
            _check(rc)
