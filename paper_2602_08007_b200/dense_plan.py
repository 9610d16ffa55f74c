"""DensePlan: dense parameters through the tsr_dense_plan calls (see include/tsr.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes
from typing import List, Optional, Sequence

import torch

from .binding import (
    DENSE_BLOCK, TSR_BF16, TSR_DENSE_NORM_ONLY, TSR_DENSE_STATE_ONLY, TSR_F32, TSR_OK, TSR_ROUND_NEAREST, TSR_STATE_F32, TSR_STATE_Q8,
    DenseDesc, DensePtrs, Hyper, TsrError, lib,
)

_DTYPE = {torch.float32: TSR_F32, torch.bfloat16: TSR_BF16}
# The handle of torch's current stream on a device, without a Stream object around it (2 us of the 6 us of a small call).
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _matrix(t: torch.Tensor, what: str):
    """(rows, columns, pitch) of a tensor whose elements, in row-major order, are rows of a pitched matrix."""
    if t.is_contiguous():
        return 1, t.numel(), t.numel()
    if t.dim() == 1:
        rows, cols, ld = t.shape[0], 1, t.stride(0)
    elif t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1):
        rows, cols, ld = t.shape[0], t.shape[1], t.stride(0)
    else:
        raise ValueError("%s must be contiguous, or a vector or matrix with unit column stride" % what)
    if ld < cols:
        raise ValueError("%s has rows that overlap" % what)
    return rows, cols, ld


class DensePlan:
    """Owns a tsr_dense_plan and references to the tensors it is bound to.

    params, grads: lists of equally shaped tensors, FP32 or BF16, contiguous or (vectors, matrices) with a row pitch.
    params None: the gradients count in grad_norm and nothing is stepped.  norm_only: further such gradients, for
    instance the G of TSR blocks, which the plan lists behind the others.
    states: per tensor (m, v) FP32, or (m8, r8, scale) with torch.float8_e4m3fn values and an FP32 scale tensor of two
    values per block of 256 elements; None: zero states of state_dtype (torch.float32 or torch.float8_e4m3fn, or a list of
    them, one per tensor).  params and grads both None: states alone, for copy_state.
    images: per tensor None or a BF16 tensor that every step fills with the updated FP32 parameter.
    lr_mult, wd_mult: per-tensor factors on hyper.lr and hyper.weight_decay.

    The tensors are taken as they lie: after replacing entries of .grads (or any other list), call bind().  A plan over the .grad
    of parameters goes on with the old tensors where torch's zero_grad has replaced them: use set_to_none=False.

    Calls go to torch's current stream, or to `stream`.  What the plan itself allocates (its tables, the result of grad_norm,
    zero states) is handed back to torch's allocator only after the work that the calls put on their streams; tensors of the
    caller need record_stream where they are dropped while another stream than their own uses them.  The norms of one plan
    run one after the other, whatever their streams (the last one's stream has to exist when another takes over).  A captured
    graph holds addresses of the plan and of its tensors, and repeats the hyper and the seed of its capture: keep the plan, do
    not bind() it again while the graph is replayed, and let no norm of the plan run beside a replayed one."""

    def __init__(self, params: Optional[Sequence[torch.Tensor]], grads: Optional[Sequence[torch.Tensor]], states=None,
                 state_dtype=torch.float32, images=None, lr_mult: Optional[Sequence[float]] = None,
                 wd_mult: Optional[Sequence[float]] = None, norm_only: Sequence[torch.Tensor] = ()):
        self.ctx = ctypes.c_void_p()
        self.params: List[torch.Tensor] = list(params or [])
        self.grads: List[torch.Tensor] = list(grads or [])
        self.norm_only: List[torch.Tensor] = list(norm_only)
        if params is not None and len(self.params) != len(self.grads):
            raise ValueError("params and grads must list the same number of tensors")
        if params is None and grads is not None:
            if states is not None:
                raise ValueError("gradients without parameters have no state")
            self.norm_only, self.grads = self.grads + self.norm_only, []
        n = len(states) if params is None and states is not None else len(self.params)
        self._stepped = params is not None
        first = next((t for t in self.params + self.norm_only), None)
        if first is None and states:
            first = states[0][0]
        self.device = first.device if first is not None else torch.device("cuda", torch.cuda.current_device())
        if self.device.type != "cuda":
            raise ValueError("tensors must live on a CUDA device")
        self._index = self.device.index
        self._lib = lib()
        self.states = self._zero_states(state_dtype) if states is None else [tuple(s) for s in states]
        self._made_states = states is None
        self._home = _current_stream(self._index)      # on which the states and the result of grad_norm are allocated
        self.images = list(images) if images is not None else [None] * n
        self.lr_mult = [1.0] * n if lr_mult is None else [float(x) for x in lr_mult]
        self.wd_mult = [1.0] * n if wd_mult is None else [float(x) for x in wd_mult]
        for what, x in (("states", self.states), ("images", self.images), ("lr_mult", self.lr_mult), ("wd_mult", self.wd_mult)):
            if len(x) != n:
                raise ValueError("%s must have one entry per tensor" % what)
        self._result = torch.zeros(2, dtype=torch.float32, device=self.device)
        self.bind()

    # -- plumbing ---------------------------------------------------------------------------
    def _zero_states(self, state_dtype):
        kinds = list(state_dtype) if isinstance(state_dtype, (list, tuple)) else [state_dtype] * len(self.params)
        if len(kinds) != len(self.params) or any(k not in (torch.float32, torch.float8_e4m3fn) for k in kinds):
            raise ValueError("state_dtype is torch.float32 or torch.float8_e4m3fn, for all tensors or in a list")
        out = []
        for p, kind in zip(self.params, kinds):
            n = p.numel()
            if kind == torch.float32:
                out.append((torch.zeros(n, dtype=kind, device=self.device), torch.zeros(n, dtype=kind, device=self.device)))
            else:
                out.append(tuple(torch.zeros(n, dtype=torch.uint8, device=self.device).view(kind) for _ in range(2)) +
                           (torch.zeros((n + DENSE_BLOCK - 1) // DENSE_BLOCK, 2, dtype=torch.float32, device=self.device),))
        return out

    def _state_desc(self, i: int, n: int):
        s = self.states[i]
        kind = torch.float32 if len(s) == 2 else torch.float8_e4m3fn
        if len(s) not in (2, 3) or any(t.dtype != kind for t in s[:2]) or (len(s) == 3 and s[2].dtype != torch.float32):
            raise ValueError("state %d must be (m, v) in FP32 or (m8, r8, scale) in torch.float8_e4m3fn and FP32" % i)
        if any(t.device != self.device or not t.is_contiguous() for t in s):
            raise ValueError("state %d must be contiguous and on %s" % (i, self.device))
        if any(t.numel() != n for t in s[:2]) or (len(s) == 3 and s[2].numel() != 2 * ((n + DENSE_BLOCK - 1) // DENSE_BLOCK)):
            raise ValueError("state %d does not have the tensor's size" % i)
        return TSR_STATE_F32 if len(s) == 2 else TSR_STATE_Q8

    def _describe(self):
        """Descriptors and pointers of all tensors, from the lists as they are now."""
        descs, ptrs = [], []
        for t in self.params + self.grads + self.norm_only + [x for x in self.images if x is not None]:
            if t.dtype not in _DTYPE or t.device != self.device:
                raise ValueError("parameters, gradients and images must be FP32 or BF16 tensors on %s" % self.device)
        for i, s in enumerate(self.states):
            if not self._stepped:
                n = s[0].numel()
                kind = self._state_desc(i, n)
                descs.append(DenseDesc(1, n, n, n, n, TSR_F32, TSR_F32, kind, TSR_DENSE_STATE_ONLY, 1.0, 1.0))
                ptrs.append(DensePtrs(None, None, s[0].data_ptr(), s[1].data_ptr(), s[2].data_ptr() if len(s) == 3 else None, None))
                continue
            p, g, image = self.params[i], self.grads[i], self.images[i]
            if p.shape != g.shape or (image is not None and (image.shape != p.shape or image.dtype != torch.bfloat16)):
                raise ValueError("tensor %d: parameter, gradient and (BF16) image must have the same shape" % i)
            forms = [_matrix(t, "tensor %d" % i) for t in (p, g) + ((image,) if image is not None else ())]
            pitched = next(((r, c) for (r, c, ld) in forms if r != 1), None)
            # one shape for all of them: that of a pitched one, in which the contiguous ones have pitch = columns
            rows, cols = pitched if pitched else forms[0][:2]
            ld = [f[2] if f[0] != 1 else cols for f in forms]
            kind = self._state_desc(i, p.numel())
            descs.append(DenseDesc(rows, cols, ld[0], ld[1], ld[2] if image is not None else cols, _DTYPE[p.dtype], _DTYPE[g.dtype], kind, 0,
                                   self.lr_mult[i], self.wd_mult[i]))
            ptrs.append(DensePtrs(p.data_ptr(), g.data_ptr(), s[0].data_ptr(), s[1].data_ptr(), s[2].data_ptr() if len(s) == 3 else None,
                                  image.data_ptr() if image is not None else None))
        for i, g in enumerate(self.norm_only):
            rows, cols, ld = _matrix(g, "norm-only gradient %d" % i)
            descs.append(DenseDesc(rows, cols, cols, ld, cols, TSR_F32, _DTYPE[g.dtype], TSR_STATE_F32, TSR_DENSE_NORM_ONLY, 1.0, 1.0))
            ptrs.append(DensePtrs(None, g.data_ptr(), None, None, None, None))
        return descs, ptrs

    def _check(self, status: int):
        if status != TSR_OK:
            raise TsrError(status, lib().tsr_dense_plan_last_error(self.ctx).decode() if self.ctx else "")

    def bind(self):
        """Points the plan at the tensors its lists hold now.  Synchronises the device."""
        descs, ptrs = self._describe()
        n = len(descs)
        with torch.cuda.device(self.device):
            self.close()
            self._check(lib().tsr_dense_plan_create(ctypes.byref(self.ctx), (DenseDesc * max(n, 1))(*descs), n))
            size = ctypes.c_size_t()
            self._check(lib().tsr_dense_plan_workspace_bytes(self.ctx, ctypes.byref(size)))
            self.workspace = torch.empty(size.value + 256, dtype=torch.uint8, device=self.device)
            # the device is idle after a binding: no norm to wait for
            self._norm_handle, self._norm_stream = None, None
            # streams that the allocator knows to use what the plan has allocated
            self._met = {self._home} if _current_stream(self._index) == self._home else set()
            at = (self.workspace.data_ptr() + 255) // 256 * 256
            self._check(lib().tsr_dense_plan_bind(self.ctx, (DensePtrs * max(n, 1))(*ptrs), n, at, size.value))

    def close(self):
        if self.ctx:
            lib().tsr_dense_plan_destroy(self.ctx)
            self.ctx = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self, stream):
        handle = _current_stream(self._index) if stream is None else stream.cuda_stream
        if handle not in self._met:
            s = torch.cuda.current_stream(self._index) if stream is None else stream
            for t in [self.workspace, self._result] + ([t for st in self.states for t in st] if self._made_states else []):
                t.record_stream(s)
            self._met.add(handle)
        return handle

    def _order_norms(self, handle: int, stream):
        """The norms of a plan share its partial sums, so one on another stream than the last waits for that stream.  (A
        capture cannot wait for work outside of it: whoever replays a captured norm orders it.)"""
        s = torch.cuda.current_stream(self._index) if stream is None else stream
        for x in (s, self._norm_stream):
            if x is not None:
                with torch.cuda.stream(x):
                    if torch.cuda.is_current_stream_capturing():
                        return
        if self._norm_stream is not None:
            s.wait_stream(self._norm_stream)
        self._norm_handle, self._norm_stream = handle, s

    # -- the C calls --------------------------------------------------------------------------
    def step(self, hyper: Hyper, grad_scale: Optional[torch.Tensor] = None, rounding: int = TSR_ROUND_NEAREST, seed: int = 0, stream=None):
        """One AdamW step.  grad_scale: None or an FP32 tensor on the device whose first element multiplies every gradient
        (a step whose factor is not finite changes nothing)."""
        scale = None
        if grad_scale is not None:
            if grad_scale.dtype != torch.float32 or grad_scale.device != self.device or grad_scale.numel() < 1:
                raise ValueError("grad_scale must be an FP32 tensor on %s" % self.device)
            scale = grad_scale.data_ptr()
        status = self._lib.tsr_dense_plan_step(self.ctx, ctypes.byref(hyper), scale, rounding, seed, self._stream(stream))
        if status != TSR_OK:
            self._check(status)

    def grad_norm(self, max_norm: float = float("inf"), out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """(norm, clipping factor) of all gradients as an FP32 tensor on the device: `out`, or one the plan owns and the next
        call overwrites."""
        if out is None:
            out = self._result
        elif out.dtype != torch.float32 or out.device != self.device or out.numel() < 2 or not out.is_contiguous():
            raise ValueError("out must be a contiguous FP32 tensor of two elements on %s" % self.device)
        handle = self._stream(stream)
        if handle != self._norm_handle:
            self._order_norms(handle, stream)
        status = self._lib.tsr_dense_plan_grad_norm(self.ctx, max_norm, out.data_ptr(), handle)
        if status != TSR_OK:
            self._check(status)
        return out

    def copy_state(self, src: "DensePlan", stream=None):
        """Takes over the moments of `src`, a plan over tensors of the same sizes, converting between FP32 and 8 bits."""
        self._check(self._lib.tsr_dense_plan_copy_state(self.ctx, src.ctx, self._stream(stream)))
        src._stream(stream)        # its tables are read there too
