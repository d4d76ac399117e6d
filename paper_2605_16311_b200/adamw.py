"""AdamW over many tensors at once, with states in 32 or in 8 bits, on the C ABI's signmuon_adamw_* functions.

    opt = AdamW([AdamWParam(w.numel(), dtype="bf16", weight_decay=0.1) for w in weights], num_workers=4, lr=3e-4)
    clip = opt.grad_norm(1.0, grads)           # device tensor [norm, coefficient]
    opt.step(weights, grads, scale=clip[1:])   # nothing here waits for the GPU

The gradients are those of `num_workers` workers, [num_workers][numel] a tensor as SignMuon takes them; a step uses
their mean.  `attach` names weights and gradients once for a program whose tensors stay where they are.
"""
from __future__ import annotations

import ctypes as C
import math
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import binding as B

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_stream = torch._C._cuda_getCurrentRawStream     # (a torch.cuda.Stream object costs 2 us)
BLOCK = 256


@dataclass(frozen=True)
class AdamWParam:
    numel: int
    dtype: str = "f32"                   # of the weights: "f32" | "bf16"
    grad_dtype: Optional[str] = None     # of the gradients; None: the weights'
    weight_decay: float = 0.0            # decoupled
    grad_stride: int = 0                 # entries between two workers' gradients; 0: numel


class AdamW:
    """A context and the torch buffers behind it.  `params` are AdamWParam-like objects; workloads.Param will do."""

    _PARTS = {"exp_avg": B.ADAMW_FIRST_MOMENT, "exp_avg_sq": B.ADAMW_SECOND_MOMENT, "rms": B.ADAMW_SECOND_MOMENT,
              "exp_avg_scale": B.ADAMW_FIRST_SCALE, "rms_scale": B.ADAMW_SECOND_SCALE, "master": B.ADAMW_MASTER_WEIGHT}

    def __init__(self, params: Sequence, num_workers: int = 1, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 state_bits: int = 32, master: bool = False, device: str = "cuda:0"):
        self.params = [AdamWParam(p.numel, p.dtype, getattr(p, "grad_dtype", None) or p.dtype,
                                  getattr(p, "weight_decay", 0.0), getattr(p, "grad_stride", 0)) for p in params]
        self.num_workers, self.state_bits, self.lr = num_workers, state_bits, lr
        self.device = B.cuda_device(device)
        self._index = self.device.index
        self._alone = torch.cuda.device_count() == 1       # (the only GPU is always the current one)
        self.ctx = None
        for p in self.params:
            if p.dtype not in _TORCH or p.grad_dtype not in _TORCH:
                raise ValueError(f"weights and gradients are 'f32' or 'bf16': got {p.dtype!r}, {p.grad_dtype!r}")
        self.ctx = B.signmuon_adamw_create(
            [(p.numel, B._DT[p.dtype], B._DT[p.grad_dtype], p.grad_stride, p.weight_decay) for p in self.params],
            num_workers, lr, betas[0], betas[1], eps, state_bits, B.ADAMW_FLAG_MASTER if master else 0)
        self._lib = B.load_library()
        state_bytes, workspace_bytes = B.signmuon_adamw_state_bytes(self.ctx)
        self.state = torch.empty(state_bytes, dtype=torch.uint8, device=self.device)
        self.workspace = torch.empty(workspace_bytes, dtype=torch.uint8, device=self.device)
        self._weights = self._grads = self._kept = None
        self._streams, self._views, self._two = set(), {}, torch.empty(2, dtype=torch.float32, device=self.device)
        self.rebind()

    # ---- buffers
    def rebind(self, zero_state: bool = True):
        """Binds the buffers again: clears the state, or (zero_state False) goes on with what `state` holds, also where another
        tensor has been put in its place; views taken before are of the old one then."""
        for t in (self.state, self.workspace):
            if t.dtype != torch.uint8 or t.device != self.device or not t.is_contiguous():
                raise ValueError(f"state and workspace are bytes on {self.device}: got {t.dtype} on {t.device}")
        self._views, stream = {}, _stream(self._index)
        self._streams = set()
        self._meet(stream)
        with torch.cuda.device(self.device):
            B._check(self._lib.signmuon_adamw_bind(self.ctx, self.state.data_ptr(), self.state.numel(), self.workspace.data_ptr(),
                                                   self.workspace.numel(), int(zero_state), stream), "signmuon_adamw_bind")

    def _meet(self, stream: int):
        """A stream that has not used the buffers yet: should they be freed, the allocator waits for what it runs by then."""
        for t in (self.state, self.workspace):
            t.record_stream(torch.cuda.current_stream(self.device))
        self._streams.add(stream)

    def close(self):
        if self.ctx:
            B.load_library().signmuon_adamw_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def state_tensor(self, name: str, param: int = -1) -> torch.Tensor:
        """A view of a part of the state, of one tensor or of all (every tensor then starts on a multiple of 256 entries):
        "exp_avg", with 32 bits "exp_avg_sq", with 8 bits (float8_e4m3fn in units of their block's scale) "rms", the root
        of the second moment, and "exp_avg_scale", "rms_scale" for each 256 entries; "master" weights."""
        if (name, param) in self._views:
            return self._views[name, param]
        if name not in self._PARTS or (name == "exp_avg_sq" and self.state_bits == 8) or (name == "rms" and self.state_bits == 32):
            raise KeyError(f"no {name!r} in a state of {self.state_bits} bits")
        offset, nbytes = B.signmuon_adamw_state_segment(self.ctx, self._PARTS[name], param)
        codes = self.state_bits == 8 and name in ("exp_avg", "rms")
        view = self.state[offset:offset + nbytes].view(torch.float8_e4m3fn if codes else torch.float32)
        self._views[name, param] = view
        return view

    def moments(self, param: int = -1):
        """(m, v) in float32, as the state stands for them."""
        if self.state_bits == 32:
            return self.state_tensor("exp_avg", param), self.state_tensor("exp_avg_sq", param)
        m, r = (self.state_tensor(c, param).float() * self.state_tensor(s, param).repeat_interleave(BLOCK)[:self.state_tensor(c, param).numel()]
                for c, s in (("exp_avg", "exp_avg_scale"), ("rms", "rms_scale")))
        return m, r.square_()

    @property
    def steps(self) -> int:
        """Steps taken (waits for the GPU)."""
        return int(self.state[:8].view(torch.int64).item())

    def set_step(self, steps: int):
        """For states that were filled in from elsewhere: the number of steps behind them."""
        stream = _stream(self._index)
        if stream not in self._streams:
            self._meet(stream)
        with torch.cuda.device(self.device):
            B._check(self._lib.signmuon_adamw_set_step(self.ctx, steps, stream), "signmuon_adamw_set_step")

    # ---- tensors
    def _pointers(self, tensors, grads: bool):
        if len(tensors) != len(self.params):
            raise ValueError(f"{len(tensors)} tensors for {len(self.params)} parameters")
        for i, (t, p) in enumerate(zip(tensors, self.params)):
            dtype = _TORCH[p.grad_dtype if grads else p.dtype]
            if t.dtype != dtype or t.device != self.device:
                raise ValueError(f"tensor {i} is {t.dtype} on {t.device}: {dtype} on {self.device} is wanted")
            if not grads:
                if t.numel() != p.numel or not t.is_contiguous():
                    raise ValueError(f"weight {i} is not {p.numel} neighbouring entries")
                continue
            one = t if self.num_workers == 1 and t.numel() == p.numel else t[0] if t.dim() and t.shape[0] == self.num_workers else None
            if one is None or one.numel() != p.numel or not one.is_contiguous():
                raise ValueError(f"gradient {i} is not {self.num_workers} x {p.numel} entries, each worker's neighbours")
            if self.num_workers > 1 and p.numel and t.stride(0) != (p.grad_stride or p.numel):
                raise ValueError(f"gradient {i}: workers lie {t.stride(0)} entries apart, not {p.grad_stride or p.numel}")
        return B._ptr_array([t.data_ptr() for t in tensors])

    def attach(self, weights, grads):
        """Names the tensors of the steps to come (weights None: of norms only), which have to stay where they are.  step()
        and grad_norm() without tensors take these; the checks and the pointers' table are done here, once."""
        w, g = None if weights is None else self._pointers(weights, False), self._pointers(grads, True)
        self._weights, self._grads = w, g
        self._kept = (None if weights is None else tuple(weights), tuple(grads))      # (the caller's lists may change)

    def _scalar(self, t: torch.Tensor):
        if t.dtype != torch.float32 or t.device != self.device or t.numel() != 1:
            raise ValueError("scale is one float32 on the optimizer's device")
        return t.data_ptr()

    def step(self, weights=None, grads=None, lr: Optional[float] = None, scale: Optional[torch.Tensor] = None):
        """One step on the current stream.  `scale`: device float32 that multiplies the mean gradient (a clip coefficient, an
        inverse loss scale); when it is not finite the device skips the step.  Tensors that are given are checked every time, about
        1.3 us each on the host; attached ones are not.  The weights change behind autograd's back: a backward pass of a graph
        that saved them has to come before."""
        if (weights is None) != (grads is None):
            raise ValueError("step takes weights and gradients, or neither")
        w, g = (self._weights, self._grads) if weights is None else (self._pointers(weights, False), self._pointers(grads, True))
        if w is None or g is None:
            raise ValueError("no tensors given, and none attached")
        if lr is not None and not 0 <= lr < math.inf:
            raise ValueError(f"lr is {lr}")
        stream = _stream(self._index)
        if stream not in self._streams:
            self._meet(stream)
        call = self._lib.signmuon_adamw_step
        if not self._alone and B._current_device() != self._index:
            call = B.on_device(self._index, call)
        code = call(self.ctx, w, g, -1.0 if lr is None else lr, None if scale is None else self._scalar(scale), stream)
        if code:
            raise B.SignMuonError(code, "signmuon_adamw_step")

    def grad_norm(self, max_norm: float = math.inf, grads=None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Device tensor of two: the norm of the mean gradient over all tensors, and min(1, max_norm / norm) (NaN when the
        norm is not finite)."""
        g = self._grads if grads is None else self._pointers(grads, True)
        if g is None:
            raise ValueError("no tensors given, and none attached")
        if out is None:
            out = torch.empty_like(self._two)
        elif out.dtype != torch.float32 or out.device != self.device or out.numel() != 2 or not out.is_contiguous():
            raise ValueError("out is two float32 on the optimizer's device")
        stream = _stream(self._index)
        if stream not in self._streams:
            self._meet(stream)
        call = self._lib.signmuon_adamw_grad_norm
        if not self._alone and B._current_device() != self._index:
            call = B.on_device(self._index, call)
        code = call(self.ctx, g, max_norm, out.data_ptr(), stream)
        if code:
            raise B.SignMuonError(code, "signmuon_adamw_grad_norm")
        return out

    @property
    def launches_per_step(self) -> int:
        return B.signmuon_adamw_launches_per_step(self.ctx)
