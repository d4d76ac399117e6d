"""Layer norm over the last axis with one weight gradient per worker, on the C ABI's signmuon_layernorm_* functions.

    ln = LayerNorm(768, num_workers=16, dtype="bf16")
    y, mean, rstd, s = ln.forward(x, gamma, beta, residual=r)          # s = x + r is normalised, and returned
    dx, dgamma, dbeta = ln.backward(dy, s, gamma, mean, rstd, dsum=ds) # dgamma, dbeta: [num_workers][cols]

One object serves every layer norm of a width; `apply` joins the two passes for torch's autograd.  The rows of x are
num_workers equal runs, worker after worker.  Threads may use one object at once, but its backward passes share the
workspace: one is called after the other has returned, and on the same stream or ordered behind it.
"""
from __future__ import annotations

import ctypes as C
import threading
from typing import Optional

import torch

from . import binding as B

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_stream = torch._C._cuda_getCurrentRawStream     # (a torch.cuda.Stream object costs 2 us)


class _Arguments(threading.local):
    """What a call fills in, for each thread its own: the library is called without the interpreter's lock."""

    def __init__(self, one: torch.Tensor):
        self.forward, self.backward = B.LayerNormForwardStruct(), B.LayerNormBackwardStruct()
        self.statistics = one


class LayerNorm:
    def __init__(self, cols: int, num_workers: int = 1, dtype: str = "bf16", weight_dtype: Optional[str] = None,
                 grad_dtype: Optional[str] = None, eps: float = 1e-5, device: str = "cuda:0", workspace: Optional[torch.Tensor] = None):
        """`workspace`: that of another object of this width, whose backward passes then count as this one's."""
        self.cols, self.num_workers, self.eps = cols, num_workers, eps
        self.device = B.cuda_device(device)
        self._index = self.device.index
        self._alone = torch.cuda.device_count() == 1       # (the only GPU is always the current one)
        self.ctx = None
        names = (dtype, weight_dtype or dtype, grad_dtype or weight_dtype or dtype)
        for n in names:
            if n not in _TORCH:
                raise ValueError(f"types are 'f32' or 'bf16': got {n!r}")
        self.dtype, self.weight_dtype, self.grad_dtype = (_TORCH[n] for n in names)
        self.ctx = B.signmuon_layernorm_create(cols, num_workers, *(B._DT[n] for n in names), eps)
        self._lib = B.load_library()
        self._names, self._whole, self._streams = names, None, set()
        self.workspace = workspace
        if workspace is None:
            self.workspace = torch.empty(B.signmuon_layernorm_workspace_bytes(self.ctx), dtype=torch.uint8, device=self.device)
        elif workspace.dtype != torch.uint8 or workspace.device != self.device or not workspace.is_contiguous():
            raise ValueError(f"workspace is not bytes on {self.device}")
        with torch.cuda.device(self.device):
            B._check(self._lib.signmuon_layernorm_bind(self.ctx, self.workspace.data_ptr(), self.workspace.numel(), _stream(self._index)),
                     "signmuon_layernorm_bind")
        # patterns to allocate by, of one entry each: empty_like costs less than half of empty
        self._weight_gradient = torch.empty(1, dtype=self.grad_dtype, device=self.device).expand(num_workers, cols)
        self._one = torch.empty(1, dtype=torch.float32, device=self.device)
        self._mine = _Arguments(self._one)

    def _meet(self, stream: int):
        """A stream that has not used the workspace yet: should it be freed, the allocator waits for what that one runs by then."""
        self.workspace.record_stream(torch.cuda.current_stream(self.device))
        self._streams.add(stream)

    def close(self):
        if self.ctx:
            B.load_library().signmuon_layernorm_destroy(self.ctx)
            self.ctx = self._whole = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _rows(self, t: torch.Tensor, name: str, like: Optional[torch.Tensor] = None) -> int:
        """Checks an activation and returns the distance of its rows."""
        if (t.dtype is self.dtype and t.get_device() == self._index and t.is_contiguous() and t.dim() and
                (t.size(-1) == self.cols if like is None else t.shape == like.shape)):
            return self.cols
        if t.dtype != self.dtype or t.device != self.device:
            raise ValueError(f"{name} is {t.dtype} on {t.device}: {self.dtype} on {self.device} is wanted")
        if t.dim() < 1 or t.shape[-1] != self.cols or (like is not None and t.shape != like.shape):
            raise ValueError(f"{name} has the shape {tuple(t.shape)}")
        flat = t.view(-1, self.cols)     # torch raises where the rows are not evenly spaced
        if flat.stride(1) != 1 and self.cols > 1:
            raise ValueError(f"{name}: the entries of a row are not neighbours")
        if flat.shape[0] < 2:
            return self.cols
        if flat.stride(0) < self.cols:
            raise ValueError(f"{name}: its rows overlap")
        return flat.stride(0)

    def _weight(self, t: Optional[torch.Tensor], name: str):
        if t is None:
            return None
        if t.dtype is not self.weight_dtype or t.get_device() != self._index or t.numel() != self.cols or not t.is_contiguous():
            raise ValueError(f"{name} is not {self.cols} neighbouring entries of {self.weight_dtype} on {self.device}")
        return t.data_ptr()

    def _statistic(self, t: torch.Tensor, rows: int, name: str):
        if t.dtype is not torch.float32 or t.get_device() != self._index or t.numel() != rows or not t.is_contiguous():
            raise ValueError(f"{name} is not {rows} neighbouring float32 on {self.device}")
        return t.data_ptr()

    def forward(self, x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                residual: Optional[torch.Tensor] = None, stats: bool = True, out: Optional[torch.Tensor] = None):
        """(y, mean, rstd, s).  s is x + residual, or x itself without one; mean and rstd are None without `stats`.
        gamma None: ones, beta None: zeros.  `out` takes y, and may be x (without a residual, s is then what y has become: no
        backward pass can follow)."""
        mine = self._mine
        a = mine.forward
        a.ld_x = self._rows(x, "x")
        rows = a.rows = x.numel() // self.cols
        y = torch.empty_like(x, memory_format=torch.contiguous_format) if out is None else out
        a.ld_y = self.cols if out is None else self._rows(out, "out", x)
        s = x
        if residual is None:
            a.residual = a.sum = None
        else:
            a.ld_residual = self._rows(residual, "residual", x)
            a.residual = residual.data_ptr()
            s = torch.empty_like(x, memory_format=torch.contiguous_format)
            a.ld_sum, a.sum = self.cols, s.data_ptr()
        mean = rstd = None
        if stats:
            if mine.statistics.numel() != rows:
                mine.statistics = self._one.expand(rows)
            mean, rstd = torch.empty_like(mine.statistics), torch.empty_like(mine.statistics)
            a.mean, a.rstd = mean.data_ptr(), rstd.data_ptr()
        else:
            a.mean = a.rstd = None
        a.x, a.y, a.gamma, a.beta = x.data_ptr(), y.data_ptr(), self._weight(gamma, "gamma"), self._weight(beta, "beta")
        call = self._lib.signmuon_layernorm_forward
        if not self._alone and B._current_device() != self._index:
            call = B.on_device(self._index, call)
        code = call(self.ctx, C.byref(a), _stream(self._index))
        if code:
            raise B.SignMuonError(code, "signmuon_layernorm_forward")
        return y, mean, rstd, s

    def backward(self, dy: torch.Tensor, s: torch.Tensor, gamma: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                 dsum: Optional[torch.Tensor] = None, bias: bool = True, out: Optional[torch.Tensor] = None,
                 dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None):
        """(dx, dgamma, dbeta) with dgamma, dbeta [num_workers][cols], dbeta None without `bias`.  s, mean and rstd are those
        of the forward pass; dsum is the gradient that reaches s on another way and is added to dx.  `out` takes dx, and may
        be dy or dsum; dgamma and dbeta may be views whose workers lie apart."""
        a = self._mine.backward
        a.ld_s = self._rows(s, "s")
        a.ld_dy = self._rows(dy, "dy", s)
        rows = a.rows = s.numel() // self.cols
        if rows % self.num_workers:
            raise ValueError(f"{rows} rows for {self.num_workers} workers")
        dx = torch.empty_like(s, memory_format=torch.contiguous_format) if out is None else out
        a.ld_dx = self.cols if out is None else self._rows(out, "out", s)
        a.dsum = None
        if dsum is not None:
            a.ld_dsum = self._rows(dsum, "dsum", s)
            a.dsum = dsum.data_ptr()
        a.mean, a.rstd = self._statistic(mean, rows, "mean"), self._statistic(rstd, rows, "rstd")
        a.dy, a.s, a.gamma, a.dx = dy.data_ptr(), s.data_ptr(), self._weight(gamma, "gamma"), dx.data_ptr()
        dgamma, a.dgamma, a.dgamma_stride = self._gradient(dgamma, "dgamma")
        if bias:
            dbeta, a.dbeta, a.dbeta_stride = self._gradient(dbeta, "dbeta")
        else:
            dbeta = a.dbeta = None
        stream = _stream(self._index)
        if stream not in self._streams:
            self._meet(stream)
        call = self._lib.signmuon_layernorm_backward
        if not self._alone and B._current_device() != self._index:
            call = B.on_device(self._index, call)
        code = call(self.ctx, C.byref(a), stream)
        if code:
            raise B.SignMuonError(code, "signmuon_layernorm_backward")
        return dx, dgamma, dbeta

    def _gradient(self, t: Optional[torch.Tensor], name: str):
        if t is None:
            t = torch.empty_like(self._weight_gradient)
            return t, t.data_ptr(), self.cols
        if t.dtype != self.grad_dtype or t.device != self.device or tuple(t.shape) != (self.num_workers, self.cols):
            raise ValueError(f"{name} is not [{self.num_workers}, {self.cols}] of {self.grad_dtype} on {self.device}")
        if (self.cols > 1 and t.stride(1) != 1) or (self.num_workers > 1 and t.stride(0) < self.cols):
            raise ValueError(f"{name}: the entries of a worker are not neighbours, or the workers overlap")
        return t, t.data_ptr(), t.stride(0) if self.num_workers > 1 else self.cols

    def _of_all_workers(self) -> "LayerNorm":
        """This norm with all rows those of one worker: its weight gradients are the sums over the workers."""
        if self.num_workers == 1:
            return self
        if self._whole is None:
            self._whole = LayerNorm(self.cols, 1, *self._names, self.eps, self.device, self.workspace)
        return self._whole

    def apply(self, x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None):
        """y, or (y, x + residual), for torch's autograd.  gamma and beta are [cols] (their gradient is then the sum over
        the workers, rounded once), or [num_workers, cols] views expanded from one row, which receive every worker's own, or
        None (ones, zeros).  There are no second derivatives: asking for one raises."""
        y, s = _Function.apply(self, x, gamma, beta, residual)
        return y if residual is None else (y, s)


class _Function(torch.autograd.Function):
    @staticmethod
    def forward(fn, ln, x, gamma, beta, residual):
        for name, w in (("gamma", gamma), ("beta", beta)):
            if w is not None and w.dim() == 2 and (w.shape != (ln.num_workers, ln.cols) or (w.shape[0] > 1 and w.stride(0) != 0)):
                raise ValueError(f"{name} is not [{ln.cols}], nor [{ln.num_workers}, {ln.cols}] expanded from one row")
        one = [w[0] if w is not None and w.dim() == 2 else w for w in (gamma, beta)]
        y, mean, rstd, s = ln.forward(x, *one, residual=residual)
        fn.save_for_backward(s, gamma, mean, rstd)
        fn.ln, fn.apart = ln, [w is not None and w.dim() == 2 for w in (beta if gamma is None else gamma, beta)]
        fn.has = (gamma is not None, beta is not None, residual is not None)
        if residual is None:
            fn.mark_non_differentiable(total := s.new_empty(0))
            return y, total
        return y, s

    @staticmethod
    def backward(fn, dy, ds):
        scaled, bias, residual = fn.has
        # (with create_graph as a function of its inputs, so that whoever differentiates it meets the refusal)
        call = _Backward.apply if torch.is_grad_enabled() else _gradients
        dx, dgamma, dbeta = call(fn.ln, fn.apart, bias, dy, ds if residual else None, *fn.saved_tensors)
        return None, dx, dgamma if scaled else None, dbeta, dx if residual else None


def _gradients(ln, apart, bias, dy, ds, s, gamma, mean, rstd):
    args = (dy.contiguous(), s, gamma[0] if gamma is not None and gamma.dim() == 2 else gamma, mean, rstd, None if ds is None else ds.contiguous(), bias)
    if apart[0]:
        dx, dgamma, dbeta = ln.backward(*args)
    else:
        dx, dgamma, dbeta = ln._of_all_workers().backward(*args)
        dgamma = dgamma[0]
    if bias and apart[1] != apart[0]:       # one weight a worker's own, the other shared: a pass for each
        dbeta = (ln if apart[1] else ln._of_all_workers()).backward(*args)[2]
    return dx, dgamma, dbeta[0] if bias and not apart[1] else dbeta


class _Backward(torch.autograd.Function):
    """The backward pass under create_graph.  once_differentiable would not do: its error hangs on a node of its own, which
    autograd.grad leaves out where the inputs asked for are reached on other ways."""

    @staticmethod
    def forward(fn, *args):
        return _gradients(*args)

    @staticmethod
    def backward(fn, *grads):
        raise RuntimeError("layer norm has no second derivatives")
