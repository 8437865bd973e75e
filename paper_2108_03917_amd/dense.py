"""ctypes binding of the dense operators of include/lattice.h: layer
normalisation, the linear classifier with its softmax cross entropy, and the
orthogonalised form of a weight gradient.

Argument marshalling only, as in ``lattice``: tensors are passed as raw device
pointers, outputs are allocated with torch, and every step runs in the
library's HIP kernels.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from .lattice import _STORAGE, _TORCH, OK, Lattice, LatticeError, _ptr, load_library

F32 = torch.float32

# the current stream's handle, without making a Stream object where torch can
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


class Dense:
    """The dense operators on the current device and on one stream (the current
    one unless given).  Called while another stream is current, an operator
    waits for that stream's work so far, and that stream for the operator.
    ``gradient_bits`` (8 or 16) are those of d loss / dz in the products that
    give ``linear_cross_entropy``'s gradients of bf16 operands; few classes of
    few channels have 16 in any case.  No operator records an autograd graph."""

    def __init__(self, stream: Optional[torch.cuda.Stream] = None, gradient_bits: int = 8):
        self._lib = load_library()
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self.device = self.stream.device
        self._index, self._raw = self.device.index, self.stream.cuda_stream
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            st = self._lib.lattice_dense_create(ctypes.c_void_p(self.stream.cuda_stream), ctypes.byref(h))
        if st != OK:
            raise LatticeError(st, f"lattice_dense_create: {self._lib.lattice_status_string(st).decode()}")
        self._h = h
        st = self._lib.lattice_dense_set_gradient_bits(h, gradient_bits)
        if st != OK:
            self.close()
            raise ValueError(f"gradient_bits must be 8 or 16, got {gradient_bits}")

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.lattice_dense_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def status(self) -> int:
        """Synchronise; the device status since the last such call (0 is ok,
        E_RANGE after a label that is neither a class nor ``ignore_index``)."""
        return int(self._lib.lattice_dense_get_status(self._h))

    # -- marshalling ------------------------------------------------------
    def _call(self, fn, what: str, *args):
        if self._h is None:
            raise ValueError("the handle is closed")
        if _raw_stream(self._index) == self._raw:
            st = fn(self._h, *args)
        else:
            here = torch.cuda.current_stream(self.device)
            self.stream.wait_stream(here)
            st = fn(self._h, *args)
            here.wait_stream(self.stream)
        if st != OK:
            msg = self._lib.lattice_dense_last_error(self._h)
            raise LatticeError(st, f"{what}: {self._lib.lattice_status_string(st).decode()}: "
                                   f"{msg.decode() if msg else ''}")

    def _dev(self, t: torch.Tensor, name: str, types):
        if t.dtype not in types:
            raise ValueError(f"{name} must be {' or '.join(map(str, types))}, got {t.dtype}")
        if t.device != self.device:
            raise ValueError(f"{name} must be on {self.device}, is on {t.device}")

    def _rows(self, t: torch.Tensor, name: str, types=_STORAGE) -> int:
        """Check a [rows, C] tensor with unit stride along C; its row stride."""
        self._dev(t, name, types)
        if t.dim() != 2:
            raise ValueError(f"{name} must be [rows, channels]")
        rows, C = t.shape
        stride = t.stride(0)
        if C > 1 and t.stride(1) != 1 or rows > 1 and stride < C:
            raise ValueError(f"{name}: the values of a row must be next to each other, and rows must not overlap")
        return stride if stride > C else C

    def _vector(self, t: Optional[torch.Tensor], n: int, name: str, dtype=F32):
        if t is not None:
            self._dev(t, name, (dtype,))
            if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous [{n}]")

    @staticmethod
    def _like(x: torch.Tensor, dtype: torch.dtype) -> torch.Tensor:
        """An empty contiguous tensor of x's shape (what empty_like gives for a
        contiguous x takes the host half as long)."""
        if dtype == x.dtype and x.is_contiguous():
            return torch.empty_like(x)
        return torch.empty(x.shape, dtype=dtype, device=x.device)

    # -- layer normalisation ----------------------------------------------
    def layer_norm(self, x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                   eps: float = 1e-5, out: Optional[torch.Tensor] = None, out_dtype: Optional[str] = None,
                   lattice: Optional[Lattice] = None, want_stats: bool = False):
        """Normalise each row of ``x`` [rows, C] (fp32 or bf16; rows may be
        strided) over its channels, with the gain ``gamma`` and shift ``beta``
        (fp32 [C], or None).  With ``lattice`` the rows are its vertices, and
        those past V are left alone.  The result is stored as ``out`` or
        ``out_dtype`` say, else as x; with ``want_stats`` also returns the rows'
        (mean, rstd), which the backward pass takes."""
        xs = self._rows(x, "x")
        rows, C = x.shape
        self._vector(gamma, C, "gamma")
        self._vector(beta, C, "beta")
        if out is None:
            out, ys = self._like(x, _TORCH[out_dtype] if out_dtype else x.dtype), C
        else:
            ys = self._rows(out, "out")
            if out.shape != x.shape:
                raise ValueError(f"out must be [{rows}, {C}]")
        mean = rstd = None
        if want_stats:
            mean, rstd = x.new_empty((2, rows), dtype=F32).unbind()
        if lattice is not None and rows < lattice._rows_needed():
            raise ValueError(f"x needs >= {lattice._rows_needed()} rows")
        self._call(self._lib.lattice_layer_norm, "layer_norm", lattice._h if lattice is not None else None,
                   x.data_ptr(), _STORAGE[x.dtype], xs, rows, C, _ptr(gamma), _ptr(beta), eps, out.data_ptr(),
                   _STORAGE[out.dtype], ys, _ptr(mean), _ptr(rstd))
        return (out, mean, rstd) if want_stats else out

    def layer_norm_backward(self, grad_y: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                            gamma: Optional[torch.Tensor] = None, lattice: Optional[Lattice] = None,
                            want_input: bool = True, want_params: bool = True,
                            grad_x: Optional[torch.Tensor] = None):
        """Gradients of ``layer_norm(x, gamma, beta)`` given ``grad_y`` and the
        forward's ``mean`` and ``rstd``: (grad_x stored as x or None, grad_gamma
        and grad_beta fp32 [C] or None)."""
        gs, xs = self._rows(grad_y, "grad_y"), self._rows(x, "x")
        rows, C = x.shape
        if grad_y.shape != x.shape:
            raise ValueError(f"grad_y must be [{rows}, {C}]")
        self._vector(mean, rows, "mean")
        self._vector(rstd, rows, "rstd")
        self._vector(gamma, C, "gamma")
        if lattice is not None and rows < lattice._rows_needed():
            raise ValueError(f"x needs >= {lattice._rows_needed()} rows")
        if grad_x is None and want_input:
            grad_x, os_ = self._like(x, x.dtype), C
        elif grad_x is None:
            os_ = C
        else:
            os_ = self._rows(grad_x, "grad_x", (x.dtype,))
            if grad_x.shape != x.shape:
                raise ValueError(f"grad_x must be [{rows}, {C}]")
        gg = gb = None
        if want_params:
            gg, gb = x.new_empty((2, C), dtype=F32).unbind()
        self._call(self._lib.lattice_layer_norm_backward, "layer_norm_backward",
                   lattice._h if lattice is not None else None, grad_y.data_ptr(), _STORAGE[grad_y.dtype], gs,
                   x.data_ptr(), _STORAGE[x.dtype], xs, rows, C, mean.data_ptr(), rstd.data_ptr(), _ptr(gamma),
                   _ptr(grad_x), os_, _ptr(gg), _ptr(gb))
        return grad_x, gg, gb

    # -- classifier loss ---------------------------------------------------
    def linear_cross_entropy(self, x: torch.Tensor, w: torch.Tensor, target: torch.Tensor,
                             bias: Optional[torch.Tensor] = None, ignore_index: int = -100, reduction: str = "mean",
                             want_rows: bool = False, want_grad: bool = False, want_input: bool = True,
                             want_weight: bool = True, want_bias: Optional[bool] = None):
        """Softmax cross entropy of the logits ``x w^T + bias`` (``x`` [N, C]
        and ``w`` [K, C], both fp32 or both bf16, ``bias`` fp32 [K] or None)
        for the classes ``target`` (int64 [N], ``ignore_index`` for a row
        without a label).  Returns ``loss`` (an fp32 scalar: the "mean" over the
        rows with a label, or the "sum"); with ``want_rows`` (loss, row_losses);
        with ``want_grad`` (loss, grad_x, grad_w, grad_bias), the gradients of
        the loss stored as their inputs (None where ``want_input``,
        ``want_weight`` or ``want_bias``, which is whether there is a bias, say
        so); with both, the row losses come second."""
        xs, ws = self._rows(x, "x"), self._rows(w, "w", (x.dtype,))
        N, C = x.shape
        K = w.shape[0]
        if w.shape[1] != C:
            raise ValueError(f"w must be [K, {C}]")
        self._vector(target, N, "target", torch.int64)
        self._vector(bias, K, "bias")
        if reduction not in ("mean", "sum"):
            raise ValueError("reduction must be 'mean' or 'sum'")
        loss = x.new_empty((), dtype=F32)
        rows = x.new_empty((N,), dtype=F32) if want_rows else None
        gx = gw = gb = None
        if want_grad:
            if want_input:
                gx = self._like(x, x.dtype)
            if want_weight:
                gw = self._like(w, w.dtype)
            if want_bias if want_bias is not None else bias is not None:
                gb = torch.empty_like(bias) if bias is not None else x.new_empty((K,), dtype=F32)
        self._call(self._lib.lattice_linear_cross_entropy, "linear_cross_entropy", _STORAGE[x.dtype], x.data_ptr(), xs,
                   N, C, w.data_ptr(), ws, K, _ptr(bias), target.data_ptr(), ignore_index, reduction == "mean",
                   loss.data_ptr(), _ptr(rows), _ptr(gx), _ptr(gw), _ptr(gb))
        out = (loss,) + ((rows,) if want_rows else ()) + ((gx, gw, gb) if want_grad else ())
        return out if len(out) > 1 else loss

    # -- orthogonalised update ---------------------------------------------
    def orthogonalize(self, g: torch.Tensor, steps: int = 5,
                      coefficients: Sequence[float] = (3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                      out: Optional[torch.Tensor] = None, out_dtype: Optional[str] = None) -> torch.Tensor:
        """``steps`` Newton-Schulz steps on ``g`` [m, n] or on each matrix of
        ``g`` [batch, m, n] (fp32 or bf16): X = g / (|g| + eps), then
        X <- a X + (b S + c S S) X with S = X X^T.  Stored as ``out`` or
        ``out_dtype`` say, else as g."""
        self._dev(g, "g", _STORAGE)
        if g.dim() not in (2, 3):
            raise ValueError("g must be [m, n] or [batch, m, n]")
        m, n = g.shape[-2:]
        batch = g.shape[0] if g.dim() == 3 else 1
        rs = g.stride(-2)
        if n > 1 and g.stride(-1) != 1 or m > 1 and rs < n:
            raise ValueError("g: the values of a row must be next to each other, and rows must not overlap")
        if out is None:
            out = self._like(g, _TORCH[out_dtype] if out_dtype else g.dtype)
        else:
            self._dev(out, "out", _STORAGE)
        if out.shape != g.shape or not out.is_contiguous():
            raise ValueError(f"out must be a contiguous {list(g.shape)}")
        a, b, c = coefficients
        self._call(self._lib.lattice_orthogonalize, "orthogonalize", g.data_ptr(), _STORAGE[g.dtype], batch, m, n,
                   g.stride(0) if g.dim() == 3 else 0, rs if rs > n else n, steps, (ctypes.c_float * 3)(a, b, c), eps,
                   out.data_ptr(), _STORAGE[out.dtype])
        return out
