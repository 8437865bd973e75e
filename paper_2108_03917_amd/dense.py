"""ctypes binding of the dense operators of include/lattice.h: layer
normalisation, the linear classifier with its softmax cross entropy, the
orthogonalised form of a weight gradient, attention over packed sequences with the
norm and rotation of its queries and keys, and clipping by the norm of all
gradients.

Argument marshalling only, as in ``lattice``: tensors are passed as raw device
pointers, outputs are allocated with torch, and every step runs in the
library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import math
from array import array
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
        E_RANGE after a label that is neither a class nor ``ignore_index``, or
        after starts or lengths of an attention that do not fit its rows)."""
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

    # -- attention -----------------------------------------------------------
    def _heads(self, t: torch.Tensor, name: str, shape=None, dtype=None):
        """Check a [rows, heads, C] tensor whose heads' values are next to each
        other; (address, values from row to row, from head to head)."""
        if t.dtype not in _STORAGE or dtype is not None and t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype or ' or '.join(map(str, _STORAGE))}, got {t.dtype}")
        if t.get_device() != self._index:
            raise ValueError(f"{name} must be on {self.device}, is on {t.device}")
        if t.dim() != 3 or shape is not None and t.shape != shape:
            raise ValueError(f"{name} must be {list(shape) if shape is not None else '[rows, heads, channels]'}, "
                             f"is {list(t.shape)}")
        row, head, one = t.stride()
        if one != 1 and t.shape[2] > 1:
            raise ValueError(f"{name}: the values of a head must be next to each other")
        return t.data_ptr(), row, head

    def _starts(self, t: torch.Tensor, n: int, name: str):
        if (t.dtype is not torch.int32 or t.get_device() != self._index or t.dim() != 1 or t.shape[0] != n
                or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous int32 [{n}] on {self.device}")
        return t.data_ptr()

    def _attention(self, q, k, v, q_starts, kv_starts, kv_lengths, scale):
        """Check what both passes take: (dtype .. C), q, k, v, (starts .. sequences), scale."""
        dtype, shape, kv_shape = q.dtype, q.shape, k.shape
        qv = self._heads(q, "q")
        kv = self._heads(k, "k", None, dtype)
        vv = self._heads(v, "v", kv_shape, dtype)
        rows, heads, C = shape
        kv_rows, kv_heads, kC = kv_shape
        if kC != C or kv_heads == 0 or heads % kv_heads:
            raise ValueError(f"k must have heads of {C} channels, as many as divide q's {heads}, is {list(kv_shape)}")
        n, starts, of_keys, lengths = 1, None, None, None
        if q_starts is not None:
            n = q_starts.shape[0] - 1 if q_starts.dim() == 1 else -1
            if n < 0:
                raise ValueError("q_starts must be [sequences + 1]")
            starts = self._starts(q_starts, n + 1, "q_starts")
            if kv_starts is not None:
                of_keys = self._starts(kv_starts, n + 1, "kv_starts")
        elif kv_starts is not None:
            raise ValueError("kv_starts without q_starts")
        if kv_lengths is not None:
            lengths = self._starts(kv_lengths, n, "kv_lengths")
        if scale is None:
            scale = 1 / math.sqrt(C) if C else 1.0
        return (_STORAGE[dtype], rows, kv_rows, heads, kv_heads, C), (*qv, *kv, *vv), (starts, of_keys, lengths, n), scale

    @staticmethod
    def _new(t: torch.Tensor) -> torch.Tensor:
        """An empty contiguous tensor of t's shape and type (what torch.empty gives
        takes the host half as long again)."""
        return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)

    def attention(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_starts: Optional[torch.Tensor] = None,
                  kv_starts: Optional[torch.Tensor] = None, kv_lengths: Optional[torch.Tensor] = None,
                  causal: bool = False, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                  want_lse: bool = False):
        """Softmax attention of ``q`` [rows, heads, C] over ``k`` and ``v``
        [kv_rows, kv_heads, C] (all fp32 or all bf16, any strides but along C; C
        up to 128), a key head for ``heads // kv_heads`` query heads next to each
        other.  ``q_starts`` (int32 [sequences + 1]) packs sequences one behind
        the other; keys have the same starts unless ``kv_starts`` gives theirs, of
        which ``kv_lengths`` (int32 [sequences]) says how many count.  Without
        starts there is one sequence.  With ``causal`` row i of a sequence of n
        sees the keys up to i + (its keys) - n.  ``scale`` is 1 / sqrt(C) unless
        given.  A row that sees no key gets zeros, one that sees a NaN gets NaN; rows
        of no sequence are left alone in a given ``out``, else zeros.  Returns out, with ``want_lse`` also
        the log of each row's sum of exponentials (fp32 [heads, rows]), which the
        backward pass takes.  Of bf16 tensors the probabilities, and the backward
        pass's gradients of scores, are rounded to bf16 for their products; of the
        same widened to fp32 they are not."""
        sizes, tensors, packing, scale = self._attention(q, k, v, q_starts, kv_starts, kv_lengths, scale)
        rest = out is None
        if rest:
            out = self._new(q)
            ov = (out.data_ptr(), sizes[3] * sizes[5], sizes[5])
        else:
            ov = self._heads(out, "out", q.shape, q.dtype)
        lse = torch.empty((q.shape[1], q.shape[0]), dtype=F32, device=q.device) if want_lse else None
        if want_lse and not rest:
            lse.fill_(-math.inf)
        self._call(self._lib.lattice_attention, "attention", *sizes, *tensors, *packing, causal, scale, rest, *ov, _ptr(lse))
        return (out, lse) if want_lse else out

    def attention_backward(self, grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                           out: torch.Tensor, lse: torch.Tensor, q_starts: Optional[torch.Tensor] = None,
                           kv_starts: Optional[torch.Tensor] = None, kv_lengths: Optional[torch.Tensor] = None,
                           causal: bool = False, scale: Optional[float] = None):
        """Gradients of ``attention`` with the same arguments, given ``grad_out``
        and the forward's ``out`` and ``lse``: (grad_q, grad_k, grad_v), contiguous
        and stored as their inputs, zeros for rows of no sequence and for keys that
        do not count."""
        sizes, tensors, packing, scale = self._attention(q, k, v, q_starts, kv_starts, kv_lengths, scale)
        gv = self._heads(grad_out, "grad_out", q.shape, q.dtype)
        ov = self._heads(out, "out", q.shape, q.dtype)
        self._dev(lse, "lse", (F32,))
        if lse.shape != (q.shape[1], q.shape[0]) or not lse.is_contiguous():
            raise ValueError(f"lse must be a contiguous [{q.shape[1]}, {q.shape[0]}]")
        gq, gk, gvv = self._new(q), self._new(k), self._new(v)
        self._call(self._lib.lattice_attention_backward, "attention_backward", *sizes, *gv, *tensors, *ov, lse.data_ptr(),
                   *packing, causal, scale, True, gq.data_ptr(), gk.data_ptr(), gvv.data_ptr())
        return gq, gk, gvv

    # -- norm and rotation of heads ------------------------------------------
    def _rotation(self, q, k, positions, freq, sections, gain_q, gain_k, norm, eps, interleaved):
        """Check q, k and what both passes take: (dtype .. C), q, k, (positions ..
        interleaved)."""
        qv = self._heads(q, "q")
        rows, heads, C = q.shape
        kv, kv_heads = (None, 0, 0), 0
        if k is not None:
            kv = self._heads(k, "k", None, q.dtype)
            k_rows, kv_heads, kC = k.shape
            if k_rows != rows or kC != C:
                raise ValueError(f"k must be [{rows}, heads, {C}], is {list(k.shape)}")
        if positions.dtype not in (F32, torch.int32) or positions.get_device() != self._index:
            raise ValueError(f"positions must be float32 or int32 on {self.device}")
        if positions.dim() == 1:
            positions = positions[:, None]
        shape = positions.shape
        if len(shape) != 2 or shape[0] != rows or shape[1] > 1 and positions.stride(1) != 1:
            raise ValueError(f"positions must be [{rows}, axes], the axes next to each other")
        axes = shape[1]
        if sections is None and freq.dim() == 1:
            sections = (freq.shape[0],)
        if sections is None or len(sections) != axes:
            raise ValueError(f"sections must hold the pairs of each of {axes} axes")
        self._vector(freq, sum(sections), "freq")
        if gain_q is not None:
            self._vector(gain_q, C, "gain_q")
        if gain_k is not None:
            self._vector(gain_k, C, "gain_k")
        return (_STORAGE[q.dtype], rows, heads, kv_heads, C), qv, kv, (
            positions.data_ptr(), positions.dtype is torch.int32, positions.stride(0) if rows > 1 else axes, axes,
            (ctypes.c_int * axes)(*sections), freq.data_ptr(), norm, _ptr(gain_q), _ptr(gain_k), eps, interleaved)

    def rotate_heads(self, q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, freq: torch.Tensor,
                     sections: Optional[Sequence[int]] = None, gain_q: Optional[torch.Tensor] = None,
                     gain_k: Optional[torch.Tensor] = None, norm: bool = True, eps: float = 1e-6,
                     interleaved: bool = False, out_q: Optional[torch.Tensor] = None,
                     out_k: Optional[torch.Tensor] = None):
        """Divide each head's row of ``q`` [rows, heads, C] and ``k`` [rows,
        kv_heads, C] (or None; both fp32 or both bf16, any strides but along C; C
        up to 256, twice ``attention``'s) by the root of its mean square (and ``eps``), multiply by the
        gains (fp32 [C] or None), and turn its pairs of channels by the row's
        ``positions`` [rows, axes] (fp32 or int32; [rows] for one axis) times
        ``freq`` (fp32, one for each pair, radians): ``sections[a]`` pairs with
        axis a, one behind the other, all with a single axis unless given.  Of P
        pairs, pair p is the channels p and p + P, or 2 p and 2 p + 1 if
        ``interleaved``; channels from 2 P on do not turn.  Without ``norm`` only
        the rotation.  Returns (out_q, out_k); the outputs may be the inputs."""
        sizes, qv, kv, rotation = self._rotation(q, k, positions, freq, sections, gain_q, gain_k, norm, eps, interleaved)
        _, _, heads, kv_heads, C = sizes
        if out_q is None:
            out_q = self._new(q)
            oq = (out_q.data_ptr(), heads * C, C)
        else:
            oq = self._heads(out_q, "out_q", q.shape, q.dtype)
        if k is None:
            out_k, ok = None, (None, 0, 0)
        elif out_k is None:
            out_k = self._new(k)
            ok = (out_k.data_ptr(), kv_heads * C, C)
        else:
            ok = self._heads(out_k, "out_k", k.shape, k.dtype)
        self._call(self._lib.lattice_rotate_heads, "rotate_heads", *sizes, *qv, *kv, *rotation, *oq, *ok)
        return out_q, out_k

    def rotate_heads_backward(self, grad_q: torch.Tensor, grad_k: Optional[torch.Tensor], q: torch.Tensor,
                              k: Optional[torch.Tensor], positions: torch.Tensor, freq: torch.Tensor,
                              sections: Optional[Sequence[int]] = None, gain_q: Optional[torch.Tensor] = None,
                              gain_k: Optional[torch.Tensor] = None, norm: bool = True, eps: float = 1e-6,
                              interleaved: bool = False, want_gains: Optional[bool] = None):
        """Gradients of ``rotate_heads`` with the same arguments, given those of
        its results: (of q, of k, of gain_q, of gain_k), the first two contiguous
        and stored as their inputs, the last two fp32 [C], or None with
        ``want_gains`` False (which is so without the norm unless given).
        Positions and frequencies get none."""
        if (k is None) != (grad_k is None):
            raise ValueError("k and grad_k go together")
        sizes, qv, kv, rotation = self._rotation(q, k, positions, freq, sections, gain_q, gain_k, norm, eps, interleaved)
        _, _, heads, kv_heads, C = sizes
        gq = self._heads(grad_q, "grad_q", q.shape, q.dtype)
        out_q, out_k = self._new(q), None
        gk = ok = (None, 0, 0)
        if k is not None:
            gk = self._heads(grad_k, "grad_k", k.shape, k.dtype)
            out_k = self._new(k)
            ok = (out_k.data_ptr(), kv_heads * C, C)
        gain = [None, None]
        if norm if want_gains is None else want_gains:
            both = q.new_empty((2, C), dtype=F32).unbind()
            gain = [both[0], both[1] if k is not None else None]
        self._call(self._lib.lattice_rotate_heads_backward, "rotate_heads_backward", *sizes, *gq, *gk, *qv, *kv, *rotation,
                   out_q.data_ptr(), heads * C, C, *ok, _ptr(gain[0]), _ptr(gain[1]))
        return out_q, out_k, gain[0], gain[1]

    # -- clipping ------------------------------------------------------------
    def clip_gradients(self, grads: Sequence[torch.Tensor], max_norm: float, eps: float = 1e-6,
                       out: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
        """Scale ``grads`` (fp32 or bf16, contiguous, of any shapes) by
        min(1, max_norm / (norm + eps)), where norm is that over all their values,
        in place or into ``out`` (fp32 or bf16, of as many values each).  Returns the norm
        before, an fp32 scalar.  A norm that is not finite is not refused: NaN
        makes every value NaN, infinity makes finite ones 0, unless ``max_norm``
        is infinite: then nothing is scaled.  (A norm of finite values past fp32's
        largest number is returned as infinity, but scales as what it is.)"""
        n = len(grads)

        def check(tensors, name):
            kinds = [_STORAGE.get(t.dtype, -1) for t in tensors]
            if (-1 in kinds or [t.get_device() for t in tensors].count(self._index) != n
                    or not all([t.is_contiguous() for t in tensors])):
                raise ValueError(f"{name} must be {n} contiguous tensors, fp32 or bf16, on {self.device}")
            return array("Q", [t.data_ptr() for t in tensors]), array("i", kinds)

        src, src_t = to, to_t = check(grads, "grads")
        sizes = array("q", [t.numel() for t in grads])
        if out is not None:
            to, to_t = check(out, "out")
            for i, (a, b) in enumerate(zip(sizes, out)):
                if a != b.numel():
                    raise ValueError(f"out[{i}] must hold as many values as grads[{i}], {a}")
        norm = torch.empty((), dtype=F32, device=self.device)
        self._call(self._lib.lattice_clip_gradients, "clip_gradients", n, *[x.buffer_info()[0] for x in (src, src_t, to, to_t,
                   sizes)], max_norm, eps, norm.data_ptr())
        return norm
