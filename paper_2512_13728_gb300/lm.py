"""Language-model operators over torch CUDA tensors: argument checks and marshalling only.

``EmbedPlan``: token embedding with scaling, and its gradient by sorted tokens.
``QKNormPlan``: norm and rotation of queries and keys, and their gradient.
``distill_loss``, ``distill_loss_grad``: distillation from a teacher's top logits.

Every call enqueues kernels of libcurvadion.so on `stream` (a raw CUDA stream; None: torch's
current stream of the tensors' device) and returns at once.  Outputs that the caller does not pass
are allocated by torch on its current stream, so a call with an explicit `stream` takes them from
the caller.  A tensor that was made on another stream is the caller's to synchronize, as with any
torch operation.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import native

_DTYPES = {torch.float32: native.DION_DTYPE_FP32, torch.bfloat16: native.DION_DTYPE_BF16}
_INDEX = {torch.int32: native.DION_INDEX_INT32, torch.int64: native.DION_INDEX_INT64}


def _stream(device, stream: Optional[int], outputs_given: bool) -> int:
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    if not outputs_given:
        raise ValueError("a call on an explicit stream takes its outputs from the caller")
    return stream


def _reshaped(name: str, t, shape, stream: Optional[int]):
    """t in another shape; torch copies on its current stream where the strides need it."""
    r = t.reshape(shape)
    if stream is not None and r.data_ptr() != t.data_ptr():
        raise ValueError(f"{name} must be contiguous for a call on an explicit stream")
    return r


def _rows(name: str, t, device):
    """dtype code and leading dimension of a row-major 2-D matrix."""
    code = _DTYPES.get(t.dtype)
    if code is None or t.dim() != 2 or t.device != device or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a row-major 2-D float32 or bfloat16 tensor on {device}")
    return code, max(t.stride(0), t.shape[1])


def _indices(name: str, t, device) -> int:
    code = _INDEX.get(t.dtype)
    if code is None or t.device != device:
        raise ValueError(f"{name} must be an int32 or int64 tensor on {device}")
    return code


class EmbedPlan:
    """Token embedding for a table of `vocab` rows of `dim` elements; the plan holds the workspace of
    the gradient's sort for up to `max_tokens` tokens a call.  Tokens outside [0, vocab) are padding:
    rows of zeros, no gradient.  Tables and activations are float32 or bfloat16, tokens int32 or int64."""

    def __init__(self, vocab: int, dim: int, max_tokens: int, device=None):
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.vocab, self.dim, self.max_tokens = vocab, dim, max_tokens
        with torch.cuda.device(self.device):
            self.handle = native.dion_embed_plan_create(vocab, dim, max_tokens)

    def lookup(self, tokens, table, scale: float = 1.0, out=None, dtype=None, stream: Optional[int] = None):
        """scale * table[tokens], shape tokens.shape + (dim,), of `dtype` (the table's by default)."""
        kind = _indices("tokens", tokens, self.device)
        code, ldt = _rows("table", table, self.device)
        if table.shape[0] != self.vocab or table.shape[1] != self.dim:
            raise ValueError(f"table must be {self.vocab} x {self.dim}")
        s = _stream(self.device, stream, out is not None)
        flat = _reshaped("tokens", tokens, -1, stream)
        n = flat.shape[0]
        if out is None:
            out = torch.empty((*tokens.shape, self.dim), dtype=dtype or table.dtype, device=self.device)
        elif tuple(out.shape) != (*tokens.shape, self.dim) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must have the shape of tokens, and dim, and the given dtype")
        rows = out if out.dim() == 2 else out.view(n, self.dim)
        out_code, ldo = _rows("out", rows, self.device)
        native.dion_embed_lookup(self.handle, flat.data_ptr(), kind, n, table.data_ptr(), code, ldt, scale,
                                 out.data_ptr(), out_code, ldo, s)
        return out

    def gradient(self, tokens, grad, scale: float = 1.0, out=None, dtype=None, accumulate: bool = False,
                 stream: Optional[int] = None):
        """Gradient of the table, vocab x dim, of `dtype` (float32 by default), from the gradient `grad`
        of the lookup's output.  accumulate: added to `out`, of which only the tokens' rows are touched."""
        kind = _indices("tokens", tokens, self.device)
        if tuple(grad.shape) != (*tokens.shape, self.dim):
            raise ValueError("grad must have the shape of tokens, and dim")
        s = _stream(self.device, stream, out is not None)
        flat = _reshaped("tokens", tokens, -1, stream)
        n = flat.shape[0]
        rows = grad if grad.dim() == 2 else _reshaped("grad", grad, (n, self.dim), stream)
        code, ldg = _rows("grad", rows, self.device)
        if out is None:
            if accumulate:
                raise ValueError("accumulate adds to a given out")
            out = torch.empty((self.vocab, self.dim), dtype=dtype or torch.float32, device=self.device)
        elif tuple(out.shape) != (self.vocab, self.dim) or (dtype is not None and out.dtype != dtype):
            raise ValueError(f"out must be {self.vocab} x {self.dim} of the given dtype")
        out_code, ldo = _rows("out", out, self.device)
        native.dion_embed_gradient(self.handle, flat.data_ptr(), kind, n, rows.data_ptr(), code, ldg, scale,
                                   out.data_ptr(), out_code, ldo, accumulate, s)
        return out

    def close(self) -> None:
        if getattr(self, "handle", None):
            native.dion_embed_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class QKNormPlan:
    """RMS norm of each query and key head, and the rotation by position of its first `rotary_dim`
    elements (all by default), in one pass; pairs (j, j + rotary_dim / 2), or neighbours with `interleaved`.
    `inv_freq`: rotary_dim / 2 angles per position, instead of theta ** (-2 j / rotary_dim).

    q, k: float32 or bfloat16, [batch, tokens, heads, head_dim] in any strides with contiguous heads
    (views of a packed projection, transposed layouts), or [tokens, heads, head_dim].  k may be None.
    Weights: float32 [head_dim] or None.  positions: int32 or int64, [batch, tokens] or [tokens]; None:
    0, 1, ... in each sequence."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, theta: float = 10000.0, interleaved: bool = False,
                 eps: float = 1e-6, inv_freq=None, device=None):
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.head_dim = head_dim
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if inv_freq is not None and len(inv_freq) != rotary_dim // 2:
            raise ValueError("inv_freq must have rotary_dim / 2 values")
        with torch.cuda.device(self.device):
            self.handle = native.dion_qknorm_plan_create(head_dim, rotary_dim, interleaved, theta, inv_freq, eps)

    def _heads(self, name: str, t, like=None):
        """dion_heads of a tensor; `like`: the tensor whose shape and dtype it must have."""
        if t is None:
            return None
        ok = t.dtype in _DTYPES and t.device == self.device and t.dim() in (3, 4) and t.shape[-1] == self.head_dim
        if not ok or t.stride(-1) != 1 or (like is not None and (t.shape != like.shape or t.dtype != like.dtype)):
            raise ValueError(f"{name} must be a float32 or bfloat16 tensor [batch, tokens, heads, {self.head_dim}] on "
                             f"{self.device} with contiguous heads, alike in shape and dtype where it belongs to another")
        st = t.stride()
        return native.dion_heads(t.data_ptr(), st[0] if t.dim() == 4 else 0, st[-3], st[-2])

    def _shape(self, q, k, positions):
        batch = q.shape[0] if q.dim() == 4 else 1
        tokens = q.shape[-3]
        if k is not None and (k.shape[:-2] != q.shape[:-2] or k.dtype != q.dtype):
            raise ValueError("q and k must agree in batch, tokens and dtype")
        ptr, kind, stride = None, 0, 0
        if positions is not None:
            kind = _indices("positions", positions, self.device)
            if positions.shape != q.shape[:-2] and positions.shape != (tokens,) or (tokens > 1 and positions.stride(-1) != 1):
                raise ValueError("positions must be [batch, tokens] or [tokens], contiguous over tokens")
            ptr, stride = positions.data_ptr(), positions.stride(0) if positions.dim() == 2 else 0
        return native.dion_qk_shape(batch, tokens, q.shape[-2], k.shape[-2] if k is not None else 0, _DTYPES[q.dtype], kind,
                                    ptr, stride)

    def _weight(self, name: str, w):
        if w is None:
            return None
        if w.dtype != torch.float32 or w.device != self.device or tuple(w.shape) != (self.head_dim,) or w.stride(0) != 1:
            raise ValueError(f"{name} must be a contiguous float32 tensor of {self.head_dim} elements on {self.device}")
        return w.data_ptr()

    def forward(self, q, k=None, wq=None, wk=None, positions=None, out=None, stream: Optional[int] = None):
        """(q', k'), written into `out` (a pair; q and k themselves: in place) or new contiguous tensors."""
        hq, hk = self._heads("q", q), self._heads("k", k)
        shape = self._shape(q, k, positions)
        s = _stream(self.device, stream, out is not None)
        if out is None:
            out = (torch.empty(q.shape, dtype=q.dtype, device=self.device),
                   None if k is None else torch.empty(k.shape, dtype=k.dtype, device=self.device))
        oq, ok = out
        if (ok is None) != (k is None):
            raise ValueError("out must have a tensor for k where there is one")
        native.dion_qknorm_forward(self.handle, shape, hq, hk, self._weight("wq", wq), self._weight("wk", wk),
                                   self._heads("out[0]", oq, q), self._heads("out[1]", ok, k), s)
        return oq, ok

    def backward(self, gq, gk, q, k=None, wq=None, wk=None, positions=None, out=None, stream: Optional[int] = None):
        """(dq, dk, dwq, dwk) from the gradients of forward's outputs and forward's inputs; the last two are
        None where the weight is.  `out`: the four to write into (dq, dk may be gq, gk: in place)."""
        hq, hk = self._heads("q", q), self._heads("k", k)
        hgq, hgk = self._heads("gq", gq, q), self._heads("gk", gk, k)
        if (gk is None) != (k is None):
            raise ValueError("gk and k go together")
        shape = self._shape(q, k, positions)
        s = _stream(self.device, stream, out is not None)
        if out is None:
            out = (torch.empty(q.shape, dtype=q.dtype, device=self.device),
                   None if k is None else torch.empty(k.shape, dtype=k.dtype, device=self.device),
                   None if wq is None else torch.empty_like(wq), None if wk is None else torch.empty_like(wk))
        dq, dk, dwq, dwk = out
        if (dk is None) != (k is None):
            raise ValueError("out must have a tensor for k where there is one")
        native.dion_qknorm_backward(self.handle, shape, hgq, hgk, hq, hk, self._weight("wq", wq), self._weight("wk", wk),
                                    self._heads("out[0]", dq, q), self._heads("out[1]", dk, k),
                                    self._weight("out[2]", dwq), self._weight("out[3]", dwk), s)
        return dq, dk, dwq, dwk

    def close(self) -> None:
        if getattr(self, "handle", None):
            native.dion_qknorm_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _distill(logits, ids, teacher, temperature, labels, hard, weights):
    if not logits.is_cuda:
        raise ValueError("logits must be on a GPU")
    dev = logits.device
    code, ld = _rows("logits", logits, dev)
    rows, vocab = logits.shape
    a = native.dion_distill(rows, vocab, 0, logits.data_ptr(), ld)
    a.dtype, a.temperature, a.hard = code, temperature, hard
    if ids is not None or teacher is not None:
        if ids is None or teacher is None or ids.shape != teacher.shape or ids.dim() != 2 or ids.shape[0] != rows:
            raise ValueError("ids and teacher must both be [rows, top]")
        a.id_dtype, a.top = _indices("ids", ids, dev), ids.shape[1]
        if a.top > 1 and ids.stride(1) != 1:
            raise ValueError("ids must be row-major")
        a.teacher_dtype, a.ld_teacher = _rows("teacher", teacher, dev)
        a.ids, a.ld_ids, a.teacher = ids.data_ptr(), max(ids.stride(0), a.top), teacher.data_ptr()
    elif hard < 1:
        raise ValueError("ids and teacher are needed unless hard is 1")
    if labels is not None:
        a.label_dtype = _indices("labels", labels, dev)
        if tuple(labels.shape) != (rows,) or (rows > 1 and labels.stride(0) != 1):
            raise ValueError("labels must be a contiguous tensor [rows]")
        a.labels = labels.data_ptr()
    if weights is not None:
        if weights.dtype != torch.float32 or weights.device != dev or tuple(weights.shape) != (rows,) or \
                (rows > 1 and weights.stride(0) != 1):
            raise ValueError("weights must be a contiguous float32 tensor [rows]")
        a.weights = weights.data_ptr()
    return a


def _loss_out(out, rows: int, dev):
    if out is None:
        return torch.empty(rows, dtype=torch.float32, device=dev)
    if out.dtype != torch.float32 or out.device != dev or tuple(out.shape) != (rows,) or (rows > 1 and out.stride(0) != 1):
        raise ValueError("the loss must be a contiguous float32 tensor [rows]")
    return out


def distill_loss(logits, ids, teacher, temperature: float = 1.0, labels=None, hard: float = 0.0, weights=None, out=None,
                 stream: Optional[int] = None):
    """Per row, weights[i] * ((1 - hard) * temperature^2 * KL(teacher || student) - hard * log q1[labels[i]]), float32:
    the teacher's softmax over its top entries `ids`, `teacher` ([rows, top], ids below 0 absent) against the
    student's softmax over `logits` ([rows, vocab], float32 or bfloat16), both at `temperature`; q1 at 1."""
    a = _distill(logits, ids, teacher, temperature, labels, hard, weights)
    dev = logits.device
    s = _stream(dev, stream, out is not None)
    loss = _loss_out(out, a.rows, dev)
    with torch.cuda.device(dev):
        native.dion_distill_loss(a, loss.data_ptr(), s)
    return loss


def distill_loss_grad(logits, ids, teacher, temperature: float = 1.0, labels=None, hard: float = 0.0, weights=None,
                      out=None, stream: Optional[int] = None):
    """(distill_loss, its gradient with respect to the logits, of their dtype).  `out`: the pair to write
    into; the gradient may take the logits' place."""
    a = _distill(logits, ids, teacher, temperature, labels, hard, weights)
    dev = logits.device
    s = _stream(dev, stream, out is not None)
    loss, grad = out if out is not None else (None, torch.empty(logits.shape, dtype=logits.dtype, device=dev))
    if grad.dtype != logits.dtype or grad.shape != logits.shape:
        raise ValueError("the gradient must have the logits' shape and dtype")
    loss = _loss_out(loss, a.rows, dev)
    ldg = _rows("the gradient", grad, dev)[1]
    with torch.cuda.device(dev):
        native.dion_distill_loss_grad(a, loss.data_ptr(), grad.data_ptr(), ldg, s)
    return loss, grad
