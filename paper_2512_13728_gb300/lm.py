"""Language-model operators over torch CUDA tensors: argument checks and marshalling only.

``EmbedPlan``: token embedding with scaling, and its gradient by sorted tokens.

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
