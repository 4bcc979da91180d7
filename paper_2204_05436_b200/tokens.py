"""A token embedding: buffers and calls around hl_token_* (plumbing only: torch for memory and streams)."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .experts import _count, _matrix, _written


class TokenEmbedding:
    """Rows of tokens and the gradient of their table, for tables of ``n_rows`` rows of ``dim`` values that the caller holds.

        embedding = TokenEmbedding(max_tokens, n_rows, dim)
        x = embedding.embed(table, tokens, scale)            # [tokens, dim]: scale * table[tokens], zeros for -1
        ...
        embedding.sort(tokens)                               # at any time before the next line, on its stream
        grad = embedding.backward(grad_x, scale)             # [n_rows, dim], summed over the tokens of a row

    The order that sort() makes and the workspace are its own: sort and backward belong in the order of one stream, and two streams
    (or two graphs replayed side by side) need an embedding each.  embed() takes neither."""

    def __init__(self, max_tokens: int, n_rows: int, dim: int, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("the Hotline library needs a CUDA device (there is no CPU fallback)")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.max_tokens, self.n_rows, self.dim = int(max_tokens), int(n_rows), int(dim)
        if not (0 <= self.max_tokens < 2 ** 30 and 0 <= self.n_rows < 2 ** 31 and 1 <= self.dim <= 2 ** 22):
            raise ValueError("less than 2^30 tokens, less than 2^31 rows, of 1 to 2^22 values")
        i32 = dict(dtype=torch.int32, device=self.device)
        self.sorted, self.order = torch.zeros(self.max_tokens, **i32), torch.zeros(self.max_tokens, **i32)
        self._status = torch.zeros(1, **i32)
        self._ws_bytes = B.hl_token_workspace_bytes(self.max_tokens, self.dim)
        self._ws = torch.empty(self._ws_bytes, dtype=torch.uint8, device=self.device)
        self.tokens: Optional[int] = None                    # of the last sort()
        self.n_tokens: Optional[torch.Tensor] = None

    def _call(self, f, *a) -> None:
        with torch.cuda.device(self.device):
            f(*a, torch.cuda.current_stream(self.device).cuda_stream)

    def _tokens(self, tokens: torch.Tensor, n_tokens: Optional[torch.Tensor], most: int) -> None:
        if tokens.device != self.device or tokens.dtype != torch.int32 or tokens.dim() != 1 or not tokens.is_contiguous() or (
                tokens.numel() > most):
            raise ValueError(f"tokens is a contiguous int32 [n] on {self.device}, n at most {most}")
        _count("n_tokens", n_tokens, self.device)

    def embed(self, table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0, n_tokens: Optional[torch.Tensor] = None,
              out: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
        """``n_tokens`` (int32 [1], on the device): how many tokens there are; rows behind them are left as they are in ``out`` (zeros
        without it).  ``dtype``: of the result, the table's by default."""
        ld = _matrix("table", table, self.device, self.n_rows, self.dim)
        self._tokens(tokens, n_tokens, 2 ** 30 - 1)
        n = tokens.numel()
        if out is None:
            out = torch.zeros(n, self.dim, dtype=table.dtype if dtype is None else dtype, device=self.device)
        ld_out = _matrix("out", out, self.device, n, self.dim, dtype)
        _written(out, ld_out, table, tokens, n_tokens)
        self._call(B.hl_token_embed, B.dtype_of(table), self.n_rows, self.dim, table, ld, tokens, n, n_tokens, scale, B.dtype_of(out), out,
                   ld_out, self._status)
        return out

    def sort(self, tokens: torch.Tensor, n_tokens: Optional[torch.Tensor] = None) -> None:
        """Puts the tokens in the order of their rows, for backward() (which reads ``n_tokens`` too)."""
        self._tokens(tokens, n_tokens, self.max_tokens)
        for own in (self.sorted, self.order):
            _written(own, own.numel(), tokens, n_tokens)
        self.tokens, self.n_tokens = tokens.numel(), n_tokens
        self._call(B.hl_token_sort, tokens, self.tokens, n_tokens, self.n_rows, self.sorted, self.order, self._status, self._ws,
                   self._ws_bytes)

    def backward(self, grad_out: torch.Tensor, scale: float = 1.0, grad_table: Optional[torch.Tensor] = None,
                 accumulate: bool = False, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """The gradient of the table from that of the sorted tokens' rows: zeros in rows without tokens, or, with ``accumulate``, added to
        ``grad_table``.  ``dtype``: of the result, where there is no grad_table."""
        if self.tokens is None:
            raise RuntimeError("sort() first")
        ld = _matrix("grad_out", grad_out, self.device, self.tokens, self.dim)
        if grad_table is None:
            if accumulate:
                raise ValueError("accumulate needs the grad_table to add to")
            grad_table = torch.empty(self.n_rows, self.dim, dtype=dtype, device=self.device)
        ld_table = _matrix("grad_table", grad_table, self.device, self.n_rows, self.dim)
        _written(grad_table, ld_table, grad_out, self.n_tokens, self.sorted, self.order)
        self._call(B.hl_token_embed_bwd, self.n_rows, self.dim, self.sorted, self.order, self.tokens, self.n_tokens, B.dtype_of(grad_out),
                   grad_out, ld, scale, B.dtype_of(grad_table), grad_table, ld_table, accumulate, self._ws, self._ws_bytes)
        return grad_table

    def status(self, raise_on_error: bool = True) -> int:
        """Waits for the device: HL_OK, or HL_EBOUNDS if a token was no row and not -1 (zeros, no gradient) since the last call."""
        torch.cuda.synchronize(self.device)
        st = int(self._status.item())
        self._status.zero_()
        torch.cuda.current_stream(self.device).synchronize()     # (before a call on another stream may set it)
        if raise_on_error:
            B._check("hl_token_embed", st)
        return st
