"""A mixture of experts' routing: buffers and calls around hl_expert_* (plumbing only: torch for memory and streams).

:class:`ExpertRoute` keeps the plan that one router's choices make -- where every token's rows lie among the experts' -- and issues
the copies there, the weighted sums back and their gradients, on torch's current stream.  No arithmetic happens here.  A route's
plan and workspace are its own: its calls belong in the order of one stream, and two streams (or two graphs replayed side by side)
need a route each.

    route = ExpertRoute(max_tokens, top_k, n_experts, align=128)
    route.sort(experts)                              # int32 [tokens, top_k], -1: no expert; tokens <= max_tokens
    y = route.dispatch(x)                            # rows by expert: expert e's are offsets[e] .. offsets[e] + counts[e]
    ...                                              # the experts, on route.counts / route.offsets
    out = route.combine(y, weights)
    grad_y, grad_weights = route.combine_backward(grad_out, y, weights)
    ...
    grad_x = route.dispatch_backward(grad_y)
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch

from . import binding as B


def _share(a: torch.Tensor, b: torch.Tensor) -> bool:
    """Whether two matrices, rows of values side by side, have a byte in common."""
    if not a.numel() or not b.numel():
        return False
    if a.shape[0] > b.shape[0]:
        a, b = b, a
    (p, w, step, n), (q, v, other, m) = ((t.data_ptr(), t.shape[1] * t.element_size(), t.stride(0) * t.element_size() if t.shape[0] > 1
                                          else 0, t.shape[0]) for t in (a, b))
    # columns of one buffer: rows begin in different places of every step
    g = math.gcd(step, other)
    if g and w <= (q - p) % g <= g - v:
        return False
    # of b's rows, those that a row of a may touch: the last that begins before it or with it, and the next
    begin = p + step * torch.arange(n, device="cpu")
    before = torch.div(begin - q, max(other, 1), rounding_mode="floor")
    rows = (q + other * (before + k).clamp(0, m - 1) for k in (0, 1))
    return any(bool(((row < begin + w) & (begin < row + v)).any()) for row in rows)


def _span(t: Optional[torch.Tensor], rows: int, ld: int):
    """A matrix with its first byte and the one behind its last (None: none)."""
    if t is None:
        return None, 0, 0
    p = t.data_ptr()
    return t, p, p + ((rows - 1) * ld + t.shape[1]) * t.element_size()


class ExpertRoute:
    def __init__(self, max_tokens: int, top_k: int, n_experts: int, align: int = 1, cap_rows: Optional[int] = None,
                 device: str = "cuda:0"):
        """``align``: an expert's rows are filled up (with zeros) to a multiple of it.  ``cap_rows``: rows of the expert-ordered
        buffers; by default as many as any choices need."""
        if not torch.cuda.is_available():
            raise RuntimeError("the Hotline library needs a CUDA device (there is no CPU fallback)")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.max_tokens, self.top_k, self.n_experts, self.align = int(max_tokens), int(top_k), int(n_experts), int(align)
        if not (0 <= self.max_tokens and 1 <= self.top_k <= B.HL_MAX_TOP_K and 1 <= self.n_experts <= B.HL_MAX_EXPERTS
                and self.max_tokens * self.top_k < 2 ** 30 and 1 <= self.align <= 65536):
            raise ValueError(f"1 to {B.HL_MAX_TOP_K} choices a token of 1 to {B.HL_MAX_EXPERTS} experts, less than 2^30 of them, "
                             "align 1 to 65536")
        n = self.max_tokens * self.top_k
        self.cap_rows = n + min(self.n_experts, n) * (self.align - 1) if cap_rows is None else int(cap_rows)
        if self.cap_rows < 0:
            raise ValueError("cap_rows is not negative")
        i32 = dict(dtype=torch.int32, device=self.device)
        self.place = torch.full((self.max_tokens, self.top_k), -1, **i32)
        self.source = torch.full((self.cap_rows,), -1, **i32)
        self.counts = torch.zeros(self.n_experts, **i32)
        self.offsets = torch.zeros(self.n_experts + 1, **i32)
        self._status = torch.zeros(1, **i32)
        self._sorted_on: Optional[torch.cuda.Stream] = None
        self._ws_bytes = B.hl_expert_workspace_bytes(self.max_tokens, self.top_k, self.n_experts)
        self._ws = torch.empty(self._ws_bytes, dtype=torch.uint8, device=self.device)
        self._set(self.max_tokens, None)

    def _set(self, tokens: int, n_tokens: Optional[torch.Tensor]) -> None:
        self.tokens, self.n_tokens = tokens, n_tokens
        self._route = B.make_route(tokens, n_tokens, self.top_k, self.n_experts, self.align, self.cap_rows, self.place, self.source,
                                   self.counts, self.offsets)

    def _call(self, f, *a) -> torch.cuda.Stream:
        with torch.cuda.device(self.device):
            stream = torch.cuda.current_stream(self.device)
            f(*a, stream.cuda_stream)
        return stream

    def _here(self, name: str, t: torch.Tensor) -> None:
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the route on {self.device}")

    def _tensor(self, name: str, t: torch.Tensor, shape, dtype) -> None:
        self._here(name, t)
        if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
            raise ValueError(f"{name} is a contiguous {dtype} tensor of shape {tuple(shape)}, not {t.dtype} of {tuple(t.shape)}")

    def _rows(self, name: str, t: torch.Tensor, rows: int, like: Optional[torch.Tensor] = None) -> int:
        """Checks a matrix of rows; returns the values from one row's begin to the next."""
        self._here(name, t)
        B.dtype_of(t)
        if t.dim() != 2 or t.shape[0] != rows or t.shape[1] < 1:
            raise ValueError(f"{name} has {rows} rows, not the shape {tuple(t.shape)}")
        if like is not None and (t.dtype != like.dtype or t.shape[1] != like.shape[1]):
            raise ValueError(f"{name} has rows of {like.shape[1]} {like.dtype}, not of {t.shape[1]} {t.dtype}")
        ld = t.stride(0) if rows > 1 else max(t.stride(0), t.shape[1])
        if (t.shape[1] > 1 and t.stride(1) != 1) or ld < t.shape[1]:
            raise ValueError(f"the values of a row of {name} lie side by side, and rows do not overlap")
        return ld

    @staticmethod
    def _apart(written, *others) -> None:
        """Of _span()s."""
        t, begin, end = written
        for o, p, q in others:
            if begin < q and p < end and _share(t, o):
                raise ValueError("what is written shares nothing with what else is read or written")

    def sort(self, experts: torch.Tensor, n_tokens: Optional[torch.Tensor] = None, expert_cap: int = 0) -> None:
        """Makes the plan from the router's choices, int32 [tokens, top_k] with at most max_tokens tokens.  ``n_tokens`` (int32 [1],
        on the device): how many of them there are (hl_fragment's counts, say); the tensor is read by all later calls too, and
        what belongs to the tokens behind them is left alone.  ``expert_cap`` > 0: most choices of an expert; later ones get no
        row."""
        if experts.dim() != 2 or not 0 <= experts.shape[0] <= self.max_tokens:
            raise ValueError(f"experts is [tokens, {self.top_k}] with at most {self.max_tokens} tokens")
        self._tensor("experts", experts, (experts.shape[0], self.top_k), torch.int32)
        if n_tokens is not None:
            self._here("n_tokens", n_tokens)
            if n_tokens.dtype != torch.int32 or n_tokens.numel() < 1:
                raise ValueError("n_tokens is an int32")
        if int(expert_cap) < 0:
            raise ValueError("expert_cap is not negative")
        begin, size = experts.data_ptr(), 4 * experts.numel()
        for own in (self.place, self.source):
            p = own.data_ptr()
            if begin < p + 4 * own.numel() and p < begin + size:
                raise ValueError("what is written shares nothing with what else is read or written")
        self._set(experts.shape[0], n_tokens)
        self._sorted_on = self._call(B.hl_expert_sort, self._route, experts, int(expert_cap), self._status, self._ws,
                                     self._ws_bytes)

    def status(self, raise_on_error: bool = True) -> int:
        """Waits for the last sort: HL_OK, HL_EBOUNDS (an id that is no expert's: counted as -1) or HL_ECAPACITY (cap_rows too small
        for the experts' rows, those that fill them up among them: the choices behind it have no row).  The sort may have been
        queued on any stream; one that is replayed with a graph, on the current one."""
        if self._sorted_on is not None:
            torch.cuda.current_stream(self.device).wait_stream(self._sorted_on)
        st = int(self._status.item())
        if raise_on_error:
            B._check("hl_expert_sort", st)
        return st

    def dispatch(self, x: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """y[place[t, k]] = x[t]; zeros in the rows that fill an expert up; rows behind the last expert's stay as they are in
        ``out`` (zeros without it)."""
        ld = self._rows("x", x, self.tokens)
        if out is None:
            out = torch.zeros(self.cap_rows, x.shape[1], dtype=x.dtype, device=x.device)
        ld_out = self._rows("out", out, self.cap_rows, x)
        self._apart(_span(out, self.cap_rows, ld_out), _span(x, self.tokens, ld))
        self._call(B.hl_expert_dispatch, self._route, B.dtype_of(x), x.shape[1], x, ld, out, ld_out)
        return out

    def dispatch_backward(self, grad_y: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The gradient of dispatch's x: the sum of each token's rows."""
        return self.combine(grad_y, None, out)

    def combine(self, y: torch.Tensor, weights: Optional[torch.Tensor], out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """out[t] = sum of weights[t, k] * y[place[t, k]] (fp32 weights [tokens, top_k]; None: the plain sum)."""
        ld = self._rows("y", y, self.cap_rows)
        if weights is not None:
            self._tensor("weights", weights, (self.tokens, self.top_k), torch.float32)
        if out is None:
            out = torch.zeros(self.tokens, y.shape[1], dtype=y.dtype, device=y.device)
        ld_out = self._rows("out", out, self.tokens, y)
        self._apart(_span(out, self.tokens, ld_out), _span(y, self.cap_rows, ld), _span(weights, self.tokens, self.top_k))
        self._call(B.hl_expert_combine, self._route, B.dtype_of(y), y.shape[1], y, ld, weights, out, ld_out)
        return out

    def combine_backward(self, grad_out: torch.Tensor, y: Optional[torch.Tensor], weights: Optional[torch.Tensor],
                         grad_y: Optional[torch.Tensor] = None,
                         grad_weights: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """The gradients of combine's y and weights (of y alone where y is None: it is not needed for that)."""
        ld_go = self._rows("grad_out", grad_out, self.tokens)
        ld_y = 0 if y is None else self._rows("y", y, self.cap_rows, grad_out)
        if weights is not None:
            self._tensor("weights", weights, (self.tokens, self.top_k), torch.float32)
        if grad_y is None:
            grad_y = torch.zeros(self.cap_rows, grad_out.shape[1], dtype=grad_out.dtype, device=grad_out.device)
        ld_gy = self._rows("grad_y", grad_y, self.cap_rows, grad_out)
        if y is None:
            if grad_weights is not None:
                raise ValueError("the gradient of the weights needs y")
        elif grad_weights is None:
            grad_weights = torch.zeros(self.tokens, self.top_k, dtype=torch.float32, device=grad_out.device)
        else:
            self._tensor("grad_weights", grad_weights, (self.tokens, self.top_k), torch.float32)
        w, gw = _span(weights, self.tokens, self.top_k), _span(grad_weights, self.tokens, self.top_k)
        read = _span(grad_out, self.tokens, ld_go), _span(y, self.cap_rows, ld_y), w
        self._apart(_span(grad_y, self.cap_rows, ld_gy), *read, gw)
        self._apart(gw, *read)
        self._call(B.hl_expert_combine_bwd, self._route, B.dtype_of(grad_out), grad_out.shape[1], grad_out, ld_go, y, ld_y, weights,
                   grad_y, ld_gy, grad_weights)
        return grad_y, grad_weights
