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


def _count(name: str, n_tokens: Optional[torch.Tensor], device: torch.device) -> None:
    if n_tokens is not None and (n_tokens.device != device or n_tokens.dtype != torch.int32 or n_tokens.numel() < 1):
        raise ValueError(f"{name} is an int32 on {device}")


def _matrix(name: str, t: torch.Tensor, device: torch.device, rows: Optional[int] = None, dim: Optional[int] = None, dtype=None) -> int:
    """Checks a matrix of rows whose values lie side by side; returns the values from one row's begin to the next."""
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    B.dtype_of(t)
    if t.dim() != 2 or t.shape[1] < 1 or (rows is not None and t.shape[0] != rows) or (dim is not None and t.shape[1] != dim) or (
            dtype is not None and t.dtype != dtype):
        raise ValueError(f"{name} is [{'rows' if rows is None else rows}, {'dim' if dim is None else dim}]"
                         f"{'' if dtype is None else f' of {dtype}'}, not {tuple(t.shape)} of {t.dtype}")
    ld = t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])
    if (t.shape[1] > 1 and t.stride(1) != 1) or ld < t.shape[1]:
        raise ValueError(f"the values of a row of {name} lie side by side, and rows do not overlap")
    return ld


def _side_by_side(name: str, t: torch.Tensor, device: torch.device, shape, dtype) -> None:
    if t.device != device or t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} is a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")


def _written(written: torch.Tensor, ld: int, *read: Optional[torch.Tensor]) -> None:
    """What is written (a matrix) shares no byte with what is read."""
    t = written if written.dim() == 2 else written.view(1, -1)
    for r in read:
        if r is not None:
            m = r if r.dim() == 2 else r.reshape(1, -1)
            ExpertRoute._apart(_span(t, t.shape[0], ld), _span(m, m.shape[0], m.stride(0) if m.shape[0] > 1 else m.shape[1]))


class ExpertRouter:
    """A router's choice: logits -> (experts, weights), as :class:`ExpertRoute` takes them, and the logits' gradient.

        router = ExpertRouter(top_k=8, n_experts=256, score="sigmoid", n_groups=8, top_groups=4, group_score="top2", scale=2.5)
        experts, weights = router.choose(logits, bias)       # int32, fp32 [tokens, top_k]
        route.sort(experts); ...; grad_y, grad_weights = route.combine_backward(grad_out, y, weights)
        grad_logits = router.backward(logits, experts, grad_weights)

    ``score``: "softmax" or "sigmoid"; ``n_groups`` groups of experts side by side, of which the ``top_groups`` best are kept (a group
    counts with its best expert, "max", or with the sum of its two best, "top2"); ``renorm``: the chosen scores are divided by their
    sum; ``scale``: of the weights.  A router has no buffers of its own but a status word: its calls may be made on any streams."""

    def __init__(self, top_k: int, n_experts: int, score: str = "softmax", n_groups: int = 1, top_groups: int = 1,
                 group_score: str = "max", renorm: bool = True, scale: float = 1.0, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("the Hotline library needs a CUDA device (there is no CPU fallback)")
        scores, groups = {"softmax": B.HL_SCORE_SOFTMAX, "sigmoid": B.HL_SCORE_SIGMOID}, {"max": B.HL_GROUP_MAX, "top2": B.HL_GROUP_TOP2}
        if score not in scores or group_score not in groups:
            raise ValueError("score is softmax or sigmoid, group_score max or top2")
        if not (1 <= n_experts <= B.HL_MAX_EXPERTS and 1 <= top_k <= min(n_experts, B.HL_MAX_TOP_K) and 1 <= n_groups <= B.HL_MAX_GROUPS
                and n_experts % n_groups == 0 and 1 <= top_groups <= n_groups and top_k <= n_experts // n_groups * top_groups
                and math.isfinite(scale)):
            raise ValueError(f"1 to {B.HL_MAX_TOP_K} of 1 to {B.HL_MAX_EXPERTS} experts, in 1 to {B.HL_MAX_GROUPS} groups of one size, "
                             "the kept ones of which have top_k; a finite scale")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.top_k, self.n_experts = int(top_k), int(n_experts)
        self._router = B.make_router(scores[score], top_k, n_experts, n_groups, top_groups, groups[group_score], renorm, scale)
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)

    def choose(self, logits: torch.Tensor, bias: Optional[torch.Tensor] = None, n_tokens: Optional[torch.Tensor] = None,
               out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """``bias`` (fp32 [n_experts]): added to the scores for the choice, not to the weights.  ``n_tokens`` (int32 [1], on the device):
        how many tokens there are; those behind them are left as they are in ``out`` (-1 and 0 without it)."""
        ld, tokens = _matrix("logits", logits, self.device, dim=self.n_experts), logits.shape[0]
        _count("n_tokens", n_tokens, self.device)
        if bias is not None:
            _side_by_side("bias", bias, self.device, (self.n_experts,), torch.float32)
        if out is None:
            experts = torch.full((tokens, self.top_k), -1, dtype=torch.int32, device=self.device)
            weights = torch.zeros(tokens, self.top_k, dtype=torch.float32, device=self.device)
        else:
            experts, weights = out
            _side_by_side("experts", experts, self.device, (tokens, self.top_k), torch.int32)
            _side_by_side("weights", weights, self.device, (tokens, self.top_k), torch.float32)
            _written(experts, self.top_k, logits, bias, weights, n_tokens)
            _written(weights, self.top_k, logits, bias, n_tokens)
        with torch.cuda.device(self.device):
            B.hl_expert_choose(self._router, B.dtype_of(logits), logits, ld, bias, tokens, n_tokens, experts, weights, self._status,
                               torch.cuda.current_stream(self.device).cuda_stream)
        return experts, weights

    def backward(self, logits: torch.Tensor, experts: torch.Tensor, grad_weights: torch.Tensor,
                 n_tokens: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The logits' gradient, from choose's logits and experts (rows behind the last token: as in ``out``, or zeros)."""
        ld, tokens = _matrix("logits", logits, self.device, dim=self.n_experts), logits.shape[0]
        _count("n_tokens", n_tokens, self.device)
        _side_by_side("experts", experts, self.device, (tokens, self.top_k), torch.int32)
        _side_by_side("grad_weights", grad_weights, self.device, (tokens, self.top_k), torch.float32)
        if out is None:
            out = torch.zeros(tokens, self.n_experts, dtype=logits.dtype, device=self.device)
        ld_out = _matrix("out", out, self.device, tokens, self.n_experts, logits.dtype)
        _written(out, ld_out, logits, experts, grad_weights, n_tokens)
        with torch.cuda.device(self.device):
            B.hl_expert_choose_bwd(self._router, B.dtype_of(logits), logits, ld, tokens, n_tokens, experts, grad_weights, out, ld_out,
                                   torch.cuda.current_stream(self.device).cuda_stream)
        return out

    def status(self, raise_on_error: bool = True) -> int:
        """Waits for the device: HL_OK, or HL_EINVAL if a logit or a bias was NaN (that expert was not chosen) since the last call."""
        torch.cuda.synchronize(self.device)
        st = int(self._status.item())
        self._status.zero_()
        torch.cuda.current_stream(self.device).synchronize()     # (before a call on another stream may set it)
        if raise_on_error:
            B._check("hl_expert_choose", st)
        return st


class Mx4Weights:
    """The weights of experts, [n_experts, outputs, dim], in 4 bits (blocks of 32 values of a row share a power of two), and the
    product with them.  For serving: there is no gradient.

        w = Mx4Weights(weights)                              # laid out once
        y = w.product(route, x)                              # x: the tokens' rows; y by expert, as route.dispatch would lay them out
        z = w2.product(route, act(y), by_token=False)        # rows by expert
        out = route.combine(z, weights)

    A product takes the workspace of its own matrix: products with one Mx4Weights belong in the order of one stream."""

    def __init__(self, weights: torch.Tensor):
        if not torch.cuda.is_available():
            raise RuntimeError("the Hotline library needs a CUDA device (there is no CPU fallback)")
        if weights.dim() != 3 or not weights.is_cuda or not 1 <= weights.shape[0] <= B.HL_MAX_EXPERTS or not weights.is_contiguous() or (
                weights.shape[1] < 1 or weights.shape[2] < 1):
            raise ValueError(f"weights is a contiguous [experts, outputs, dim] on a CUDA device, of 1 to {B.HL_MAX_EXPERTS} experts")
        self.device = weights.device
        self.n_experts, self.outputs, self.dim = weights.shape
        self._q = torch.empty(self.n_experts * B.hl_mx4_bytes(self.outputs, self.dim), dtype=torch.uint8, device=self.device)
        self._ws: list = []                                  # the last is the largest; a captured graph may hold on to any
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)       # of all products, with any of them
        self._call(B.hl_mx4_quantise, B.dtype_of(weights), self.n_experts, self.outputs, self.dim, weights, self.dim,
                   self.outputs * self.dim, self._q)

    def _call(self, f, *a) -> None:
        with torch.cuda.device(self.device):
            f(*a, torch.cuda.current_stream(self.device).cuda_stream)

    def dequantise(self, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        out = torch.empty(self.n_experts, self.outputs, self.dim, dtype=dtype, device=self.device)
        self._call(B.hl_mx4_dequantise, self.n_experts, self.outputs, self.dim, self._q, B.dtype_of(out), out, self.dim,
                   self.outputs * self.dim)
        return out

    def product(self, route: ExpertRoute, x: torch.Tensor, by_token: bool = True, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Rows by expert times their expert's weights, both in 4 bits, added up in fp32.  ``by_token``: x has the rows of the route's
        tokens, which go to their experts on the way; else the experts' rows.  Rows that fill an expert up become zeros, rows
        behind the last expert's stay as they are in ``out`` (zeros without it)."""
        if route.device != self.device or route.n_experts != self.n_experts:
            raise ValueError(f"the route is of {route.n_experts} experts on {route.device}, the weights of {self.n_experts} on {self.device}")
        ld = _matrix("x", x, self.device, route.tokens if by_token else route.cap_rows, self.dim)
        if out is None:
            out = torch.zeros(route.cap_rows, self.outputs, dtype=x.dtype, device=self.device)
        ld_out = _matrix("out", out, self.device, route.cap_rows, self.outputs, x.dtype)
        _written(out, ld_out, x)
        need = B.hl_expert_mx4_workspace_bytes(route.cap_rows, self.n_experts, self.dim)
        if not self._ws or self._ws[-1].numel() < need:
            self._ws.append(torch.zeros(need, dtype=torch.uint8, device=self.device))
        self._call(B.hl_expert_mx4_checked, route._route, B.dtype_of(x), self.dim, self.outputs, x, ld, by_token, self._q, out, ld_out,
                   self._ws[-1], self._ws[-1].numel(), self._status)
        return out

    def status(self, raise_on_error: bool = True) -> int:
        """Waits for the device: HL_OK, or HL_ETIMEOUT if a wait inside any product since the last call gave up."""
        torch.cuda.synchronize(self.device)
        st = int(self._status.item())
        self._status.zero_()
        torch.cuda.current_stream(self.device).synchronize()     # (before a call on another stream may set it)
        if raise_on_error:
            B._check("hl_expert_mx4", st)
        return st
