"""The operators between an embedding's pooled rows and its update whose speed counts: tokens sorted by expert and back,
and the global norm of the gradients with clipping.

Kinds of work (``case["kind"]``):

* ``sort``      the expert of every (token, choice) becomes a row of an expert-ordered buffer (hl_expert_sort);
* ``dispatch``  token rows are copied to their experts' rows (hl_expert_dispatch), and in training (``train``) the
                gradients of those copies are summed per token;
* ``combine``   the experts' rows are summed per token with the router's weights (hl_expert_combine), and in training the
                gradients of rows and weights are made (hl_expert_combine_bwd);
* ``clip``      the global norm of many gradient tensors, and every tensor scaled by the clipping factor (hl_grad_clip);
* ``rowclip``   the same where most gradients are an embedding's: the norm is that of the tables' row gradients, in which
                the lookups of a row are added up before they are squared (hl_embbag_grad_sumsq, hl_grad_clip).

``run`` computes them in elementary torch operations where ``own`` is false and calls the library where it is true.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ---- the cases ------------------------------------------------------------------------------------------------------
def _experts(kind, tokens, top_k, experts, live=None, skew=0.0, dropped=0.0, cap=0.0, align=1, dim=0, dtype="f32", pad=0,
             train=False):
    """``tokens``: rows of the buffers, of which the first ``live`` hold tokens (a device-side count, as hl_fragment
    gives it); ``skew``: exponent of the power law that the experts' loads follow; ``dropped``: share of the choices that
    name no expert; ``cap``: most rows of an expert, as a multiple of an even share (0: any); ``align``: an expert's rows
    are filled up to a multiple of it; ``pad``: values between the end of a row and the next."""
    return dict(kind=kind, tokens=tokens, top_k=top_k, experts=experts, live=tokens if live is None else live, skew=skew,
                dropped=dropped, cap=cap, align=align, dim=dim, dtype=dtype, pad=pad, train=train)


def _clip(tensors, smallest, largest, src="f32", dst="f32", step=8, in_place=False, factor=0.5):
    """``tensors`` of ``smallest`` to ``largest`` values, which begin at multiples of ``step`` values of one buffer;
    ``in_place``: the tensors themselves are scaled, and are already short enough; ``factor``: what clipping scales by."""
    return dict(kind="clip", tensors=tensors, smallest=smallest, largest=largest, src=src, dst=dst, step=step,
                in_place=in_place, factor=factor)


def _rowclip(tables, rows, dim, batch, steps=1, bag=1, cap=1, alpha=1.1, dense=100_000):
    """``rows`` of all tables together, ``batch`` inputs with ``steps`` bags per table of exactly one or
    min(Poisson(bag), cap) lookups; ``dense``: values of the dense model's gradient, which is clipped with the tables'."""
    return dict(kind="rowclip", tables=tables, rows=rows, dim=dim, batch=batch, steps=steps, bag=bag, cap=cap, alpha=alpha,
                dense=dense)


def listed():
    cases = {
        # serving one input at a time: two of eight experts
        "sort one token": _experts("sort", 1, 2, 8),
        # a training mini-batch of 16,384 inputs, of which the popular 36 % are routed, tiles of 128 rows for the products
        "sort popular inputs": _experts("sort", 16384, 4, 64, live=5899, skew=0.7, align=128),
        # many small experts, long packed input, uneven loads, a capacity of 1.25 even shares
        "sort large": _experts("sort", 262_144, 8, 256, skew=0.9, dropped=0.05, cap=1.25, align=16),
        # a few requests: pooled vectors of 26 tables x 64 to their experts
        "dispatch few": _experts("dispatch", 4, 2, 8, dim=1664, dtype="bf16"),
        # the pooled vectors of a training mini-batch (26 tables x 64, fp32) and their gradient
        "dispatch train": _experts("dispatch", 16384, 2, 16, skew=0.5, align=64, dim=1664, dtype="f32", train=True),
        # back from the experts for a few requests
        "combine few": _experts("combine", 4, 2, 8, dim=1664, dtype="bf16"),
        # many tokens, eight of 64 experts, bf16, forward and backward
        "combine train": _experts("combine", 16384, 8, 64, skew=0.7, align=128, dim=2048, dtype="bf16", train=True),
        # ragged: 21 tables x 16 and one dense feature (a row of 337 values), padded batch, dropped tokens
        "combine ragged": _experts("combine", 30_011, 3, 37, live=28_657, skew=0.7, dropped=0.1, dim=337, dtype="f16",
                                   pad=2, train=True),
        # the gradients of a dense model of a few layers
        "clip few": _clip(14, 64, 300_000),
        # a large model's gradients in bf16, scaled into the fp32 buffer that its update reads
        "clip many": _clip(420, 500, 4_000_000, src="bf16", dst="f32", step=1),
        # the benchmark's mini-batch: 26 tables, dim 64, 16,384 inputs
        "rowclip large": _rowclip(26, 7_725_000, 64, 16384, alpha=1.2, dense=800_000),
        # a time-series model: 21 steps x 3 tables, dim 16; rows looked up many times
        "rowclip time series": _rowclip(3, 5_010_000, 16, 2048, steps=21, alpha=1.2),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["sort", "sort", "dispatch", "dispatch", "combine", "combine", "clip", "clip", "rowclip", "rowclip"])
    if kind == "clip":
        tensors = _log_int(rng, 1, 1500)
        largest = _log_int(rng, 1000, 4_000_000)
        largest = max(100, min(largest, 200_000_000 // tensors))
        in_place = rng.random() < 0.3
        src = rng.choice(["f32", "bf16", "f16"])
        dst = src if in_place else rng.choice(["f32", "f32", src])
        return _clip(tensors, rng.randint(1, min(largest, 700)), largest, src, dst, rng.choice([1, 8, 64]), in_place,
                     round(rng.uniform(0.05, 0.95), 3))
    if kind == "rowclip":
        dim = 4 * _log_int(rng, 2, 32)
        tables = _log_int(rng, 1, 40)
        bag, cap, steps = rng.choice([(1, 1, 1), (1, 1, 1), (1, 1, rng.randint(2, 21)), (4, 12, 1), (20, 64, 1)])
        batch = _log_int(rng, 16, 16384) | rng.randint(0, 1)
        batch = max(1, min(batch, 25_000_000 // (dim * tables * steps * bag)))
        return _rowclip(tables, _log_int(rng, 1000, 8_000_000), dim, batch, steps, bag, cap,
                        round(rng.uniform(1.05, 1.25), 3), _log_int(rng, 100, 2_000_000))
    top_k = rng.choice([1, 2, 2, 3, 4, 6, 8])
    experts = rng.choice([4, 8, 16, 37, 64, 128, 256, 500])
    tokens = _log_int(rng, 1, 262_144 if kind == "sort" else 65_536)
    dim, dtype = 0, rng.choice(["f32", "bf16", "f16"])
    pad = 0
    if kind != "sort":
        dim = rng.choice([8 * _log_int(rng, 2, 512), _log_int(rng, 10, 4096)])
        pad = rng.choice([0, 0, 8, rng.randint(1, 20)])
        most = 150_000_000 if dtype != "f32" else 75_000_000              # values of the experts' rows
        tokens = max(1, min(tokens, most // (dim * top_k)))
    live = tokens if rng.random() < 0.5 else rng.randint((tokens + 1) // 2, tokens)
    return _experts(kind, tokens, top_k, experts, live, round(rng.uniform(0.0, 1.0), 2), rng.choice([0.0, 0.0, 0.1]),
                    rng.choice([0.0, 0.0, 1.25, 2.0]), rng.choice([1, 1, 16, 100, 128]), dim, dtype, pad,
                    kind != "sort" and rng.random() < 0.6)


# ---- sizes that follow from a case ----------------------------------------------------------------------------------
def _expert_cap(case):
    return math.ceil(case["cap"] * case["live"] * case["top_k"] / case["experts"])


def _row_capacity(case):
    """Rows that hold whatever the router chooses."""
    n = case["tokens"] * case["top_k"]
    return n + min(case["experts"], n) * (case["align"] - 1)


def _tensor_sizes(case):
    r = random.Random(f"{case['tensors']}/{case['smallest']}/{case['largest']}")
    return [_log_int(r, case["smallest"], case["largest"]) for _ in range(case["tensors"])]


def _tensor_starts(case):
    starts, at = [], 0
    for n in _tensor_sizes(case):
        starts.append(at)
        at += -(-n // case["step"]) * case["step"]
    return starts, at


def _mean_lookups(case):
    return case["tables"] * case["batch"] * case["steps"] * case["bag"]


def work(case):
    if case["kind"] == "clip":
        n = sum(_tensor_sizes(case))
        out = 0 if case["in_place"] else SIZE[case["dst"]]
        return {"bytes": n * (SIZE[case["src"]] + out), "flops": 3.0 * n}
    if case["kind"] == "rowclip":
        bags = case["tables"] * case["batch"] * case["steps"]
        lookups = _mean_lookups(case)
        values = bags * case["dim"] + case["dense"]
        return {"bytes": 8 * lookups + 8 * values, "flops": 2.0 * lookups * case["dim"] + 3.0 * values}
    n = case["live"] * case["top_k"]
    if case["kind"] == "sort":
        return {"bytes": 4 * n + 4 * n + 4 * n + 8 * case["experts"], "flops": 4.0 * n}
    kept = n * (1.0 - case["dropped"])
    size, dim, live = SIZE[case["dtype"]], case["dim"], case["live"]
    if case["kind"] == "dispatch":
        one = (live + kept) * dim * size + 4 * n
        return {"bytes": one * (2 if case["train"] else 1), "flops": kept * dim}
    moved = (live + kept) * dim * size + 8 * n
    if case["train"]:
        moved += (live + 2 * kept) * dim * size + 12 * n
    return {"bytes": moved, "flops": (6.0 if case["train"] else 2.0) * kept * dim}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _choices(case, g):
    """int32 [tokens, top_k]: different experts for a token where there are enough, loads by a power law over a random
    order of the experts, -1 where none is chosen."""
    T, K, E = case["tokens"], case["top_k"], case["experts"]
    load = torch.arange(1, E + 1, device=DEVICE, dtype=torch.float32) ** -case["skew"]
    load = load[torch.randperm(E, generator=g, device=DEVICE)]
    noise = torch.rand(T, E, generator=g, device=DEVICE).clamp_(1e-7, 1.0 - 1e-7)
    scores = load.log() - (-noise.log()).log()                 # the largest of these: a draw by the loads
    if K <= E:
        e = scores.topk(K, dim=1).indices
    else:
        e = scores.argmax(dim=1, keepdim=True).expand(T, K)
    e = torch.where(torch.rand(T, K, generator=g, device=DEVICE) < case["dropped"], -1, e)
    return e.to(torch.int32).contiguous()


def _sorted(case, experts):
    """The expert-ordered rows of the live tokens' choices, from the definition: place, source, counts, offsets."""
    T, K, E, align, cap = case["tokens"], case["top_k"], case["experts"], case["align"], _expert_cap(case)
    rows = _row_capacity(case)
    n = case["live"] * K
    e = experts[: case["live"]].reshape(-1).long()
    key = torch.where((e >= 0) & (e < E), e, E)
    order = torch.argsort(key, stable=True)
    ranked = key[order]
    ones = torch.ones_like(key)
    seen = torch.zeros(E + 1, dtype=torch.int64, device=DEVICE).index_add_(0, key, ones)
    first = seen.cumsum(0) - seen
    rank = torch.arange(n, device=DEVICE) - first[ranked]
    counts = seen[:E].clamp(max=cap) if cap else seen[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=DEVICE)
    offsets[1:] = (((counts + align - 1) // align) * align).cumsum(0)
    at = torch.where((ranked < E) & (rank < counts[ranked.clamp(max=E - 1)]), offsets[ranked] + rank, -1)
    place = torch.full((T * K,), -7, dtype=torch.int32, device=DEVICE)       # (behind the live tokens: left as it was)
    place[:n] = torch.empty(n, dtype=torch.int32, device=DEVICE).scatter_(0, order, at.int())
    row = torch.arange(rows + 1, device=DEVICE)
    source = torch.where(row < offsets[E], -1, -7).int()
    source[torch.where(at >= 0, at, rows)] = order.int()                     # (one row more, for what has no place)
    return place.view(T, K), source[:rows], counts.int(), offsets.int()


def _rows(case, g, n):
    """n rows of a buffer with `pad` values between them."""
    t = torch.randn(n, case["dim"] + case["pad"], generator=g, device=DEVICE).to(TYPES[case["dtype"]])
    return t[:, : case["dim"]]


def _empty_rows(case, n):
    return torch.full((n, case["dim"] + case["pad"]), 2.0, dtype=TYPES[case["dtype"]], device=DEVICE)[:, : case["dim"]]


def _prepare_experts(case, seed):
    g = _generator(seed)
    T, K, E, rows = case["tokens"], case["top_k"], case["experts"], _row_capacity(case)
    s = {"case": case, "experts": _choices(case, g)}
    s["n_tokens"] = torch.tensor([case["live"]], dtype=torch.int32, device=DEVICE)
    if case["kind"] == "sort":
        s["place"] = torch.full((T, K), -7, dtype=torch.int32, device=DEVICE)
        s["source"] = torch.full((rows,), -7, dtype=torch.int32, device=DEVICE)
        s["counts"] = torch.zeros(E, dtype=torch.int32, device=DEVICE)
        s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device=DEVICE)
    else:
        s["place"], s["source"], s["counts"], s["offsets"] = _sorted(case, s["experts"])
        s["x"] = _rows(case, g, T)                               # in token order
        s["y"] = _rows(case, g, rows)                            # in expert order
        w = torch.rand(T, K, generator=g, device=DEVICE)
        s["w"] = (w / w.sum(dim=1, keepdim=True)).contiguous()
        s["to_tokens"], s["to_rows"] = _empty_rows(case, T), _empty_rows(case, rows)
        s["grad_w"] = torch.full((T, K), 2.0, device=DEVICE)
    if own:
        import paper_2204_05436_b200 as hl

        s["hl"], s["stream"] = hl, torch.cuda.current_stream().cuda_stream
        s["type"] = hl.dtype_of(s["x"]) if "x" in s else 0
        s["route"] = hl.make_route(T, s["n_tokens"], K, E, case["align"], rows, s["place"], s["source"], s["counts"],
                                   s["offsets"])
        s["ws_bytes"] = hl.hl_expert_workspace_bytes(T, K, E)
        s["ws"] = torch.empty(max(1, s["ws_bytes"]), dtype=torch.uint8, device=DEVICE)
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEVICE)
    return s


def _prepare_clip(case, seed):
    g = _generator(seed)
    starts, total = _tensor_starts(case)
    sizes = _tensor_sizes(case)
    src = torch.randn(total, generator=g, device=DEVICE).mul_(1e-3).to(TYPES[case["src"]])
    inside = torch.zeros(total + 1, dtype=torch.int32, device=DEVICE)
    at = torch.tensor(starts, device=DEVICE)
    one = torch.ones(len(sizes), dtype=torch.int32, device=DEVICE)
    inside.index_add_(0, at, one)
    inside.index_add_(0, at + torch.tensor(sizes, device=DEVICE), -one)
    src *= inside.cumsum(0)[:total].to(src.dtype)                # (nothing between the tensors)
    dst = src if case["in_place"] else torch.zeros(total, dtype=TYPES[case["dst"]], device=DEVICE)
    norm = 1e-3 * math.sqrt(sum(sizes))
    s = {"case": case, "src": src, "dst": dst, "norm": torch.zeros(1, device=DEVICE)}
    s["max_norm"] = norm * (1.1 if case["in_place"] else case["factor"])
    if case["in_place"]:
        s["max_norm"] += 1.0
    if own:
        import paper_2204_05436_b200 as hl

        s["hl"], s["stream"] = hl, torch.cuda.current_stream().cuda_stream
        s["tensors"] = hl.make_tensors([(src[a:a + n], dst[a:a + n]) for a, n in zip(starts, sizes)])
        s["ws_bytes"] = hl.hl_grad_workspace_bytes()
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEVICE)
    return s


def _prepare_rowclip(case, seed):
    """Lookups as a data loader gives them, the popular rows of every table many times; their (row, bag) pairs sorted by
    row, as hl_embbag_bwd_prepare leaves them."""
    g = _generator(seed)
    T, D = case["tables"], case["dim"]
    bags = T * case["batch"] * case["steps"]
    if case["bag"] == 1:
        size = torch.ones(bags, dtype=torch.int64, device=DEVICE)
    else:
        mean = torch.full((bags,), float(case["bag"]), device=DEVICE)
        size = torch.poisson(mean, generator=g).long().clamp(max=case["cap"])
    bag = torch.repeat_interleave(torch.arange(bags, device=DEVICE), size)
    n = bag.numel()
    per_table = max(1, case["rows"] // T)
    u = torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64)
    tail = per_table ** (1.0 - case["alpha"])                    # a power law over [1, per_table]
    rank = ((1.0 - u * (1.0 - tail)) ** (1.0 / (1.0 - case["alpha"])) - 1.0).long().clamp(max=per_table - 1)
    slot = (bag // (case["batch"] * case["steps"])) * per_table + (rank * 2_654_435_761 + 97) % per_table
    order = torch.argsort(slot, stable=True)
    s = {"case": case, "slots": slot[order].int(), "bags": bag[order].int()}
    s["n"] = torch.tensor([n], dtype=torch.int32, device=DEVICE)
    s["grad"] = torch.randn(bags, D, generator=g, device=DEVICE).mul_(1e-3)
    s["dense"] = torch.randn(case["dense"], generator=g, device=DEVICE).mul_(1e-3)
    s["grad_out"], s["dense_out"] = torch.zeros_like(s["grad"]), torch.zeros_like(s["dense"])
    s["norm"] = torch.zeros(1, device=DEVICE)
    s["max_norm"] = 0.5e-3 * math.sqrt(bags * D + case["dense"])
    if own:
        import paper_2204_05436_b200 as hl

        s["hl"], s["stream"] = hl, torch.cuda.current_stream().cuda_stream
        geom = hl.make_geometry([per_table] * T, D, case["steps"])
        ws = hl.hl_workspace_bytes(geom, case["batch"], max(1, n), per_table * T, 0)
        s["workspace"] = torch.empty(ws, dtype=torch.uint8, device=DEVICE)
        s["ctx"] = _Context(hl, hl.hl_create(geom, case["batch"], max(1, n), per_table * T, 0, s["workspace"], ws))
        s["sumsq"] = torch.zeros(1, dtype=torch.float64, device=DEVICE)
        s["tensors"] = hl.make_tensors([(s["grad"], s["grad_out"], hl.HL_TENSOR_NOT_IN_NORM), (s["dense"], s["dense_out"])])
        s["ws_bytes"] = hl.hl_grad_workspace_bytes()
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEVICE)
    return s


class _Context:
    """A library context that goes with its state."""

    def __init__(self, hl, ctx):
        self.hl, self.ctx = hl, ctx

    def __del__(self):
        self.hl.hl_destroy(self.ctx)


def prepare(case, seed):
    return {"clip": _prepare_clip, "rowclip": _prepare_rowclip}.get(case["kind"], _prepare_experts)(case, seed)


# ---- one pass -------------------------------------------------------------------------------------------------------
def _run_sort(s):
    if not own:
        return _sorted(s["case"], s["experts"])
    s["hl"].hl_expert_sort(s["route"], s["experts"], _expert_cap(s["case"]), s["status"], s["ws"], s["ws_bytes"],
                           s["stream"])
    return s["place"], s["source"], s["counts"], s["offsets"]


def _to_rows(s, x, weights, out):
    """x[t] times the choice's weight in the rows of its experts, zeros in the rows that fill an expert up."""
    src = s["source"].long()
    a = src.clamp(min=0)
    v = x[a // s["case"]["top_k"]].float()
    if weights is not None:
        v = v * weights.view(-1)[a].unsqueeze(1)
    v = torch.where((src >= 0).unsqueeze(1), v, 0.0).to(x.dtype)
    return torch.where((src >= -1).unsqueeze(1), v, out)


def _to_tokens(s, y, weights, out):
    """The experts' rows of every live token, summed with the choices' weights."""
    live = s["case"]["live"]
    place = s["place"][:live].long()
    v = torch.where((place >= 0).unsqueeze(2), y[place.clamp(min=0)].float(), 0.0)
    if weights is not None:
        v = v * weights[:live].unsqueeze(2)
    return torch.cat([v.sum(dim=1).to(y.dtype), out[live:]])


def _run_dispatch(s):
    c, x, y = s["case"], s["x"], s["y"]
    if not own:
        there = _to_rows(s, x, None, s["to_rows"])
        return (there, _to_tokens(s, y, None, s["to_tokens"])) if c["train"] else there
    hl, route, there, back = s["hl"], s["route"], s["to_rows"], s["to_tokens"]
    ld = c["dim"] + c["pad"]
    hl.hl_expert_dispatch(route, s["type"], c["dim"], x, ld, there, ld, s["stream"])
    if not c["train"]:
        return there
    hl.hl_expert_combine(route, s["type"], c["dim"], y, ld, None, back, ld, s["stream"])
    return there, back


def _run_combine(s):
    c, x, y, w = s["case"], s["x"], s["y"], s["w"]
    if not own:
        out = _to_tokens(s, y, w, s["to_tokens"])
        if not c["train"]:
            return out
        place = s["place"][: c["live"]].long()
        dot = (y[place.clamp(min=0)].float() * x[: c["live"]].float().unsqueeze(1)).sum(dim=2)
        grad_w = torch.cat([torch.where(place >= 0, dot, 0.0), s["grad_w"][c["live"]:]])
        return out, _to_rows(s, x, w, s["to_rows"]), grad_w
    hl, route, ld = s["hl"], s["route"], c["dim"] + c["pad"]
    hl.hl_expert_combine(route, s["type"], c["dim"], y, ld, w, s["to_tokens"], ld, s["stream"])
    if not c["train"]:
        return s["to_tokens"]
    hl.hl_expert_combine_bwd(route, s["type"], c["dim"], x, ld, y, ld, w, s["to_rows"], ld, s["grad_w"], s["stream"])
    return s["to_tokens"], s["to_rows"], s["grad_w"]


def _factor(norm, max_norm):
    return (max_norm / (norm + 1e-6)).clamp(max=1.0)


def _run_clip(s):
    if own:
        s["hl"].hl_grad_clip(s["tensors"], None, 0, s["max_norm"], s["norm"], s["ws"], s["ws_bytes"], s["stream"])
        return s["dst"], s["norm"]
    norm = s["src"].double().square().sum().sqrt().view(1)
    return (s["src"].float() * _factor(norm, s["max_norm"]).float()).to(s["dst"].dtype), norm.float()


def _run_rowclip(s):
    if own:
        hl = s["hl"]
        hl.hl_embbag_grad_sumsq(s["ctx"].ctx, s["slots"], s["bags"], s["n"], s["grad"], s["sumsq"], s["stream"])
        hl.hl_grad_clip(s["tensors"], s["sumsq"], 1, s["max_norm"], s["norm"], s["ws"], s["ws_bytes"], s["stream"])
        return s["grad_out"], s["dense_out"], s["norm"]
    slots, grad = s["slots"], s["grad"]
    first = torch.ones_like(slots)
    first[1:] = (slots[1:] != slots[:-1]).int()
    row = first.cumsum(0) - 1
    rows = torch.zeros(slots.numel(), grad.shape[1], dtype=torch.float64, device=DEVICE)
    rows.index_add_(0, row, grad[s["bags"].long()].double())
    norm = (rows.square().sum() + s["dense"].double().square().sum()).sqrt().view(1)
    f = _factor(norm, s["max_norm"]).float()
    return grad * f, s["dense"] * f, norm.float()


def run(state):
    return {"sort": _run_sort, "dispatch": _run_dispatch, "combine": _run_combine, "clip": _run_clip,
            "rowclip": _run_rowclip}[state["case"]["kind"]](state)


# ---- the same in 64 bits, choice by choice and table by table ---------------------------------------------------------
def _exact_sums(s, y, weights):
    """Row `live` of the sums takes what has no token; a choice at a time."""
    live, place = s["case"]["live"], s["place"]
    out = s["to_tokens"].double()
    out[:live] = 0.0
    for k in range(s["case"]["top_k"]):
        t = torch.nonzero(place[:live, k] >= 0).view(-1)
        v = y[place[t, k].long()].double()
        out[t] += v if weights is None else weights[t, k].double().unsqueeze(1) * v
    return out


def _exact_rows(s, x, weights):
    live, place, end = s["case"]["live"], s["place"], int(s["offsets"][-1])
    out = s["to_rows"].double()
    out[:end] = 0.0
    for k in range(s["case"]["top_k"]):
        t = torch.nonzero(place[:live, k] >= 0).view(-1)
        v = x[t].double()
        out[place[t, k].long()] = v if weights is None else weights[t, k].double().unsqueeze(1) * v
    return out


def exact(case, seed):
    if case["kind"] == "sort":
        return None
    s = prepare(case, seed)
    if case["kind"] == "dispatch":
        there = _exact_rows(s, s["x"], None)
        return (there, _exact_sums(s, s["y"], None)) if case["train"] else there
    if case["kind"] == "combine":
        out = _exact_sums(s, s["y"], s["w"])
        if not case["train"]:
            return out
        grad_w = s["grad_w"].double()
        grad_w[: case["live"]] = 0.0
        for k in range(case["top_k"]):
            t = torch.nonzero(s["place"][: case["live"], k] >= 0).view(-1)
            grad_w[t, k] = torch.einsum("td,td->t", s["x"][t].double(), s["y"][s["place"][t, k].long()].double())
        return out, _exact_rows(s, s["x"], s["w"]), grad_w
    if case["kind"] == "clip":
        squares = 0.0
        for a, n in zip(_tensor_starts(case)[0], _tensor_sizes(case)):
            v = s["src"][a:a + n].double()
            squares += float(torch.dot(v, v))
        norm = math.sqrt(squares)
        return s["src"].double() * min(1.0, s["max_norm"] / (norm + 1e-6)), np.array([norm])
    slots, bags = s["slots"].cpu().numpy(), s["bags"].cpu().numpy()
    ends = np.concatenate([np.flatnonzero(slots[1:] != slots[:-1]) + 1, [slots.size]]) if slots.size else np.zeros(0, int)
    squares, d = 0.0, s["grad"].double().cpu().numpy()
    for c in range(0, d.shape[1], 8):                            # eight columns at a time: sums of runs by differences
        upto = np.concatenate([np.zeros((1, d[:, c:c + 8].shape[1])), np.cumsum(d[bags, c:c + 8], axis=0, dtype=np.longdouble)])
        of_run = np.diff(upto[np.concatenate([[0], ends]).astype(np.int64)], axis=0)
        squares += float(np.sum(of_run.astype(np.longdouble) ** 2))
    v = s["dense"].double()
    norm = math.sqrt(squares + float(torch.dot(v, v)))
    f = min(1.0, s["max_norm"] / (norm + 1e-6))
    return s["grad"].double() * f, v * f, np.array([norm])
