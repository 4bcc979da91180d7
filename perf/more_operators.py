"""The operators in front of a mixture of experts, and inside it, whose speed counts: the rows of a token embedding and their
gradient, the router's choices and their gradient, 4-bit quantisation and the experts' product.

Kinds of work (``case["kind"]``):

* ``choose``    logits become the chosen experts and their weights (hl_expert_choose), and in training (``train``) the weights'
                gradient becomes the logits' (hl_expert_choose_bwd);
* ``embed``     the scaled rows of tokens (hl_token_embed), and in training the gradient of the table, summed over the tokens
                of a row (hl_token_sort, hl_token_embed_bwd);
* ``quantise``  matrices in blocks of 32 values with one power of two, 4 bits a value (hl_mx4_quantise), and back
                (hl_mx4_dequantise);
* ``product``   rows times the weights of their experts, both in that form (hl_expert_mx4).

``run`` computes them in elementary torch operations where ``own`` is false and calls the library where it is true.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ---- the cases ------------------------------------------------------------------------------------------------------
def _choose(tokens, top_k, experts, live=None, score="softmax", bias=False, groups=1, top_groups=1, pair=False, renorm=True,
            scale=1.0, masked=0.0, dtype="f32", pad=0, train=False):
    """``live``: the tokens there are (a device-side count) of the ``tokens`` that the buffers hold; ``pair``: a group counts
    with its two best experts instead of its best; ``masked``: share of the logits that are -inf; ``pad``: values between the
    end of a row and the next."""
    return dict(kind="choose", tokens=tokens, top_k=top_k, experts=experts, live=tokens if live is None else live, score=score,
                bias=bias, groups=groups, top_groups=top_groups, pair=pair, renorm=renorm, scale=scale, masked=masked,
                dtype=dtype, pad=pad, train=train)


def _embed(tokens, rows, dim, live=None, alpha=1.1, padding=0.0, table="bf16", out="bf16", pad=0, train=False):
    """``rows`` of the table; ``alpha``: exponent of the power law of the tokens; ``padding``: share of tokens that are -1."""
    return dict(kind="embed", tokens=tokens, rows=rows, dim=dim, live=tokens if live is None else live, alpha=alpha,
                padding=padding, table=table, out=out, pad=pad, train=train)


def _quantise(matrices, rows, dim, dtype="bf16", pad=0):
    return dict(kind="quantise", matrices=matrices, rows=rows, dim=dim, dtype=dtype, pad=pad)


def _product(tokens, top_k, experts, dim, out, live=None, skew=0.0, dropped=0.0, align=1, by_token=True, dtype="bf16", pad=0):
    """``by_token``: the rows come in the tokens' order, not in the experts'; ``skew``: exponent of the power law of the experts'
    loads; ``dropped``: share of the choices that name no expert; ``align``: an expert's rows are filled up to a multiple."""
    return dict(kind="product", tokens=tokens, top_k=top_k, experts=experts, dim=dim, out=out,
                live=tokens if live is None else live, skew=skew, dropped=dropped, align=align, by_token=by_token, dtype=dtype,
                pad=pad)


def listed():
    cases = {
        # serving one input at a time: two of eight experts
        "choose one token": _choose(1, 2, 8, dtype="bf16"),
        # a training mini-batch of 16,384 inputs of which the popular 36 % are routed, four of 64 experts
        "choose popular inputs": _choose(16384, 4, 64, live=5899, dtype="f32", train=True),
        # many small experts in groups, balanced by a bias, a long packed mini-batch
        "choose grouped": _choose(65536, 8, 256, score="sigmoid", bias=True, groups=8, top_groups=4, pair=True, scale=2.5,
                                  dtype="bf16", train=True),
        # one step of decoding for four requests
        "embed few": _embed(4, 32000, 2048),
        # a long training mini-batch, gradient of the table in fp32 for its optimizer
        "embed train": _embed(16384, 32000, 2048, train=True),
        # a large table, a packed mini-batch of short rows
        "embed large": _embed(131_072, 200_000, 512, alpha=1.05, table="f32", out="bf16", train=True),
        # ragged: rows of 337 values (21 tables x 16 and one dense feature), a padded batch
        "embed ragged": _embed(30_011, 9_973, 337, live=28_657, padding=0.15, table="f16", out="f16", pad=2, train=True),
        # the weights of 16 experts, once they are loaded
        "quantise weights": _quantise(16, 4096, 2048),
        # rows of activations that begin anywhere
        "quantise ragged": _quantise(1, 4099, 337, dtype="f32", pad=2),
        # one input, two of eight experts
        "product one token": _product(1, 2, 8, 2048, 4096),
        # a prompt, four of 64 experts, uneven loads, experts' rows in their order
        "product ragged": _product(3001, 4, 64, 1664, 1001, live=2900, skew=0.7, dropped=0.05, align=16, by_token=False,
                                   dtype="f16"),
        # a large mini-batch, two of 16 experts
        "product large": _product(16384, 2, 16, 4096, 4096, skew=0.3),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["choose", "choose", "embed", "embed", "quantise", "product", "product"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    pad = rng.choice([0, 0, 8, rng.randint(1, 20)])
    if kind == "choose":
        experts, groups = rng.choice([(4, 1), (8, 1), (16, 4), (37, 1), (60, 5), (64, 1), (64, 8), (128, 1), (160, 8), (256, 8),
                                      (256, 1), (384, 1), (500, 1)])
        top_groups = rng.randint((groups + 1) // 2, groups)
        top_k = min(rng.choice([1, 2, 2, 3, 4, 6, 8]), experts // groups * top_groups)
        tokens = min(_log_int(rng, 1, 131_072), 16_000_000 // experts)
        live = tokens if rng.random() < 0.5 else rng.randint((tokens + 1) // 2, tokens)
        return _choose(tokens, top_k, experts, live, rng.choice(["softmax", "sigmoid"]), rng.random() < 0.5, groups, top_groups,
                       groups < experts and rng.random() < 0.5, rng.random() < 0.7, rng.choice([1.0, 1.0, 2.5]),
                       rng.choice([0.0, 0.0, 0.1]), dtype, pad, rng.random() < 0.6)
    if kind == "embed":
        dim = rng.choice([8 * _log_int(rng, 2, 512), _log_int(rng, 10, 4096)])
        rows = _log_int(rng, 500, 200_000)
        rows = min(rows, 100_000_000 // dim)
        tokens = min(_log_int(rng, 1, 262_144), 60_000_000 // dim)
        live = tokens if rng.random() < 0.5 else rng.randint((tokens + 1) // 2, tokens)
        return _embed(tokens, rows, dim, live, round(rng.uniform(1.02, 1.3), 3), rng.choice([0.0, 0.0, 0.2]), dtype,
                      rng.choice([dtype, "f32", "bf16"]), pad, rng.random() < 0.6)
    if kind == "quantise":
        dim = rng.choice([32 * _log_int(rng, 1, 256), _log_int(rng, 10, 8192)])
        matrices = rng.choice([1, 1, 2, 8, 37])
        return _quantise(matrices, max(1, min(_log_int(rng, 1, 65_536), 100_000_000 // (dim * matrices))), dim, dtype, pad)
    top_k, experts = rng.choice([1, 2, 2, 3, 4, 8]), rng.choice([1, 4, 8, 16, 37, 64, 128])
    dim = rng.choice([64 * _log_int(rng, 1, 64), _log_int(rng, 30, 4096)])
    out = rng.choice([64 * _log_int(rng, 1, 64), _log_int(rng, 30, 4096)])
    experts = max(1, min(experts, 200_000_000 // (dim * out)))
    tokens = max(1, min(_log_int(rng, 1, 16_384), 60_000_000 // (top_k * max(dim, out))))
    live = tokens if rng.random() < 0.5 else rng.randint((tokens + 1) // 2, tokens)
    return _product(tokens, top_k, experts, dim, out, live, round(rng.uniform(0.0, 1.0), 2), rng.choice([0.0, 0.0, 0.1]),
                    rng.choice([1, 1, 16, 128]), rng.random() < 0.5, dtype, pad)


# ---- sizes that follow from a case ----------------------------------------------------------------------------------
def _row_capacity(case):
    """Rows that hold whatever the router chooses."""
    n = case["tokens"] * case["top_k"]
    return n + min(case["experts"], n) * (case["align"] - 1)


def work(case):
    if case["kind"] == "choose":
        T, E, K, size = case["live"], case["experts"], case["top_k"], SIZE[case["dtype"]]
        moved = T * E * size + 8 * T * K
        if case["train"]:
            moved += T * E * size + 4 * T * K
        return {"bytes": moved, "flops": (10.0 if case["train"] else 5.0) * T * E}
    if case["kind"] == "embed":
        n, D = case["live"], case["dim"]
        touched = min(n, case["rows"])
        moved = touched * D * SIZE[case["table"]] + n * D * SIZE[case["out"]] + 4 * n
        if case["train"]:
            moved += n * D * SIZE[case["out"]] + case["rows"] * D * 4
        return {"bytes": moved, "flops": (2.0 if case["train"] else 1.0) * n * D}
    if case["kind"] == "quantise":
        n = case["matrices"] * case["rows"] * case["dim"]
        return {"bytes": n * (SIZE[case["dtype"]] + 4), "flops": 4.0 * n}
    kept = case["live"] * case["top_k"] * (1.0 - case["dropped"])
    rows = case["live"] if case["by_token"] else kept
    weights = min(case["experts"], kept) * case["out"] * case["dim"] * 17 / 32
    size = SIZE[case["dtype"]]
    return {"bytes": rows * case["dim"] * size + weights + kept * case["out"] * size,
            "flops": 2.0 * kept * case["dim"] * case["out"]}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _rows(case, g, n, dim, dtype):
    """n rows of a buffer with `pad` values between them."""
    return torch.randn(n, dim + case["pad"], generator=g, device=DEVICE).to(TYPES[dtype])[:, :dim]


def _empty_rows(case, n, dim, dtype):
    return torch.full((n, dim + case["pad"]), 2.0, dtype=TYPES[dtype], device=DEVICE)[:, :dim]


def _count(n):
    return torch.tensor([n], dtype=torch.int32, device=DEVICE)


def _prepare_choose(case, seed):
    g = _generator(seed)
    T, K, E = case["tokens"], case["top_k"], case["experts"]
    s = {"case": case, "logits": _rows(case, g, T, E, case["dtype"])}
    if case["masked"]:
        s["logits"][torch.rand(T, E, generator=g, device=DEVICE) < case["masked"]] = -math.inf
    s["bias"] = 0.1 * torch.randn(E, generator=g, device=DEVICE) if case["bias"] else None
    s["grad_w"] = torch.randn(T, K, generator=g, device=DEVICE)
    s["experts"] = torch.full((T, K), -7, dtype=torch.int32, device=DEVICE)
    s["w"] = torch.full((T, K), 2.0, device=DEVICE)
    s["grad"] = _empty_rows(case, T, E, case["dtype"])
    s["n_tokens"] = _count(case["live"])
    if own:
        import paper_2204_05436_b200 as hl

        s["hl"], s["stream"] = hl, torch.cuda.current_stream().cuda_stream
        s["type"] = hl.dtype_of(s["logits"])
        s["router"] = hl.make_router(hl.HL_SCORE_SOFTMAX if case["score"] == "softmax" else hl.HL_SCORE_SIGMOID, K, E,
                                     case["groups"], case["top_groups"],
                                     hl.HL_GROUP_TOP2 if case["pair"] else hl.HL_GROUP_MAX, case["renorm"], case["scale"])
        s["status"] = _count(0)
    return s


def _prepare_embed(case, seed):
    g = _generator(seed)
    n, V, D = case["tokens"], case["rows"], case["dim"]
    u = torch.rand(n, generator=g, device=DEVICE, dtype=torch.float64)
    tail = V ** (1.0 - case["alpha"])                            # a power law over [1, rows]
    rank = ((1.0 - u * (1.0 - tail)) ** (1.0 / (1.0 - case["alpha"])) - 1.0).long().clamp(max=V - 1)
    token = torch.randperm(V, generator=g, device=DEVICE)[rank]
    token = torch.where(torch.rand(n, generator=g, device=DEVICE) < case["padding"], -1, token)
    s = {"case": case, "token": token.int(), "scale": math.sqrt(D), "n_tokens": _count(case["live"])}
    s["table"] = _rows(case, g, V, D, case["table"])
    s["out"] = _empty_rows(case, n, D, case["out"])
    if case["train"]:
        s["grad_out"] = _rows(case, g, n, D, case["out"])
        s["grad"] = _empty_rows(case, V, D, "f32")
    if own:
        import paper_2204_05436_b200 as hl

        s["hl"], s["stream"] = hl, torch.cuda.current_stream().cuda_stream
        s["status"] = _count(0)
        s["types"] = hl.dtype_of(s["table"]), hl.dtype_of(s["out"])
        s["sorted"] = torch.empty(n, dtype=torch.int32, device=DEVICE)
        s["order"] = torch.empty(n, dtype=torch.int32, device=DEVICE)
        s["ws_bytes"] = hl.hl_token_workspace_bytes(n, D)
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEVICE)
    return s


def _prepare_quantise(case, seed):
    g = _generator(seed)
    M, R, D = case["matrices"], case["rows"], case["dim"]
    s = {"case": case, "x": _rows(case, g, M * R, D, case["dtype"])}
    s["x"] *= torch.exp(0.5 * torch.randn(M * R, 1, generator=g, device=DEVICE)).to(s["x"].dtype)
    if own:
        import paper_2204_05436_b200 as hl

        s["hl"], s["stream"] = hl, torch.cuda.current_stream().cuda_stream
        s["type"] = hl.dtype_of(s["x"])
        s["q"] = torch.empty(M * hl.hl_mx4_bytes(R, D), dtype=torch.uint8, device=DEVICE)
        s["out"] = _empty_rows(dict(case, pad=0), M * R, D, "f32")
    return s


def _choices(case, g):
    """int32 [tokens, top_k]: different experts for a token where there are enough, loads by a power law over a random
    order of the experts, -1 where none is chosen."""
    T, K, E = case["tokens"], case["top_k"], case["experts"]
    load = torch.arange(1, E + 1, device=DEVICE, dtype=torch.float32) ** -case["skew"]
    load = load[torch.randperm(E, generator=g, device=DEVICE)]
    noise = torch.rand(T, E, generator=g, device=DEVICE).clamp_(1e-7, 1.0 - 1e-7)
    scores = load.log() - (-noise.log()).log()                 # the largest of these: a draw by the loads
    e = scores.topk(K, dim=1).indices if K <= E else scores.argmax(dim=1, keepdim=True).expand(T, K)
    e = torch.where(torch.rand(T, K, generator=g, device=DEVICE) < case["dropped"], -1, e)
    return e.to(torch.int32).contiguous()


def _plan(case, experts):
    """The expert-ordered rows of the live tokens' choices: place, source, counts, offsets, as hl_expert_sort makes them."""
    T, K, E, align = case["tokens"], case["top_k"], case["experts"], case["align"]
    rows, n = _row_capacity(case), case["live"] * K
    e = experts[: case["live"]].reshape(-1).long()
    key = torch.where(e >= 0, e, E)
    order = torch.argsort(key, stable=True)
    ranked = key[order]
    seen = torch.zeros(E + 1, dtype=torch.int64, device=DEVICE).index_add_(0, key, torch.ones_like(key))
    first = seen.cumsum(0) - seen
    rank = torch.arange(n, device=DEVICE) - first[ranked]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=DEVICE)
    offsets[1:] = (((seen[:E] + align - 1) // align) * align).cumsum(0)
    at = torch.where(ranked < E, offsets[ranked] + rank, -1)
    place = torch.full((T * K,), -1, dtype=torch.int32, device=DEVICE)
    place[:n] = torch.empty(n, dtype=torch.int32, device=DEVICE).scatter_(0, order, at.int())
    source = torch.full((rows + 1,), -1, dtype=torch.int32, device=DEVICE)
    source[torch.where(at >= 0, at, rows)] = order.int()                     # (one row more, for what has no place)
    return place.view(T, K), source[:rows], seen[:E].int(), offsets.int()


def _prepare_product(case, seed):
    g = _generator(seed)
    T, K, E, D, F = case["tokens"], case["top_k"], case["experts"], case["dim"], case["out"]
    cap = _row_capacity(case)
    s = {"case": case, "n_tokens": _count(case["live"])}
    s["place"], s["source"], s["counts"], s["offsets"] = _plan(case, _choices(case, g))
    s["x"] = _rows(case, g, T if case["by_token"] else cap, D, case["dtype"])
    s["y"] = _empty_rows(case, cap, F, case["dtype"])
    w = (torch.randn(E * F, D, generator=g, device=DEVICE) / math.sqrt(D)).to(TYPES[case["dtype"]])
    if own:                                                      # laid out once, when the weights are loaded
        import paper_2204_05436_b200 as hl

        s["hl"], s["stream"] = hl, torch.cuda.current_stream().cuda_stream
        s["type"] = hl.dtype_of(s["x"])
        s["w"] = torch.empty(E * hl.hl_mx4_bytes(F, D), dtype=torch.uint8, device=DEVICE)
        hl.hl_mx4_quantise(s["type"], E, F, D, w, D, F * D, s["w"], s["stream"])
        s["route"] = hl.make_route(T, s["n_tokens"], K, E, case["align"], cap, s["place"], s["source"], s["counts"],
                                   s["offsets"])
        s["ws_bytes"] = hl.hl_expert_mx4_workspace_bytes(cap, E, D)
        s["ws"] = torch.empty(max(1, s["ws_bytes"]), dtype=torch.uint8, device=DEVICE)
    else:                                                        # (4-bit values times powers of two fit any of the types)
        s["w"] = torch.cat([_mx4(w[e * F:(e + 1) * F].float()).to(w.dtype) for e in range(E)]).view(E, F, D)
        s["host_counts"], s["host_offsets"] = s["counts"].tolist(), s["offsets"].tolist()
    return s


def prepare(case, seed):
    return {"choose": _prepare_choose, "embed": _prepare_embed, "quantise": _prepare_quantise,
            "product": _prepare_product}[case["kind"]](case, seed)


# ---- one pass -------------------------------------------------------------------------------------------------------
def _group_mask(case, keys, for_groups):
    """Which experts are in the groups that are kept: the best, the lowest number first where groups are equal."""
    T, E, G = keys.shape[0], case["experts"], case["groups"]
    best = for_groups.view(T, G, E // G).sort(dim=2, descending=True).values
    score = best[:, :, 0]
    if case["pair"] and E // G > 1:
        score = score + torch.where(best[:, :, 1] > -math.inf, best[:, :, 1], 0.0)
    kept = score.sort(dim=1, descending=True, stable=True).indices[:, : case["top_groups"]]
    mask = torch.zeros(T, G, dtype=torch.bool, device=DEVICE).scatter_(1, kept, True)
    return mask.unsqueeze(2).expand(T, G, E // G).reshape(T, E)


def _scores(case, logits):
    if case["score"] == "sigmoid":
        return torch.sigmoid(logits)
    top = logits.max(dim=1, keepdim=True).values
    e = torch.exp(logits - torch.where(top > -math.inf, top, 0.0))
    return e / e.sum(dim=1, keepdim=True).clamp(min=1e-300)


def _run_choose(s):
    c = s["case"]
    if own:
        hl, ld = s["hl"], c["experts"] + c["pad"]
        hl.hl_expert_choose(s["router"], s["type"], s["logits"], ld, s["bias"], c["tokens"], s["n_tokens"], s["experts"], s["w"],
                            s["status"], s["stream"])
        if not c["train"]:
            return s["experts"], s["w"]
        hl.hl_expert_choose_bwd(s["router"], s["type"], s["logits"], ld, c["tokens"], s["n_tokens"], s["experts"], s["grad_w"],
                                s["grad"], ld, s["stream"])
        return s["experts"], s["w"], s["grad"]
    live, K = c["live"], c["top_k"]
    logits = s["logits"][:live].double()                         # (scores next to one another decide who is chosen)
    score = _scores(c, logits)
    there = logits > -math.inf
    keys = logits if s["bias"] is None else torch.where(there, score + s["bias"].double(), -math.inf)
    if c["groups"] > 1:
        by = torch.where(there, score, -math.inf) if c["pair"] and s["bias"] is None else keys
        keys = torch.where(_group_mask(c, keys, by), keys, -math.inf)
    order = keys.sort(dim=1, descending=True, stable=True)
    e, valid = order.indices[:, :K], order.values[:, :K] > -math.inf
    chosen = torch.where(valid, score.gather(1, e), 0.0)
    total = chosen.sum(dim=1, keepdim=True).clamp(min=1e-300) if c["renorm"] else 1.0
    w = c["scale"] * chosen / total
    out = (torch.cat([torch.where(valid, e, -1).int(), s["experts"][live:]]), torch.cat([w.float(), s["w"][live:]]))
    if not c["train"]:
        return out
    gw = torch.where(valid, s["grad_w"][:live].double(), 0.0)
    gs = c["scale"] * gw
    if c["renorm"]:
        gs = (gs - (gw * w).sum(dim=1, keepdim=True)) / total
    gs = torch.zeros_like(score).scatter_add_(1, e, torch.where(valid, gs, 0.0))
    grad = gs * score * (1.0 - score) if c["score"] == "sigmoid" else score * (gs - (gs * score).sum(dim=1, keepdim=True))
    return out + (torch.cat([grad.to(s["grad"].dtype), s["grad"][live:]]),)


def _run_embed(s):
    c = s["case"]
    V, D, live = c["rows"], c["dim"], c["live"]
    if own:
        hl, ld = s["hl"], D + c["pad"]
        table, out = s["types"]
        hl.hl_token_embed(table, V, D, s["table"], ld, s["token"], c["tokens"], s["n_tokens"], s["scale"], out, s["out"], ld,
                          s["status"], s["stream"])
        if not c["train"]:
            return s["out"]
        hl.hl_token_sort(s["token"], c["tokens"], s["n_tokens"], V, s["sorted"], s["order"], s["status"], s["ws"], s["ws_bytes"],
                         s["stream"])
        hl.hl_token_embed_bwd(V, D, s["sorted"], s["order"], c["tokens"], s["n_tokens"], out, s["grad_out"], ld, s["scale"],
                              hl.HL_F32, s["grad"], ld, False, s["ws"], s["ws_bytes"], s["stream"])
        return s["out"], s["grad"]
    token = s["token"][:live].long()
    there = (token >= 0).unsqueeze(1)
    out = torch.where(there, s["table"][token.clamp(min=0)].float() * s["scale"], 0.0)
    out = torch.cat([out.to(s["out"].dtype), s["out"][live:]])
    if not c["train"]:
        return out
    grad = torch.zeros(V + 1, D, device=DEVICE)
    grad.index_add_(0, torch.where(token >= 0, token, V), s["grad_out"][:live].float())
    return out, grad[:V] * s["scale"]


def _power_of_two(n):
    return ((n + 127) << 23).view(torch.float32)                 # (exactly, which torch.ldexp is not)


def _mx4(x):
    """The values that x (fp32 [rows, dim]) has in 4 bits: blocks of 32 with a power of two each, of which the largest value's
    lies two above; values of one mantissa bit, rounded to even."""
    rows, dim = x.shape
    blocks = -(-dim // 32)
    v = torch.zeros(rows, blocks * 32, device=x.device)
    v[:, :dim] = x
    v = v.view(rows, blocks, 32)
    power = (torch.frexp(v.abs().amax(dim=2, keepdim=True)).exponent - 3).clamp(-127, 127)
    a = v * _power_of_two(-power)
    step = torch.where(a.abs() < 2.0, 0.5, torch.where(a.abs() < 4.0, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(-6.0, 6.0)
    return (0.5 * a * _power_of_two(power + 1)).reshape(rows, blocks * 32)[:, :dim]


def _run_quantise(s):
    c = s["case"]
    if not own:
        return _mx4(s["x"].float())
    hl, M, R, D, ld = s["hl"], c["matrices"], c["rows"], c["dim"], c["dim"] + c["pad"]
    hl.hl_mx4_quantise(s["type"], M, R, D, s["x"], ld, R * ld, s["q"], s["stream"])
    hl.hl_mx4_dequantise(M, R, D, s["q"], hl.HL_F32, s["out"], D, R * D, s["stream"])
    return s["out"]


def _run_product(s):
    c = s["case"]
    if own:
        s["hl"].hl_expert_mx4(s["route"], s["type"], c["dim"], c["out"], s["x"], c["dim"] + c["pad"], c["by_token"], s["w"], s["y"],
                              c["out"] + c["pad"], s["ws"], s["ws_bytes"], s["stream"])
        return s["y"]
    y = s["y"].clone()
    x = _mx4(s["x"].float())
    for e in range(c["experts"]):
        n, a, b = s["host_counts"][e], s["host_offsets"][e], s["host_offsets"][e + 1]
        if n:
            rows = x[s["source"][a:a + n].long() // c["top_k"]] if c["by_token"] else x[a:a + n]
            y[a:a + n] = (rows @ s["w"][e].float().t()).to(y.dtype)
        y[a + n:b] = 0.0                                         # (rows that fill an expert up)
    return y


def run(state):
    return {"choose": _run_choose, "embed": _run_embed, "quantise": _run_quantise,
            "product": _run_product}[state["case"]["kind"]](state)


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------
def _exact_choose(case, s):
    """One choice after the other; every score from the ratio of two sums of exponentials, the gradient from differences of
    the weights' definition written out."""
    live, K, E, G = case["live"], case["top_k"], case["experts"], case["groups"]
    l = s["logits"][:live].double()
    there = l > -math.inf
    if case["score"] == "softmax":
        p = torch.exp(l - torch.logsumexp(l, dim=1, keepdim=True))
        p = torch.where(there, p, 0.0)
    else:
        p = torch.where(there, 1.0 / (1.0 + torch.exp(-l)), 0.0)
    key = l if s["bias"] is None else torch.where(there, p + s["bias"].double(), -math.inf)
    open_ = there.clone()
    if G > 1:
        by = (p if s["bias"] is None and case["pair"] else key).masked_fill(~there, -math.inf).view(live, G, E // G)
        value = by.amax(dim=2)
        if case["pair"] and E // G > 1:
            second = by.topk(2, dim=2).values[:, :, 1]
            value = value + torch.where(second > -math.inf, second, 0.0)
        rank = torch.arange(G, device=DEVICE)
        better = (value.unsqueeze(1) > value.unsqueeze(2)) | ((value.unsqueeze(1) == value.unsqueeze(2)) & (rank < rank.view(G, 1)))
        kept = better.sum(dim=2) < case["top_groups"]
        open_ &= kept.repeat_interleave(E // G, dim=1)
    number = torch.arange(E, device=DEVICE).expand(live, E)
    chosen, ids = torch.zeros(live, E, dtype=torch.bool, device=DEVICE), []
    for _ in range(K):
        v = key.masked_fill(~open_, -math.inf)
        e = torch.where(open_ & (v == v.amax(dim=1, keepdim=True)), number, E).amin(dim=1)
        ids.append(e)
        hit = number == e.unsqueeze(1)
        chosen |= hit
        open_ &= ~hit
    ids = torch.stack(ids, dim=1)
    valid, at = ids < E, ids.clamp(max=E - 1)
    raw = p.gather(1, at) * valid
    whole = raw.sum(dim=1, keepdim=True) if case["renorm"] else torch.ones(live, 1, dtype=torch.float64, device=DEVICE)
    whole = torch.where(whole > 0, whole, 1.0)
    w = case["scale"] * raw / whole
    result = (None, torch.cat([w, s["w"][live:].double()]))
    if not case["train"]:
        return result
    # d w_k / d l_e: of the scores, and of their sum
    gw = s["grad_w"][:live].double() * valid
    g_p = torch.zeros_like(p).scatter_add_(1, at, case["scale"] * gw / whole)
    if case["renorm"]:
        g_p -= chosen * (gw * w).sum(dim=1, keepdim=True) / whole
    g_l = p * g_p
    g_l = g_l - p * (g_l if case["score"] == "sigmoid" else g_l.sum(dim=1, keepdim=True))
    return result + (torch.cat([g_l, s["grad"][live:].double()]),)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "choose":
        return _exact_choose(case, s)
    if case["kind"] == "embed":
        live, scale = case["live"], s["scale"]
        out = s["out"].double()
        token = s["token"][:live].long()
        there = token >= 0
        out[:live] = 0.0
        out[:live][there] = scale * s["table"].double()[token[there]]
        if not case["train"]:
            return out
        grad = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device=DEVICE)
        grad.index_put_((token[there],), scale * s["grad_out"][:live][there].double(), accumulate=True)
        return out, grad
    if case["kind"] == "quantise":
        return _exact_mx4(s["x"])
    D, F = case["dim"], case["out"]
    g = _generator(seed)                                         # (the weights are drawn again, before they were quantised)
    cap = _row_capacity(case)
    _choices(case, g)
    x = _rows(case, g, case["tokens"] if case["by_token"] else cap, D, case["dtype"])
    w = (torch.randn(case["experts"] * F, D, generator=g, device=DEVICE) / math.sqrt(D)).to(TYPES[case["dtype"]])
    x = _exact_mx4(x)
    y = s["y"].double()
    counts, offsets = s["counts"].tolist(), s["offsets"].tolist()
    for e, n in enumerate(counts):
        y[offsets[e]:offsets[e + 1]] = 0.0
        rows = torch.arange(offsets[e], offsets[e] + n, device=DEVICE)
        if n:
            y[rows] = x[s["source"][rows].long() // case["top_k"] if case["by_token"] else rows] @ _exact_mx4(w[e * F:(e + 1) * F]).t()
    return y


def _two_to(power):
    return ((power + 1023) << 52).view(torch.float64)


def _exact_mx4(x):
    """The nearest of the fifteen values, and of two as near the one whose place in the list is even."""
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEVICE)
    between = (values[1:] + values[:-1]) / 2
    out = torch.empty(x.shape, dtype=torch.float64, device=DEVICE)
    for c in range(0, x.shape[1], 32):
        v = x[:, c:c + 32].double()
        largest = v.abs().amax(dim=1, keepdim=True)
        largest = torch.where(largest > 0, largest, 1.0)
        power = torch.floor(torch.log2(largest)).long()          # (of a power of two the logarithm may lie next to it)
        power += (largest >= _two_to(power + 1)).long()
        power -= (largest < _two_to(power)).long()
        unit = _two_to(power - 2)
        a = v.abs() / unit
        low = torch.bucketize(a, between)                        # a tie counts to the lower one,
        high = torch.bucketize(a, between, right=True)           # and to the higher one
        out[:, c:c + 32] = values[torch.where(low % 2 == 0, low, high)] * torch.sign(v) * unit
    return out
