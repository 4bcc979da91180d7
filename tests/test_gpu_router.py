"""The router's choices (hl_expert_choose) and their gradient, against the definition in 64 bits, one choice after the other.

Tolerances, with s = 2^-24 (a rounding of fp32): a score is an exponential (2 ulp = 4 s, and its argument's rounding, s times the
logits' range R), one or two roundings for a sigmoid, and a quotient; a sum of n of them adds n s (n: the chosen K, or all E in
the order of a tree and at most 32 in a row).  So weights are within (R + n + 16) 2 s of themselves.  A logit's gradient is a
share times a difference of gradients: within (R + 2 n + 24) 4 s of scale * max|grad_w|, plus half a step of the logits' type."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

S = 2.0 ** -24
INF = float("inf")


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _scores(l, softmax):
    """fp64 scores of fp64 logits [T, E] (no NaN)."""
    if not softmax:
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-l))
    top = l.max(axis=1, keepdims=True)
    same = l == top
    with np.errstate(invalid="ignore"):
        e = np.where(same & (top > -INF), 1.0, np.exp(l - top))
    e = np.where(l > -INF, e, 0.0)
    z = e.sum(axis=1, keepdims=True)
    return e / np.where(z > 0, z, 1.0)


def _expected(l, K, softmax, G, TG, pair, renorm, scale, bias):
    T, E = l.shape
    l = np.where(np.isnan(l), -INF, l)
    s = _scores(l, softmax)
    there = l > -INF
    key = l.copy()
    if bias is not None:
        with np.errstate(invalid="ignore"):
            key = np.where(there, s + bias, -INF)
        key = np.where(np.isnan(key), -INF, key)
    by = np.where(there, s, -INF) if bias is None and pair else key
    experts = np.full((T, K), -1, np.int64)
    for t in range(T):
        k = key[t].copy()
        if G > 1:
            values = []
            for g in range(G):
                v = np.sort(by[t, g * (E // G):(g + 1) * (E // G)])[::-1]
                values.append(v[0] + (v[1] if pair and len(v) > 1 and v[1] > -INF else 0.0))
            order = sorted(range(G), key=lambda g: (-values[g], g))
            for g in order[TG:]:
                k[g * (E // G):(g + 1) * (E // G)] = -INF
        order = np.lexsort((np.arange(E), -k))
        for i, e in enumerate(order[:K]):
            if k[e] > -INF:
                experts[t, i] = e
    valid = experts >= 0
    at = np.where(valid, experts, 0)
    lc = np.where(valid, np.take_along_axis(l, at, axis=1), -INF)
    if renorm:
        # relative to the largest, so that nothing is lost to underflow
        m = lc.max(axis=1, keepdims=True)
        if not softmax:
            m = np.minimum(m, 0.0)
        with np.errstate(over="ignore", invalid="ignore"):
            r = np.where(lc == m, 1.0, np.exp(lc - m)) if softmax else np.where(
                lc > 0, 1.0 / (1.0 + np.exp(-lc)), np.where(lc == m, 1.0, np.exp(lc - m)) / (1.0 + np.exp(lc)))
        r = np.where(valid, r, 0.0)
        z = r.sum(axis=1, keepdims=True)
        w = scale * r / np.where(z > 0, z, 1.0)
    else:
        w = scale * np.where(valid, np.take_along_axis(s, at, axis=1), 0.0)
    return experts, w, s


def _choose(hl, l, bias=None, live=None, **r):
    """Through the C boundary, into buffers that are longer than what may be written."""
    T, E = l.shape
    K = r["top_k"]
    router = hl.make_router(r.get("score", 0), K, E, r.get("G", 1), r.get("TG", 1), int(r.get("pair", False)), r.get("renorm", True),
                            r.get("scale", 1.0))
    e = torch.full((T + 3, K), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T + 3, K), -7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda")
    hl.hl_expert_choose(router, hl.dtype_of(l), l, l.stride(0) if T > 1 else max(E, l.stride(0)), bias, T, n, e, w, status,
                        torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    rows = T if live is None else min(max(live, 0), T)
    assert (e[rows:] == -7).all() and (w[rows:] == -7).all()
    return router, e[:rows], w[:rows], int(status.item())


def _check(hl, l, bias=None, live=None, bad=False, **r):
    T = l.shape[0] if live is None else min(max(live, 0), l.shape[0])
    router, e, w, status = _choose(hl, l, bias, live, **r)
    assert status == (hl.HL_EINVAL if bad else hl.HL_OK)
    l64 = l[:T].double().cpu().numpy()
    b64 = None if bias is None else bias.double().cpu().numpy()
    args = (r["top_k"], r.get("score", 0) == 0, r.get("G", 1), r.get("TG", 1), r.get("pair", False), r.get("renorm", True), r.get("scale", 1.0))
    experts, weights, _ = _expected(l64, *args, b64)
    assert np.array_equal(e.cpu().numpy(), experts)
    finite = l64[np.isfinite(l64)]
    R = min(float(finite.max() - finite.min()), 200.0) if finite.size else 0.0
    n = r["top_k"] if r.get("renorm", True) else 32 + 5
    err = np.abs(w.double().cpu().numpy() - weights)
    assert (err <= (R + n + 16) * 2 * S * np.abs(weights) + 1e-37).all(), err.max()
    return router, e, w


def _logits(T, E, dtype, seed, spread=1.5, steps=None):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E, generator=g) * spread
    if steps:
        l = (l * steps).round() / steps                          # many equal ones
    return l.to(dtype).cuda()


SHAPES = [(1, 1), (2, 2), (3, 7), (8, 8), (2, 9), (5, 16), (4, 31), (6, 33), (8, 64), (64, 64), (33, 65), (8, 100), (1, 128), (15, 128),
          (16, 129), (8, 256), (31, 256), (32, 250), (64, 256), (6, 257), (8, 500), (64, 512), (2, 513), (8, 1000), (64, 1024)]


@pytest.mark.parametrize("K,E", SHAPES)
@pytest.mark.parametrize("score", [0, 1])
def test_choices(hl, K, E, score):
    for i, dtype in enumerate((torch.float32, torch.bfloat16, torch.float16)):
        l = _logits(37, E, dtype, 10 * E + K + i)
        bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(E))).cuda()
        for renorm in (True, False):
            _check(hl, l, top_k=K, score=score, renorm=renorm, scale=2.5)
            _check(hl, l, bias, top_k=K, score=score, renorm=renorm)


@pytest.mark.parametrize("E,G,TG,K", [(8, 2, 1, 3), (8, 8, 3, 2), (16, 4, 2, 8), (60, 5, 3, 6), (64, 8, 3, 8), (64, 2, 1, 4), (64, 64, 9, 9),
                                      (128, 16, 5, 8), (160, 8, 3, 6), (256, 8, 4, 8), (256, 8, 2, 8), (256, 8, 1, 32), (256, 2, 1, 8),
                                      (256, 16, 16, 8), (500, 4, 2, 8), (512, 8, 2, 16), (1024, 32, 4, 8), (1000, 50, 7, 64),
                                      (32, 8, 3, 4), (96, 8, 3, 4), (192, 4, 2, 8), (384, 8, 4, 8), (480, 10, 4, 8), (800, 25, 5, 20)])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("pair", [False, True])
def test_groups(hl, E, G, TG, K, score, pair):
    l = _logits(29, E, torch.bfloat16 if K % 2 else torch.float32, E + G)
    bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(G))).cuda()
    l[3, : E // 2] = -INF
    l[4] = -INF
    l[5, 1:] = -INF
    for b in (None, bias):
        _check(hl, l, b, top_k=K, score=score, G=G, TG=TG, pair=pair)


@pytest.mark.parametrize("E,G,TG", [(8, 1, 1), (64, 8, 3), (100, 1, 1), (256, 1, 1), (256, 8, 4), (700, 1, 1)])
@pytest.mark.parametrize("score", [0, 1])
def test_ties_go_to_the_lowest_number(hl, E, G, TG, score):
    K = min(8, E // G * TG)
    flat = torch.full((5, E), 0.25, device="cuda")
    flat[1] = 0.0
    flat[1, ::2] = -0.0
    flat[2] = torch.finfo(torch.float32).min
    flat[3] = -INF
    few = _logits(40, E, torch.float32, E, steps=2)
    zeros, bias = torch.zeros(E, device="cuda"), (torch.arange(E, device="cuda") % 3).float() * 0.125
    for l in (flat, few):
        for b in (None, zeros, bias):
            for pair in (False, True):
                _check(hl, l, b, top_k=K, score=score, G=G, TG=TG, pair=pair)


@pytest.mark.parametrize("E", [8, 64, 130, 256, 1000])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("G", [1, 2])
def test_keys_that_32_bits_cannot_tell_apart(hl, E, score, G):
    """Scores plus biases that differ by 2^-27 and less: the order is that of 64 bits."""
    g = torch.Generator().manual_seed(E)
    l = (0.5 + torch.randint(-4, 5, (60, E), generator=g) * 2.0 ** -24).cuda()
    bias = (0.25 + torch.randint(-4, 5, (E,), generator=g) * 2.0 ** -26).cuda()
    _check(hl, l, bias, top_k=min(8, E // 2), score=score, G=G, TG=1, pair=True)
    # large logits, whose sigmoids differ from 1 by less than that
    _check(hl, (20 + torch.rand(60, E, generator=g)).cuda(), bias, top_k=min(8, E // 2), score=score, G=G, TG=1, pair=False)


@pytest.mark.parametrize("E", [4, 64, 256, 600])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_masks_infinities_and_nan(hl, E, score, dtype):
    K = min(E, 6)
    l = _logits(12, E, dtype, E)
    l[0] = -INF                                                  # nobody is left
    l[1, 2:] = -INF
    l[2] = torch.finfo(dtype).min                                # the lowest value is a logit like others
    l[3, 1] = torch.finfo(dtype).min
    l[4, E - 1] = INF
    l[5, : E // 2] = INF
    l[6] = -80.0                                                 # their scores are next to nothing, not their ratios
    l[6, 1], l[6, 0] = -79.0, -100.0
    if dtype != torch.float16:
        l[7] = -200.0
        l[7, E - 1] = -199.0
    for renorm in (True, False):
        _check(hl, l, top_k=K, score=score, renorm=renorm)
    bias = torch.zeros(E, device="cuda")
    bias[1] = -INF
    bias[E - 1] = INF
    _check(hl, l, bias, top_k=K, score=score)
    l[8, 0] = float("nan")
    l[9] = float("nan")
    _check(hl, l, top_k=K, score=score, bad=True)
    l[8:10] = 0.0
    bias[2] = float("nan")
    _check(hl, l, bias, top_k=K, score=score, bad=True)


@pytest.mark.parametrize("E", [5, 64, 96, 256, 515])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_anywhere_and_counts_on_the_device(hl, E, dtype):
    wide = torch.full((50, E + 13), float("nan"), dtype=dtype, device="cuda")
    for at in (0, 1, 8):
        l = wide[:, at:at + E]
        l[:] = _logits(50, E, dtype, E + at)
        bias = torch.randn(E + 1, device="cuda")[at % 2:at % 2 + E] * 0.1
        for live in (None, 0, 1, 49, 50, 1000, -3):
            _check(hl, l, bias, live=live, top_k=min(4, E), score=1)
        wide[:] = float("nan")


def test_one_token_and_many(hl):
    for T in (1, 2, 31, 33, 1000):
        for E in (8, 64, 256):
            _check(hl, _logits(T, E, torch.float32, T), top_k=2)


# ---- the gradient ---------------------------------------------------------------------------------------------------------
def _formula(l, experts, gw, softmax, renorm, scale):
    """By torch's differentiation, in 64 bits, of the weights of the experts that were chosen."""
    x = torch.where(torch.isnan(l), -INF, l.double()).requires_grad_()
    valid = experts >= 0
    at = experts.clamp(min=0).long()
    if softmax and not renorm:
        w = torch.softmax(x.masked_fill((x == -INF).all(dim=1, keepdim=True), 0.0), dim=1).gather(1, at)
    else:
        log = x if softmax else torch.nn.functional.logsigmoid(x)
        c = torch.where(valid, log.gather(1, at), -INF)
        if renorm:
            none = ~valid.any(dim=1, keepdim=True)
            w = torch.softmax(c.masked_fill(none, 0.0), dim=1)
        else:
            w = torch.sigmoid(x).gather(1, at)
    w = torch.where(valid, scale * w, 0.0)
    (w * gw.double()).sum().backward()
    return torch.nan_to_num(x.grad, nan=0.0)


def _check_grad(hl, l, gw, router, e, softmax, renorm, scale, live=None):
    T, E = l.shape
    K = e.shape[1]
    full = torch.full((T, K), -1, dtype=torch.int32, device="cuda")
    full[: e.shape[0]] = e
    wide = torch.full((T + 2, E + 5), -7.0, dtype=l.dtype, device="cuda")
    for at in (0, 1):
        wide[:] = -7.0
        out = wide[:T, at:at + E]
        n = None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda")
        hl.hl_expert_choose_bwd(router, hl.dtype_of(l), l, l.stride(0), T, n, full, gw, out, out.stride(0),
                                torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        rows = T if live is None else live
        want = _formula(l[:rows], full[:rows], gw[:rows], softmax, renorm, scale)
        finite = l[:rows].double()
        finite = finite[torch.isfinite(finite)]
        R = min(float(finite.max() - finite.min()), 200.0) if finite.numel() else 0.0
        n_sum = K if renorm else 32 + 5
        top = float(gw.abs().max()) * abs(scale)
        tol = (R + 2 * n_sum + 24) * 4 * S * top + torch.finfo(l.dtype).eps / 2 * want.abs() + (2.0 ** -25 if l.dtype == torch.float16 else 0)
        err = (out[:rows].double() - want).abs()
        assert (err <= tol).all(), float((err - tol).max())
        assert (wide[:rows, :at] == -7).all() and (wide[:rows, at + E:] == -7).all() and (wide[rows:] == -7).all()


@pytest.mark.parametrize("K,E", [(1, 1), (2, 8), (3, 7), (8, 64), (17, 33), (8, 256), (64, 300), (4, 1000)])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gradient(hl, K, E, score, renorm, dtype):
    l = _logits(33, E, dtype, E + K)
    if E > 4:
        l[2, : E // 2] = -INF
        l[3] = -INF
        l[4, 1:] = -INF
    bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(E))).cuda()
    gw = torch.randn(33, K, generator=torch.Generator().manual_seed(K)).cuda()
    for live in (None, 20):
        router, e, _ = _check(hl, l, bias, live=live, top_k=K, score=score, renorm=renorm, scale=1.5)
        _check_grad(hl, l, gw, router, e, score == 0, renorm, 1.5, live)


@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("K,E", [(1, 8), (1, 64), (1, 300), (4, 37), (8, 256), (20, 64)])
def test_shares_that_cannot_change(hl, K, E, score):
    """A share of one alone is 1, and gradients that are all alike (here and there infinite) change no share: exactly 0."""
    l = _logits(500, E, torch.float32, E + K)
    gw = torch.randn(500, K, generator=torch.Generator().manual_seed(K)).cuda()
    if K > 1:
        l[::2, 1:] = -INF
        gw[::2, 1:] = INF                                        # (of choices that are not there)
        gw[1::2] = gw[1::2, :1]
    router, e, _ = _check(hl, l, top_k=K, score=score, renorm=True, scale=2.5)
    out = torch.full((500, E), -7.0, device="cuda")
    hl.hl_expert_choose_bwd(router, hl.HL_F32, l, E, 500, None, e, gw, out, E, torch.cuda.current_stream().cuda_stream)
    assert (out == 0).all(), float(out.abs().max())


@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_against_differences(hl, score, renorm):
    """Of the sum of grad_w * weights, by central differences of the 64-bit definition (the choice stays the same)."""
    T, E, K, scale, h = 6, 24, 3, 2.0, 1e-5
    l = _logits(T, E, torch.float32, 5)
    gw = torch.randn(T, K, generator=torch.Generator().manual_seed(1)).cuda()
    router, e, _ = _check(hl, l, top_k=K, score=score, renorm=renorm, scale=scale)
    out = torch.zeros(T, E, device="cuda")
    hl.hl_expert_choose_bwd(router, hl.HL_F32, l, E, T, None, e, gw, out, E, torch.cuda.current_stream().cuda_stream)
    l64, g64, experts = l.double().cpu().numpy(), gw.double().cpu().numpy(), e.cpu().numpy()

    def value(x):
        s = np.take_along_axis(_scores(x, score == 0), experts.astype(np.int64), axis=1)
        return (g64 * scale * s / (s.sum(axis=1, keepdims=True) if renorm else 1.0)).sum(axis=1)

    for j in range(E):
        up, down = l64.copy(), l64.copy()
        up[:, j] += h
        down[:, j] -= h
        want = (value(up) - value(down)) / (2 * h)
        # (differences: h^2 times a third derivative of at most some ten, and 2^-53 / h)
        assert np.abs(out[:, j].double().cpu().numpy() - want).max() < 1e-7 + 200 * S * scale * np.abs(g64).max()


def test_an_expert_that_is_there_twice_gets_the_sum(hl):
    l = _logits(4, 16, torch.float32, 3)
    gw = torch.randn(4, 3, generator=torch.Generator().manual_seed(2)).cuda()
    e = torch.tensor([[1, 1, 2], [5, 5, 5], [0, -1, 0], [7, 99, -5]], dtype=torch.int32).cuda()
    for score in (0, 1):
        router = hl.make_router(score, 3, 16, renorm=False)
        out = torch.zeros(4, 16, device="cuda")
        hl.hl_expert_choose_bwd(router, hl.HL_F32, l, 16, 4, None, e, gw, out, 16, torch.cuda.current_stream().cuda_stream)
        want = _formula(l, torch.where(e < 16, e, -1), gw, score == 0, False, 1.0)
        assert (out.double() - want).abs().max() < 200 * S * 4


def test_class(hl):
    router = hl.ExpertRouter(4, 64, score="sigmoid", n_groups=8, top_groups=4, group_score="top2", scale=2.5)
    l = _logits(50, 64, torch.bfloat16, 7)
    bias = torch.randn(64, device="cuda") * 0.1
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        e, w = router.choose(l, bias)
        grad = router.backward(l, e, torch.ones_like(w))
    assert router.status() == hl.HL_OK
    _, e2, w2 = _check(hl, l, bias, top_k=4, score=1, G=8, TG=4, pair=True, scale=2.5)
    assert torch.equal(e, e2) and torch.equal(w, w2) and grad.shape == l.shape
    # (weights of a sum that is given: their gradients for equal ones cancel)
    assert grad.double().abs().max() <= 400 * S * 2.5 + 2.0 ** -8 * 1e-3
    l[0, 0] = float("nan")
    router.choose(l, bias)
    assert router.status(raise_on_error=False) == hl.HL_EINVAL and router.status() == hl.HL_OK
    for bad in (l.float()[:, :63], l.int(), l.t(), l[:, ::2]):
        with pytest.raises((ValueError, TypeError)):
            router.choose(bad)
    with pytest.raises(ValueError):
        router.choose(l, bias.double())
    with pytest.raises(ValueError):
        router.choose(l, bias, out=(e, e.view(torch.float32)))
    with pytest.raises(ValueError):
        router.backward(l, e, w, out=l)


def test_captured_and_replayed(hl):
    router = hl.ExpertRouter(8, 256, score="sigmoid", scale=2.0)
    l, bias = _logits(300, 256, torch.float32, 1), torch.randn(256, device="cuda") * 0.1
    out = (torch.zeros(300, 8, dtype=torch.int32, device="cuda"), torch.zeros(300, 8, device="cuda"))
    grad, gw = torch.zeros_like(l), torch.randn(300, 8, device="cuda")
    router.choose(l, bias, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        router.choose(l, bias, out=out)
        router.backward(l, out[0], gw, out=grad)
    for seed in (2, 3):
        l.copy_(_logits(300, 256, torch.float32, seed))
        graph.replay()
        torch.cuda.synchronize()
        e, w = router.choose(l, bias)
        assert torch.equal(e, out[0]) and torch.equal(w, out[1]) and torch.equal(grad, router.backward(l, e, gw))
