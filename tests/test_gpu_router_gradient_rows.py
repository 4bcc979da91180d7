"""The router's gradient row by row: what one expert with nearly all of a token's share leaves to the others is small, and has to be
right all the same.

Tolerance.  A logit's gradient does not change when the same number b is taken from every expert's gradient (shares add up to 1); with b
that of the expert with the largest share, g_l = scale share_l (d_l - sum_j share_j d_j) (1 - s_l for renormalised sigmoids) with d = g - b,
of which no term is larger than D = scale sum_j share_j |d_j| over all experts that a token's shares add up to 1 over.  With s = 2^-24
each term is off by what test_gpu_router.py gives a share -- (R + n + 16) 2 s, the logits' range R, n terms added up --, a difference's
rounding and the sum's n; two of them make (R + 2 n + 24) 4 s of D, plus half a step of the logits' type (2^-25 of fp16 below its normal
range, 2^-126 of others)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_router import INF, S, _check, _formula, _logits        # noqa: E402


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _distance(l, e, gw, softmax, renorm, scale):
    """D of every row, in 64 bits."""
    l, gw = torch.where(torch.isnan(l), -INF, l.double()), gw.double()
    valid = e >= 0
    at = e.clamp(min=0).long()
    if renorm:
        key = l if softmax else torch.nn.functional.logsigmoid(l)
        c = torch.where(valid, key.gather(1, at), -INF)
        share, g = torch.softmax(c.masked_fill(~valid.any(dim=1, keepdim=True), 0.0), dim=1), torch.where(valid, gw, 0.0)
    else:
        share = torch.softmax(l.masked_fill((l == -INF).all(dim=1, keepdim=True), 0.0), dim=1)
        g = torch.zeros_like(share).scatter_add_(1, at, torch.where(valid, gw, 0.0))
    most = share == share.amax(dim=1, keepdim=True)              # (of several, any may be taken)
    low, high = (torch.where(most, g, sign * INF).aminmax(dim=1, keepdim=True)[i] for i, sign in ((0, 1.0), (1, -1.0)))
    return scale * (share * torch.maximum((g - low).abs(), (g - high).abs())).sum(dim=1, keepdim=True)


def _check_rows(hl, l, e, gw, router, softmax, renorm, scale):
    T, E = l.shape
    out = torch.full((T, E), -7.0, dtype=l.dtype, device="cuda")
    hl.hl_expert_choose_bwd(router, hl.dtype_of(l), l, E, T, None, e, gw, out, E, torch.cuda.current_stream().cuda_stream)
    want = _formula(l, e, gw, softmax, renorm, scale)
    finite = l[torch.isfinite(l)].double()
    R = min(float(finite.max() - finite.min()), 200.0)
    n = e.shape[1] if renorm else 32 + 5
    half = torch.finfo(l.dtype).eps / 2 * want.abs() + (2.0 ** -25 if l.dtype == torch.float16 else 2.0 ** -126)
    # (the formula's own 64 bits: the same factor of what it adds up, 2^-53 a rounding)
    own = (R + 2 * n + 24) * 4 * 2.0 ** -53 * scale * gw.abs().double().amax(dim=1, keepdim=True)
    tol = (R + 2 * n + 24) * 4 * S * _distance(l, e, gw, softmax, renorm, scale) + half + own
    err = (out.double() - want).abs()
    assert (err <= tol).all(), (float((err / tol).max()), int((err / tol).max(dim=1).values.argmax()))
    return out


MODES = [(0, True), (1, True)]                                   # score, renorm


@pytest.mark.parametrize("K,E", [(2, 8), (3, 7), (8, 64), (8, 256), (20, 64), (8, 500)])
@pytest.mark.parametrize("score,renorm", MODES)
@pytest.mark.parametrize("apart", [0.0, 3.0, 9.0, 14.0, 30.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_expert_with_nearly_all(hl, K, E, score, renorm, apart, dtype):
    l = _logits(200, E, torch.float32, E + K)
    l = l - apart if score else l                                # (sigmoids: shares differ where logits are below 0)
    l[torch.arange(200), torch.arange(200) % E] += apart
    l = l.to(dtype)
    gw = torch.randn(200, K, generator=torch.Generator().manual_seed(K)).cuda()
    gw[::5] *= 1e4
    gw[1::5] = gw[1::5, :1]                                      # all alike
    router, e, _ = _check(hl, l, top_k=K, score=score, renorm=renorm, scale=2.5)
    _check_rows(hl, l, e, gw, router, score == 0, renorm, 2.5)


@pytest.mark.parametrize("score,renorm", MODES)
@pytest.mark.parametrize("E", [5, 64, 300])
def test_a_large_gradient_of_a_tiny_share(hl, score, renorm, E):
    K, T = 3, 6
    l = torch.full((T, E), -100.0, device="cuda")
    for t, (a, b, c) in enumerate([(0, 0, -50), (0, 0, -30), (0, -30, -31), (-1, 0, -20), (0, -0.5, -16), (0, -10, -12)]):
        l[t, :3] = torch.tensor([a, b, c]) - (20.0 if score else 0.0)
    gw = torch.tensor([[1, 2, 1e8], [1, 1.001, 1e4], [1e6, 1, -1e6], [5, 5, 1e7], [-1, 1, 1e6], [0, 0, 1]], device="cuda")
    router, e, _ = _check(hl, l, top_k=K, score=score, renorm=renorm)
    _check_rows(hl, l, e, gw, router, score == 0, renorm, 1.0)
    if (score, renorm) == (0, True):
        out = _check_rows(hl, l[:1], e[:1], gw[:1], router, True, True, 1.0)
        assert torch.allclose(out[0, :2].cpu(), torch.tensor([-0.25, 0.25]), rtol=1e-5)
