"""The gradient of a softmax over all experts (no sum of the chosen below), row by row: where the chosen ones have nearly all of it or
next to nothing, what is left is small, and has to be right all the same.  Tolerance: test_gpu_router_gradient_rows.py's, with shares
over all experts and a gradient of 0 for those that were not chosen."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_router import S, _check, _formula, _logits   # noqa: E402
from tests.test_gpu_router_gradient_rows import _check_rows      # noqa: E402


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


@pytest.mark.parametrize("K,E", [(2, 8), (3, 7), (8, 64), (8, 256), (20, 64), (8, 500)])
@pytest.mark.parametrize("apart", [0.0, 3.0, 9.0, 14.0, 30.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_expert_with_nearly_all(hl, K, E, apart, dtype):
    l = _logits(200, E, torch.float32, E + K)
    l[torch.arange(200), torch.arange(200) % E] += apart
    l = l.to(dtype)
    gw = torch.randn(200, K, generator=torch.Generator().manual_seed(K)).cuda()
    gw[::5] *= 1e4
    gw[1::5] = gw[1::5, :1]                                      # all alike
    router, e, _ = _check(hl, l, top_k=K, renorm=False, scale=2.5)
    _check_rows(hl, l, e, gw, router, True, False, 2.5)


@pytest.mark.parametrize("E", [5, 64, 300])
def test_a_large_gradient_of_a_tiny_share(hl, E):
    K, T = 3, 6
    l = torch.full((T, E), -100.0, device="cuda")
    for t, (a, b, c) in enumerate([(0, 0, -50), (0, 0, -30), (0, -30, -31), (-1, 0, -20), (0, -0.5, -16), (0, -10, -12)]):
        l[t, :3] = torch.tensor([a, b, c])
    gw = torch.tensor([[1, 2, 1e8], [1, 1.001, 1e4], [1e6, 1, -1e6], [5, 5, 1e7], [-1, 1, 1e6], [0, 0, 1]], device="cuda")
    router, e, _ = _check(hl, l, top_k=K, renorm=False)
    _check_rows(hl, l, e, gw, router, True, False, 1.0)


@pytest.mark.parametrize("K,E", [(1, 8), (2, 16), (8, 64), (8, 256), (8, 600)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_softmax_over_all_with_a_bias(hl, K, E, dtype):
    """The expert with nearly all of the softmax chosen, and not chosen (a bias against it), and all but nothing of it chosen."""
    l = _logits(120, E, dtype, E)
    l[:, 1] += 12.0
    l[::3, 1] -= 12.0
    gw = torch.randn(120, K, generator=torch.Generator().manual_seed(K)).cuda()
    gw[40:80] = 1.5
    for against in (0.0, -3.0):
        bias = torch.zeros(E, device="cuda")
        bias[1] = against
        router, e, _ = _check(hl, l, bias, top_k=K, renorm=False)
        _check_rows(hl, l, e, gw, router, True, False, 1.0)
    few = l.clone()
    few[:, K:] = -15.0                                           # what is not chosen has next to nothing
    router, e, _ = _check(hl, few, top_k=K, renorm=False)
    _check_rows(hl, few, e, gw, router, True, False, 1.0)
    _check_rows(hl, few, e, torch.ones_like(gw), router, True, False, 1.0)


def test_chosen_twice_in_a_softmax_over_all(hl):
    l = _logits(4, 16, torch.float32, 3)
    l[0, 1] = l[1, 5] = 15.0
    gw = torch.randn(4, 3, generator=torch.Generator().manual_seed(2)).cuda()
    e = torch.tensor([[1, 1, 2], [5, 5, 5], [0, 3, 0], [7, 2, 2]], dtype=torch.int32).cuda()
    router = hl.make_router(0, 3, 16, renorm=False)
    # (what is taken from an expert's gradient is taken from its first place's: D counts its gradients one by one)
    out = torch.zeros(4, 16, device="cuda")
    hl.hl_expert_choose_bwd(router, hl.HL_F32, l, 16, 4, None, e, gw, out, 16, torch.cuda.current_stream().cuda_stream)
    want = _formula(l, e, gw, True, False, 1.0)
    assert (out.double() - want).abs().max() < (20 + 2 * 37 + 24) * 4 * S * 2 * float(gw.abs().sum(dim=1).max())
