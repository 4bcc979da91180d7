"""A NaN among the biases says HL_EINVAL whatever the logits are; logits of -inf and infinite biases by themselves do not."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_router import INF, _check, _logits           # noqa: E402


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


@pytest.mark.parametrize("E,G", [(5, 1), (8, 1), (64, 8), (60, 5), (256, 8), (515, 1), (1000, 1)])
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("pair", [False, True])
def test_a_nan_bias_of_an_expert_without_a_logit(hl, E, G, score, pair):
    for dtype in (torch.float32, torch.bfloat16):
        l = _logits(9, E, dtype, E)
        for at in (0, E // 2, E - 1):
            masked = l.clone()
            masked[:, at] = -INF
            bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(E)).cuda()
            _check(hl, masked, bias, top_k=2, score=score, G=G, pair=pair)
            bias[at] = float("nan")
            _check(hl, masked, bias, top_k=2, score=score, G=G, pair=pair, bad=True)
            _check(hl, masked, bias, live=1, top_k=2, score=score, G=G, pair=pair, bad=True)
            _check(hl, masked, bias, live=0, top_k=2, score=score, G=G, pair=pair)


@pytest.mark.parametrize("E,G", [(5, 1), (64, 8), (60, 5), (256, 8), (515, 1)])
@pytest.mark.parametrize("score", [0, 1])
def test_rows_without_experts_and_infinite_biases_say_nothing(hl, E, G, score):
    l = _logits(9, E, torch.float32, E)
    l[::2] = -INF
    l[3, 0] = INF
    bias = torch.zeros(E, device="cuda")
    bias[1], bias[2] = INF, -INF
    for pair in (False, True):
        for rows in (l, l[::2].contiguous()):
            _check(hl, rows, bias, top_k=2, score=score, G=G, pair=pair)
