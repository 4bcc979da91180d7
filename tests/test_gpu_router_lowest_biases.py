"""Groups that count with the sum of their two best, where that sum is beyond fp32: biases near the lowest (and the largest) number
of the type, as masks.  The ranking is that of 64 bits, in which such a sum is a number like others; only a group in which nobody can
be chosen counts -inf."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_router import INF, _check, _logits           # noqa: E402

LOWEST = torch.finfo(torch.float32).min


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


# groups of whole lanes (8 and 32 experts a group, one and two lanes), and groups that are not
LAYOUTS = [(64, 8), (256, 8), (4, 2), (16, 4), (60, 5), (500, 4)]


@pytest.mark.parametrize("E,G", LAYOUTS)
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("low", [LOWEST, -3e38, -1.75e38])
def test_a_masked_group_comes_before_one_without_experts(hl, E, G, score, low):
    per = E // G
    l = torch.zeros(7, E, device="cuda")
    l[:, :per] = -INF                                            # the first group has nobody
    l[1] = _logits(1, E, torch.float32, 3)[0]
    l[2, E - 1] = -INF
    l[3, per:] = torch.arange(E - per, device="cuda") * 1e-3
    l[4, per:E - per] = -INF                                     # nobody but in the last
    l[5] = -INF
    bias = torch.full((E,), low, device="cuda")
    bias[:per] = 0.0
    _check(hl, l, bias, top_k=min(2, per), score=score, G=G, TG=1, pair=True)
    if G > 2:
        _check(hl, l, bias, top_k=2, score=score, G=G, TG=2, pair=True)


@pytest.mark.parametrize("E,G", LAYOUTS)
@pytest.mark.parametrize("score", [0, 1])
@pytest.mark.parametrize("TG", [1, 2])
def test_sums_beyond_32_bits_are_ranked(hl, E, G, score, TG):
    if TG >= G and G > 2:
        pytest.skip("as many as there are")
    g = torch.Generator().manual_seed(E + G)
    values = torch.tensor([LOWEST, -3e38, -2.5e38, -1.7014119e38, -1e38, -INF, -1.5e38, 0.0])
    for seed in range(12):
        bias = values[torch.randint(0, 8 if seed % 3 == 0 else 5, (E,), generator=g)].cuda()
        if seed % 4 == 3:
            bias = -bias.clamp(min=LOWEST)                       # the same above
        l = _logits(40, E, torch.float32, seed)
        l[torch.rand(40, E, generator=g).cuda() < 0.3] = -INF
        _check(hl, l, bias, top_k=min(3, E // G * TG), score=score, G=G, TG=TG, pair=True)
