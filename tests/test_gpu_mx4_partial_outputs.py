"""The experts' product where a warp's last lanes have no output (outputs that are no multiple of 32) and the others go on storing
rows for several rounds: every warp reads the tensor memory as a whole each time.  Tolerances: test_gpu_mx4.py's."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_mx4 import TYPES, _Case                      # noqa: E402


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


@pytest.mark.parametrize("F", [1, 9, 31, 33, 95, 105, 127, 137, 1001])
@pytest.mark.parametrize("dtype", TYPES)
def test_rounds_of_partial_warps(hl, F, dtype):
    """65 to 240 rows a tile: two to four rounds of 32, whole and cut ones."""
    for T, E in ((65, 1), (97, 1), (240, 1), (400, 3), (700, 2)):
        c = _Case(hl, T, 1, E, 96, F, dtype, none=0.0, seed=F)
        c.check(True)
        c.check(False)
        first = c.y.clone()
        c.run(False)
        assert torch.equal(c.y, first)


def test_partial_warps_of_rows_that_fill_up(hl):
    c = _Case(hl, 900, 2, 4, 300, 137, torch.bfloat16, align=128, pad=3, at=1)
    c.check(True)
    c.check(False)
