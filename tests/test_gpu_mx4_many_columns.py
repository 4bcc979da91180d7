"""The product's rows in 4 bits where a warp takes eight parts of a row at a time (seven tiles of 256 columns and more, of enough rows to fill
the chip), and two such turns one behind the other (of eight times as many): whole last turns and cut ones.  Tolerances: test_gpu_mx4.py's."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_mx4 import TYPES, _Case                      # noqa: E402


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


# one turn of seven parts, of eight, two of which the last has two, one of 148 x 3 x 8 rows exactly and one less
@pytest.mark.parametrize("T,K,dim", [(4000, 1, 1537), (4000, 2, 2048), (4001, 1, 2500), (3552, 1, 1792), (3551, 1, 1792), (1777, 2, 2304)])
@pytest.mark.parametrize("pad,at", [(0, 0), (8, 8), (5, 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_eight_parts_at_a_time(hl, T, K, dim, pad, at, dtype):
    c = _Case(hl, T, K, 7, dim, 40, dtype, align=16, pad=pad, at=at)
    c.check(True)
    c.check(False)


# two turns: of 3 each row one and a half, of 4, of 1
@pytest.mark.parametrize("T,dim", [(9600, 4500), (7200, 8192), (28_500, 1800)])
@pytest.mark.parametrize("pad,at", [(0, 0), (5, 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_two_turns(hl, T, dim, pad, at, dtype):
    c = _Case(hl, T, 1, 3, dim, 24, dtype, pad=pad, at=at, live=T - 7, none=0.02)
    c.check(True)
    c.check(False)
