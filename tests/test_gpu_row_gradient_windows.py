"""hl_embbag_grad_sumsq where runs of lookups end at the borders of the kernel's windows: 512 lookups for rows of up to 16 values, 256
for up to 64, 128 beyond (tolerance: that of the other tests of the call, sums in fp64)."""
import numpy as np
import pytest

from tests.test_gpu_grad_norm import _check_rows

pytestmark = pytest.mark.gpu

WINDOW = {4: 512, 16: 512, 20: 256, 32: 256, 36: 256, 64: 256, 68: 128, 128: 128, 260: 128}


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


@pytest.mark.parametrize("D", WINDOW)
def test_runs_that_end_at_a_windows_border(hl, D):
    w = WINDOW[D]
    for lengths in ([w], [w, 1], [1, w], [w, w], [w - 1, w + 1, 1], [w + 1, 2 * w, w - 1], [w // 2, w, w // 2], [3 * w, 1, 3 * w - 1, 5],
                    [w - 1, 1, w - 1, 1], [1] * (w - 1) + [2] + [1] * (w - 1), [w - 8] + [8] * 4 + [w - 24, w]):
        _check_rows(hl, np.repeat(np.arange(len(lengths)), lengths), D)


@pytest.mark.parametrize("D", WINDOW)
def test_runs_of_few_and_many_windows(hl, D):
    """Up to 32 windows behind the one in which it starts a run is joined by a warp, beyond by a CTA of 256 threads."""
    w = WINDOW[D]
    for windows in (2, 31, 32, 33, 34, 35, 255 + 33, 256 + 33, 257 + 33, 600):
        for lengths in ([windows * w], [5, windows * w, 5], [w - 1, windows * w + 1, 3], [1, windows * w - 1, w + 7]):
            n = sum(lengths)
            _check_rows(hl, np.repeat(np.arange(len(lengths)), lengths), D, bags=np.arange(n) * 7 % 1001, batch=1001)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_several_long_runs_with_lookups_that_add_nothing(hl, D):
    w = WINDOW[D]
    lengths = [40 * w + 3, 2, 33 * w, 5 * w - 1, 300 * w + 1, 1, 7]
    n = sum(lengths)
    bags = np.arange(n) * 11 % 997
    bags[::13] = -1
    bags[5::1009] = 2 ** 31 - 1
    _check_rows(hl, np.repeat(np.arange(len(lengths)) * 2, lengths), D, bags=bags, batch=997)
