"""Rows that fill experts up are part of what cap_rows has to hold: a product that walks tiles of `align` rows reads and writes them."""
import numpy as np
import pytest
import torch

from tests.test_gpu_experts import _choices, _Route

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


@pytest.mark.parametrize("last", ["the last has some", "the last has none", "capped"])
@pytest.mark.parametrize("T,K,E", [(1, 3, 1), (20, 2, 4), (3000, 2, 17), (20_000, 2, 64), (60_000, 2, 100)],
                         ids=["one CTA, one expert", "one CTA", "eight CTAs", "sixteen CTAs", "three kernels"])
def test_rows_that_fill_up_have_to_fit(hl, T, K, E, last):
    align, n = 16, T * K
    e = _choices(T, K, max(1, E - (last == "the last has none")), 3, skew=0.4)
    limit = int(np.bincount(e.reshape(-1)).max()) - 1 if last == "capped" else 0
    counts = np.bincount(e.reshape(-1), minlength=E)
    counts = np.minimum(counts, limit) if limit else counts
    owner = int(np.flatnonzero(counts)[-1])                    # whose rows are the last
    if counts[owner] % align == 0:                             # (its rows are to need filling up: one choice of its goes elsewhere)
        e.reshape(-1)[np.flatnonzero(e.reshape(-1) == owner)[-1]] = -1
        counts = np.bincount(e[e >= 0], minlength=E)
        counts = np.minimum(counts, limit) if limit else counts
    filled = -(-counts // align) * align
    full = int(filled.sum())
    end = full - int(filled[owner]) + int(counts[owner])       # behind the last choice
    assert counts[owner] % align and end < full
    for rows in (full + 1, full, full - 1, end, end - 1):
        p = _Route(hl, T, K, E, align, cap_rows=rows)
        p.sort(torch.from_numpy(e).cuda(), limit)
        torch.cuda.synchronize()
        assert p.status.item() == (hl.HL_OK if rows >= full else hl.HL_ECAPACITY), (rows, full, end)
        np.testing.assert_array_equal(p.offsets.cpu().numpy()[:E + 1], np.minimum(np.append(0, np.cumsum(filled)), rows))
        # every choice that is kept has its row, as long as there is one
        assert int((p.place[:n] >= 0).sum()) == int(counts.sum()) - max(0, end - rows)
        assert (p.source[rows:] == -7).all() and (p.source[end:min(full, rows)] == -1).all()
