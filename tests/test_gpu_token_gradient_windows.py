"""The token embedding's gradient where the windows of sorted tokens are longer than 16: 32, 64 and 128, by many values and by many
tokens, with runs of lengths around the windows' and around the 16 windows from which on a run is the whole CTA's.  Tolerances:
test_gpu_token_embedding.py's."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_token_embedding import BF16, F16, F32, _Backward, _rows  # noqa: E402


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _runs(n, w, seed):
    """n tokens in an order of their own, and how many rows they name: runs around multiples of w, and one of what is left."""
    some = [1, w - 1, w, w + 1, 2 * w, 2, 3 * w + 1, 15 * w, 16 * w - 1, 16 * w, 3, 16 * w + 1, 17 * w + 1, 31 * w, w // 2, 40 * w]
    lengths, left = [], n
    while left > max(some):
        lengths.append(some[len(lengths) % len(some)])
        left -= lengths[-1]
    lengths.append(left)
    tokens = torch.repeat_interleave(torch.arange(len(lengths)), torch.tensor(lengths))
    return tokens[torch.randperm(n, generator=torch.Generator().manual_seed(seed))].int().cuda(), len(lengths)


def _check(hl, n, w, dim, dtype, pad=0, at=0):
    tokens, rows = _runs(n, w, n)
    V = rows + 50
    b = _Backward(hl, tokens, V, dim, live=n - 3)
    grad_out = _rows(n, dim, dtype, pad, at, 1)
    table = torch.full((V, dim), 3.0, device="cuda")
    b.check(grad_out, 1.5, table)
    again = torch.full((V, dim), 4.0, device="cuda")
    b(grad_out, 1.5, again)
    assert torch.equal(table, again)
    b.check(grad_out, -0.5, table, accumulate=True)
    low = torch.zeros(V, dim, dtype=dtype, device="cuda")
    b.check(grad_out, 1.0, low)


# (the windows' threads, of eight columns, fill the chip more than once: 303 104 of them)
@pytest.mark.parametrize("n,w", [(18_800, 16), (20_000, 32), (40_000, 64), (80_000, 128)])
@pytest.mark.parametrize("dim,dtype", [(2056, BF16), (2056, F32), (2051, F16), (2051, F32)])
def test_windows_by_values(hl, n, w, dim, dtype):
    _check(hl, n, w, dim, dtype)


# (more than 8 192 windows)
@pytest.mark.parametrize("n,w", [(131_072, 16), (131_073, 32), (262_145, 64), (524_289, 128), (1_200_000, 128)])
@pytest.mark.parametrize("dim,dtype,pad,at", [(8, BF16, 0, 0), (24, F32, 0, 0), (13, F16, 3, 1), (37, F32, 0, 0)])
def test_windows_by_tokens(hl, n, w, dim, dtype, pad, at):
    _check(hl, n, w, dim, dtype, pad, at)
