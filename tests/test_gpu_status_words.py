"""status() of the classes with a word of their own: when it returns the word is HL_OK again, so that an error of a call that is made next, on
whatever stream, is not cleared with what was told."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _all(hl):
    return [hl.ExpertRouter(2, 8), hl.TokenEmbedding(10, 10, 8), hl.Mx4Weights(torch.ones(2, 8, 32, device="cuda"))]


def test_the_word_is_cleared_when_status_returns(hl):
    for own in _all(hl):
        stream = torch.cuda.Stream()
        for _ in range(300):
            with torch.cuda.stream(stream):
                own._status.fill_(hl.HL_EINVAL)
                assert own.status(raise_on_error=False) == hl.HL_EINVAL
            assert stream.query()
            assert own.status(raise_on_error=False) == hl.HL_OK


def test_an_error_on_another_stream_right_after(hl):
    router, embedding = hl.ExpertRouter(2, 8), hl.TokenEmbedding(10, 10, 8)
    bad = torch.full((4, 8), float("nan"), device="cuda")
    table, tokens = torch.ones(10, 8, device="cuda"), torch.full((3,), 11, dtype=torch.int32, device="cuda")
    out = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda")
    rows = torch.zeros(3, 8, device="cuda")
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(50):
        with torch.cuda.stream(first):
            router.status(raise_on_error=False)
            embedding.status(raise_on_error=False)
        with torch.cuda.stream(second):
            router.choose(bad, out=out)
            embedding.embed(table, tokens, out=rows)
        with torch.cuda.stream(first):
            assert router.status(raise_on_error=False) == hl.HL_EINVAL
            assert embedding.status(raise_on_error=False) == hl.HL_EBOUNDS
