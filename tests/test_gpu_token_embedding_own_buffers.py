"""TokenEmbedding's own order is read and written by its calls: it is refused as a count of tokens, and as a table's gradient."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_own_buffers_are_refused():
    import paper_2204_05436_b200 as hl
    emb = hl.TokenEmbedding(64, 8, 4)
    tokens = torch.arange(32, dtype=torch.int32, device="cuda") % 8
    emb.sort(tokens)
    for own in (emb.sorted, emb.order):
        with pytest.raises(ValueError):
            emb.sort(tokens, own[3:4])
        with pytest.raises(ValueError):
            emb.sort(own[:32])
        emb.sort(tokens)
        with pytest.raises(ValueError):
            emb.backward(torch.ones(32, 4, device="cuda"), grad_table=own[:32].view(torch.float32).view(8, 4))
    assert torch.equal(emb.backward(torch.ones(32, 4, device="cuda")), torch.full((8, 4), 4.0, device="cuda"))
    empty = hl.TokenEmbedding(0, 8, 4)
    empty.sort(tokens[:0])
    assert (empty.backward(torch.ones(0, 4, device="cuda")) == 0).all()
