"""The status of the experts' products: one whose wait ran out stays known until it is asked for, whatever products follow it.  (The
word that such a product writes is written here; no product is made to wait in vain.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _one(hl, T, K=2, E=4, dim=96):
    route = hl.ExpertRoute(T, K, E)
    route.sort(torch.randint(0, E, (T, K), device="cuda").int())
    return route, torch.randn(T, dim, device="cuda").to(BF16)


def test_kept_over_later_products_and_larger_workspaces(hl):
    weights = hl.Mx4Weights(torch.randn(4, 64, 96, device="cuda").to(BF16))
    assert weights.status() == hl.HL_OK
    route, x = _one(hl, 30)
    y = weights.product(route, x)
    assert weights.status() == hl.HL_OK
    weights._status.fill_(hl.HL_ETIMEOUT)
    weights._ws[-1][:4].view(torch.int32).fill_(hl.HL_ETIMEOUT)
    assert torch.equal(weights.product(route, x), y)
    larger, rows = _one(hl, 3000)
    weights.product(larger, rows)
    few, row = _one(hl, 1)                                       # (one kernel)
    weights.product(few, row)
    assert weights.status(raise_on_error=False) == hl.HL_ETIMEOUT
    assert weights.status() == hl.HL_OK                          # (told once)
    weights.product(route, x)
    assert weights.status() == hl.HL_OK
    weights._status.fill_(hl.HL_ETIMEOUT)
    with pytest.raises(hl.HotlineError):
        weights.status()


@pytest.mark.parametrize("T", [0, 1, 5, 300])
def test_the_word_is_left_alone(hl, T):
    """Through the C boundary, plain and replayed; without a word, too."""
    E, F, dim = 4, 40, 96
    w = torch.randn(E * F, dim, device="cuda").to(BF16)
    q = torch.empty(E * hl.hl_mx4_bytes(F, dim), dtype=torch.uint8, device="cuda")
    hl.hl_mx4_quantise(hl.HL_BF16, E, F, dim, w, dim, F * dim, q, torch.cuda.current_stream().cuda_stream)
    route, x = _one(hl, T)
    cap = route.cap_rows
    y, ws = torch.zeros(cap, F, dtype=BF16, device="cuda"), torch.empty(hl.hl_expert_mx4_workspace_bytes(cap, E, dim), dtype=torch.uint8,
                                                                        device="cuda")
    status = torch.zeros(3, dtype=torch.int32, device="cuda")

    def run(word):
        hl.hl_expert_mx4_checked(route._route, hl.HL_BF16, dim, F, x, dim, True, q, y, F, ws, ws.numel(), word,
                                 torch.cuda.current_stream().cuda_stream)

    run(None)
    plain = y.clone()
    for value in (hl.HL_OK, hl.HL_ETIMEOUT):
        status.fill_(value)
        y.zero_()
        run(status[1:])
        torch.cuda.synchronize()
        assert (status == value).all() and torch.equal(y, plain) and int(ws[:4].view(torch.int32)) == hl.HL_OK
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(status[1:])
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert (status == value).all() and torch.equal(y, plain)
        del graph
