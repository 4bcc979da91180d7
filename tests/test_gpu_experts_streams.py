"""ExpertRoute.status() waits for the last sort, whatever stream it was queued on."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_status_waits_for_a_sort_on_another_stream():
    import paper_2204_05436_b200 as hl
    r = hl.ExpertRoute(300, 2, 6)
    good = torch.randint(0, 6, (300, 2), dtype=torch.int32, device="cuda")
    bad = torch.full((300, 2), 6, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for experts, status in [(bad, hl.HL_EBOUNDS), (good, hl.HL_OK), (bad, hl.HL_EBOUNDS)]:
        with torch.cuda.stream(s):
            torch.cuda._sleep(200_000_000)                     # (some 100 ms)
            r.sort(experts)
        assert r.status(False) == status
        assert torch.cuda.current_stream() != s
    # a sort that is a graph's, replayed on the current stream
    with torch.cuda.stream(s):
        r.sort(good)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        r.sort(bad)
    assert r.status(False) == hl.HL_OK
    torch.cuda._sleep(200_000_000)
    g.replay()
    assert r.status(False) == hl.HL_EBOUNDS
