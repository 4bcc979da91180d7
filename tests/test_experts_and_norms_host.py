"""What ExpertRoute and Hotline check and allocate before anything is queued, on tensors in host memory with the library's calls
taken out (no GPU needed)."""
import pytest
import torch


@pytest.fixture(scope="module")
def hl():
    import importlib.util
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("hotline_build", os.path.join(root, "paper_2204_05436_b200", "csrc", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    build.build_library()
    import paper_2204_05436_b200 as hl
    return hl


@pytest.fixture
def route(hl):
    """A route of 8 tokens, two of four experts each, whose calls go to `calls`."""
    r = hl.ExpertRoute.__new__(hl.ExpertRoute)
    r.device = torch.device("cpu")
    r.max_tokens, r.top_k, r.n_experts, r.align, r.cap_rows = 8, 2, 4, 1, 16
    i32 = dict(dtype=torch.int32)
    r.place, r.source = torch.full((8, 2), -1, **i32), torch.full((16,), -1, **i32)
    r.counts, r.offsets = torch.zeros(4, **i32), torch.zeros(5, **i32)
    r.calls = []
    r._call = lambda f, *a: r.calls.append((f, a))
    r._set(8, None)
    return r


@pytest.mark.parametrize("default", [torch.float32, torch.bfloat16, torch.float16, torch.float64])
@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16, torch.float16])
def test_gradients_of_weights_are_fp32_whatever_torchs_default(route, rows, default):
    x, y, w = torch.zeros(8, 6, dtype=rows), torch.zeros(16, 6, dtype=rows), torch.zeros(8, 2, dtype=torch.float32)
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        grad_y, grad_w = route.combine_backward(x, y, w)
        others = route.dispatch(x), route.combine(y, w), route.dispatch_backward(y)
    finally:
        torch.set_default_dtype(before)
    assert grad_w.dtype == torch.float32 and grad_w.shape == (8, 2)
    assert grad_y.dtype == rows and all(t.dtype == rows for t in others)
    assert len(route.calls) == 4
