"""The clipping threshold is a number of 64 bits: the factor max_norm / (norm + 1e-6) is rounded to fp32 once."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_threshold_is_not_rounded_before_the_factor():
    """One tensor {1}: the norm is 1, exactly, and what is written is the factor: the fp32 number next to max_norm / (1 + 1e-6).  (A
    threshold rounded to fp32 first gives its neighbour for a good part of these.)"""
    import paper_2204_05436_b200 as hl
    stream = torch.cuda.current_stream().cuda_stream
    src, norm = torch.ones(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(hl.hl_grad_workspace_bytes(), dtype=torch.uint8, device="cuda")
    limits = np.random.RandomState(1).uniform(0.01, 1.0, 400)
    exact = (limits / (1.0 + 1e-6)).astype(np.float32)
    assert (exact != (limits.astype(np.float32).astype(np.float64) / (1.0 + 1e-6)).astype(np.float32)).sum() > 100
    out = torch.zeros(len(limits), device="cuda")
    for i, limit in enumerate(limits):
        hl.hl_grad_clip(hl.make_tensors([(src, out[i:i + 1])]), None, 0, float(limit), norm, ws, ws.numel(), stream)
    assert norm.item() == 1.0
    np.testing.assert_array_equal(out.cpu().numpy(), exact)


@pytest.mark.parametrize("limit", [0.0, 5e-324, 1e-60, 1e60, float("inf")])
def test_thresholds_outside_of_fp32(limit):
    import paper_2204_05436_b200 as hl
    stream = torch.cuda.current_stream().cuda_stream
    src, out, norm = torch.full((5,), 1e-3, device="cuda"), torch.zeros(5, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(hl.hl_grad_workspace_bytes(), dtype=torch.uint8, device="cuda")
    hl.hl_grad_clip(hl.make_tensors([(src, out)]), None, 0, limit, norm, ws, ws.numel(), stream)
    assert torch.equal(out, src if limit > 1 else torch.zeros_like(src))
