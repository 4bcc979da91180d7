"""What hl_expert_* and hl_grad_* refuse on the host, before anything is queued (no GPU needed)."""
import pytest


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


P = 0x7000_0000_0000                   # addresses that nothing is read from or written to
ROUTE = dict(max_tokens=100, n_tokens=P, top_k=2, n_experts=8, align=4, cap_rows=300, place=P, source=P, counts=P, offsets=P)


def _refused(hl, status, f, *a):
    with pytest.raises(hl.HotlineError) as e:
        f(*a)
    assert e.value.status == status


@pytest.mark.parametrize("change", [dict(max_tokens=-1), dict(max_tokens=2 ** 30), dict(max_tokens=2 ** 62), dict(top_k=0), dict(top_k=65),
                                    dict(max_tokens=2 ** 29, top_k=2), dict(n_experts=0), dict(n_experts=1025), dict(align=0),
                                    dict(align=65537), dict(cap_rows=-1), dict(cap_rows=2 ** 31), dict(place=None), dict(place=P + 2),
                                    dict(n_tokens=P + 1), dict(counts=P + 2), dict(offsets=P + 1), dict(source=P + 3)])
def test_routes(hl, change):
    r = hl.make_route(**{**ROUTE, **change})
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, r, P, 0, None, P, 1 << 40, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_dispatch, r, hl.HL_F32, 16, P, 16, P, 16, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine, r, hl.HL_F32, 16, P, 16, None, P, 16, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine_bwd, r, hl.HL_F32, 16, P, 16, P, 16, None, P, 16, None, None)


def test_sort(hl):
    r = hl.make_route(**ROUTE)
    need = hl.hl_expert_workspace_bytes(100, 2, 8)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, r, None, 0, None, P, need, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, r, P, -1, None, P, need, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, r, P + 1, 0, None, P, need, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, r, P, 0, P + 2, P, need, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, r, P, 0, None, None, need, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, r, P, 0, None, P + 128, need, None)
    _refused(hl, hl.HL_ECAPACITY, hl.hl_expert_sort, r, P, 0, None, P, need - 1, None)
    for missing in ("counts", "offsets"):
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_sort, hl.make_route(**{**ROUTE, missing: None}), P, 0, None, P, need, None)
    for bad in ((-1, 2, 8), (100, 0, 8), (100, 65, 8), (100, 2, 0), (100, 2, 1025), (2 ** 30, 1, 8), (2 ** 62, 64, 8)):
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_workspace_bytes, *bad)


def test_rows(hl):
    r = hl.make_route(**ROUTE)
    for dtype, dim, x, ldx, y, ldy in [(3, 16, P, 16, P, 16), (-1, 16, P, 16, P, 16), (0, 0, P, 16, P, 16), (0, 16, None, 16, P, 16),
                                       (0, 16, P, 15, P, 16), (0, 16, P, 16, None, 16), (0, 16, P, 16, P, 15),
                                       (0, 16, P + 2, 16, P, 16), (1, 16, P, 16, P + 1, 16), (0, 2 ** 25, P, 2 ** 25, P, 2 ** 25),
                                       (2, 16, P, 2 ** 32, P, 16)]:
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_dispatch, r, dtype, dim, x, ldx, y, ldy, None)
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine, r, dtype, dim, x, ldx, None, y, ldy, None)
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine_bwd, r, dtype, dim, x, ldx, P, max(dim, 1), None, y, ldy, None, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine_bwd, r, 0, 16, P, 16, None, 16, None, P, 16, P, None)      # y, for weights' gradient
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine, r, 0, 16, P, 16, P + 2, P, 16, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine_bwd, r, 0, 16, P, 16, P, 16, P + 1, P, 16, P, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine_bwd, r, 0, 16, P, 16, P, 16, P, P, 16, P + 2, None)
    for missing in ("counts", "offsets"):                                      # what fills experts up needs them
        q = hl.make_route(**{**ROUTE, missing: None})
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_dispatch, q, 0, 16, P, 16, P, 16, None)
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_combine_bwd, q, 0, 16, P, 16, P, 16, None, P, 16, None, None)


def _tensors(hl, *rows):
    return (hl.hl_tensor * len(rows))(*rows)


def test_gradient_lists(hl):
    T, need = hl.hl_tensor, hl.hl_grad_workspace_bytes()
    good = T(P, P, 10, 0, 0, 0, 0)
    bad = [T(None, P, 10, 0, 0, 0, 0), T(P + 2, P, 10, 0, 0, 0, 0), T(P, P + 2, 10, 1, 0, 0, 0), T(P, P, -1, 0, 0, 0, 0),
           T(P, P, 2 ** 40, 0, 0, 0, 0), T(P, P, 10, 3, 0, 0, 0), T(P, P, 10, 0, -1, 0, 0), T(P, P, 10, 0, 0, 2, 0),
           T(P, P, 10, 1, 2, 0, 0), T(P, P, 10, 0, 0, 0, 1)]
    for b in bad:
        for ts in (_tensors(hl, b), _tensors(hl, good, b)):
            _refused(hl, hl.HL_EINVAL, hl.hl_grad_norm, ts, None, 0, P, P, need, None)
            _refused(hl, hl.HL_EINVAL, hl.hl_grad_clip, ts, None, 0, 1.0, P, P, need, None)
    ts = _tensors(hl, good)
    for further, n, max_norm, norm, ws, size, status in [(None, 1, 1.0, P, P, need, -1), (P, -1, 1.0, P, P, need, -1),
                                                         (None, 0, -1.0, P, P, need, -1), (None, 0, float("nan"), P, P, need, -1),
                                                         (None, 0, 1.0, P, None, need, -1), (None, 0, 1.0, P, P + 8, need, -1),
                                                         (None, 0, 1.0, P, P, need - 1, -3), (P + 4, 1, 1.0, P, P, need, -1)]:
        _refused(hl, status, hl.hl_grad_clip, ts, further, n, max_norm, norm, ws, size, None)
        if max_norm == 1.0:
            _refused(hl, status, hl.hl_grad_norm, ts, further, n, norm, ws, size, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_grad_norm, ts, None, 0, None, P, need, None)


def test_lists_from_tensors(hl):
    torch = pytest.importorskip("torch")
    a, b = torch.zeros(6, 4), torch.zeros(24, dtype=torch.bfloat16)
    c = torch.zeros(24, dtype=torch.bfloat16)
    ts = hl.make_tensors([(a, None), (a, b), (c, c, hl.HL_TENSOR_NOT_IN_NORM)])
    assert [(t.n, t.src_dtype, t.dst_dtype, t.flags, bool(t.dst)) for t in ts] == [(24, 0, 0, 0, False), (24, 0, 1, 0, True),
                                                                                  (24, 1, 1, 1, True)]
    with pytest.raises(ValueError):
        hl.make_tensors([(a, b), (a.half(), b)])
    d = torch.zeros(6, 4)
    for bad in ([(a, d), (d, None)], [(d, None), (a, d)], [(a, a), (a, d)], [(a, d), (a, a)], [(a, a), (a, None)]):
        with pytest.raises(ValueError):
            hl.make_tensors(bad)
    hl.make_tensors([(a, d), (a, None), (a, torch.zeros(6, 4))])
    hl.make_tensors([(a, None), (a, None), (torch.zeros(0), torch.zeros(0)), (torch.zeros(0), torch.zeros(0))])
    for bad, error in [((a.t(), None), ValueError), ((a, torch.zeros(23)), ValueError), ((a, b[::2]), ValueError),
                       ((a.double(), None), TypeError), ((a, torch.zeros(24, dtype=torch.int32)), TypeError)]:
        with pytest.raises(error):
            hl.make_tensors([bad])
    assert hl.dtype_of(a) == hl.HL_F32 and hl.dtype_of(a.half()) == hl.HL_F16


def test_row_gradients(hl):
    _refused(hl, hl.HL_EINVAL, hl.hl_embbag_grad_sumsq, None, P, P, P, P, P, None)
