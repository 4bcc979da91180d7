"""What hl_token_*, hl_expert_choose* and hl_*mx4* refuse on the host, before anything is queued (no GPU needed)."""
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
BIG = 1 << 50


def _refused(hl, status, f, *a):
    with pytest.raises(hl.HotlineError) as e:
        f(*a)
    assert e.value.status == status


def _with(args, **change):
    return list({**args, **change}.values())


EMBED = dict(table_dtype=0, n_rows=100, dim=16, table=P, ld_table=16, tokens=P, max_tokens=10, n_tokens=P, scale=1.0, out_dtype=1,
             out=P, ld_out=16, status=P, stream=None)


@pytest.mark.parametrize("change", [
    dict(table_dtype=3), dict(table_dtype=-1), dict(out_dtype=4), dict(n_rows=-1), dict(n_rows=2 ** 31), dict(dim=0), dict(dim=2 ** 25),
    dict(table=None), dict(table=P + 2), dict(ld_table=15), dict(ld_table=2 ** 32), dict(tokens=None), dict(tokens=P + 2),
    dict(max_tokens=-1), dict(max_tokens=2 ** 30), dict(n_tokens=P + 1), dict(out=None), dict(out=P + 1), dict(ld_out=15),
    dict(status=P + 2)])
def test_embed(hl, change):
    _refused(hl, hl.HL_EINVAL, hl.hl_token_embed, *_with(EMBED, **change))


def test_no_tokens(hl):
    hl.hl_token_embed(*_with(EMBED, max_tokens=0, tokens=None, out=None))
    hl.hl_token_sort(None, 0, None, 100, None, None, None, P, BIG, None)
    r = hl.make_router(hl.HL_SCORE_SOFTMAX, 2, 8)
    hl.hl_expert_choose(r, 0, None, 8, None, 0, None, None, None, None, None)
    hl.hl_expert_choose_bwd(r, 0, None, 8, 0, None, None, None, None, 8, None)
    hl.hl_mx4_quantise(0, 3, 0, 16, None, 16, 0, None, None)
    hl.hl_mx4_quantise(0, 0, 3, 16, None, 16, 0, None, None)
    hl.hl_mx4_dequantise(0, 3, 16, None, 0, None, 16, 0, None)


SORT = dict(tokens=P, max_tokens=1000, n_tokens=None, n_rows=100, sorted=P, order=P, status=None, ws=P, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("change", [
    dict(tokens=None), dict(tokens=P + 1), dict(max_tokens=-1), dict(max_tokens=2 ** 30), dict(n_tokens=P + 2), dict(n_rows=-1),
    dict(n_rows=2 ** 31), dict(sorted=None), dict(order=None), dict(sorted=P + 2), dict(order=P + 1), dict(status=P + 1), dict(ws=None),
    dict(ws=P + 128)])
def test_sort(hl, change):
    _refused(hl, hl.HL_EINVAL, hl.hl_token_sort, *_with(SORT, **change))


BWD = dict(n_rows=100, dim=16, sorted=P, order=P, max_tokens=1000, n_tokens=None, grad_dtype=1, grad=P, ld_grad=16, scale=1.0,
           table_dtype=0, table=P, ld_table=16, accumulate=False, ws=P, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("change", [
    dict(n_rows=-1), dict(n_rows=2 ** 31), dict(dim=0), dict(dim=2 ** 25), dict(sorted=None), dict(sorted=P + 1), dict(order=None),
    dict(order=P + 2), dict(max_tokens=-1), dict(max_tokens=2 ** 30), dict(n_tokens=P + 2), dict(grad_dtype=3), dict(grad=None),
    dict(grad=P + 1), dict(ld_grad=15), dict(table_dtype=-1), dict(table=None), dict(table=P + 2), dict(ld_table=15), dict(ws=None),
    dict(ws=P + 8)])
def test_embed_bwd(hl, change):
    _refused(hl, hl.HL_EINVAL, hl.hl_token_embed_bwd, *_with(BWD, **change))


def test_token_workspace(hl):
    need = hl.hl_token_workspace_bytes(1000, 16)
    _refused(hl, hl.HL_ECAPACITY, hl.hl_token_embed_bwd, *_with(BWD, ws_bytes=need - 1))
    _refused(hl, hl.HL_ECAPACITY, hl.hl_token_sort, *_with(SORT, ws_bytes=1023))
    for bad in ((-1, 16), (2 ** 30, 16), (10, 0), (10, 2 ** 25)):
        _refused(hl, hl.HL_EINVAL, hl.hl_token_workspace_bytes, *bad)


@pytest.mark.parametrize("dim", [1, 8, 337, 512, 4096, 100_000])
def test_a_workspace_does_for_fewer_tokens(hl, dim):
    """Also where fewer tokens are cut into shorter windows."""
    sizes = sorted({s for k in range(24) for s in (2 ** k - 1, 2 ** k, 2 ** k + 1, 3 * 2 ** k)} |
                   {w * 148 * 2048 * 8 // max(dim, 8) + d for w in (16, 32, 64, 128) for d in (-1, 0, 1)})
    needs = [hl.hl_token_workspace_bytes(n, dim) for n in sizes if 0 <= n < 2 ** 30]
    assert needs == sorted(needs)


ROUTER = dict(score=0, top_k=4, n_experts=64, n_groups=8, top_groups=4, group_score=0, renorm=True, scale=1.0)


@pytest.mark.parametrize("change", [
    dict(score=2), dict(score=-1), dict(top_k=0), dict(top_k=65), dict(n_experts=0), dict(n_experts=1025), dict(n_experts=1032),
    dict(n_groups=0), dict(n_groups=65, n_experts=130), dict(n_groups=7), dict(top_groups=0), dict(top_groups=9), dict(group_score=2),
    dict(top_k=33), dict(top_k=9, top_groups=1), dict(scale=float("nan")), dict(scale=float("inf")), dict(n_experts=3, n_groups=1,
                                                                                                         top_groups=1)])
def test_routers(hl, change):
    r = hl.make_router(*_with(ROUTER, **change))
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_choose, r, 0, P, 2000, None, 10, None, P, P, None, None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_choose_bwd, r, 0, P, 2000, 10, None, P, P, P, 2000, None)


CHOOSE = dict(dtype=1, logits=P, ld=64, bias=P, max_tokens=10, n_tokens=P, experts=P, weights=P, status=P, stream=None)
CHOOSE_BWD = dict(dtype=1, logits=P, ld=64, max_tokens=10, n_tokens=P, experts=P, grad_weights=P, grad=P, ld_grad=64, stream=None)


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(logits=P + 1), dict(ld=63), dict(ld=2 ** 31), dict(bias=P + 2),
    dict(max_tokens=-1), dict(max_tokens=2 ** 30), dict(max_tokens=2 ** 28), dict(n_tokens=P + 2), dict(experts=None),
    dict(experts=P + 2), dict(weights=None), dict(weights=P + 1), dict(status=P + 3), dict(grad_weights=None), dict(grad_weights=P + 2),
    dict(grad=None), dict(grad=P + 1), dict(ld_grad=63), dict(ld_grad=2 ** 31)])
def test_choose(hl, change):
    r = hl.make_router(*_with(ROUTER))
    for f, args in ((hl.hl_expert_choose, CHOOSE), (hl.hl_expert_choose_bwd, CHOOSE_BWD)):
        if set(change) <= set(args):
            _refused(hl, hl.HL_EINVAL, f, r, *_with(args, **change))
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_choose, None, *CHOOSE.values())
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_choose_bwd, None, *CHOOSE_BWD.values())


QUANTISE = dict(dtype=1, n=2, rows=100, dim=64, x=P, ld=64, stride=6400, q=P, stream=None)
DEQUANTISE = dict(n=2, rows=100, dim=64, q=P, dtype=1, out=P, ld=64, stride=6400, stream=None)


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(n=-1), dict(n=2 ** 31), dict(rows=-1), dict(rows=2 ** 31), dict(dim=0), dict(dim=2 ** 25), dict(x=None),
    dict(x=P + 1), dict(ld=63), dict(stride=-1), dict(q=None), dict(q=P + 8), dict(out=None), dict(out=P + 1),
    dict(n=2 ** 30, rows=2 ** 20)])
def test_matrices(hl, change):
    for f, args in ((hl.hl_mx4_quantise, QUANTISE), (hl.hl_mx4_dequantise, DEQUANTISE)):
        if set(change) <= set(args):
            _refused(hl, hl.HL_EINVAL, f, *_with(args, **change))


def test_matrix_bytes(hl):
    assert hl.hl_mx4_bytes(128, 256) == 17408 and hl.hl_mx4_bytes(129, 257) == 4 * 17408 and hl.hl_mx4_bytes(0, 5) == 0
    for bad in ((-1, 5), (2 ** 31, 5), (5, 0), (5, 2 ** 25)):
        _refused(hl, hl.HL_EINVAL, hl.hl_mx4_bytes, *bad)
    for bad in ((-1, 8, 64), (2 ** 31, 8, 64), (100, 0, 64), (100, 1025, 64), (100, 8, 0), (100, 8, 2 ** 25)):
        _refused(hl, hl.HL_EINVAL, hl.hl_expert_mx4_workspace_bytes, *bad)
    sizes = [hl.hl_expert_mx4_workspace_bytes(n, 64, 1000) for n in range(0, 2000)]
    assert sizes == sorted(sizes)


ROUTE = dict(max_tokens=100, n_tokens=P, top_k=2, n_experts=8, align=4, cap_rows=300, place=P, source=P, counts=P, offsets=P)
PRODUCT = dict(dtype=1, dim=64, outputs=32, x=P, ld_x=64, by_token=True, weights=P, y=P, ld_y=32, ws=P, ws_bytes=BIG, stream=None)


@pytest.mark.parametrize("change", [
    dict(max_tokens=-1), dict(max_tokens=2 ** 30), dict(max_tokens=2 ** 29), dict(top_k=0), dict(top_k=65), dict(n_experts=0),
    dict(n_experts=1025), dict(cap_rows=-1), dict(cap_rows=2 ** 31), dict(place=None), dict(place=P + 2), dict(counts=None),
    dict(counts=P + 1), dict(offsets=None), dict(offsets=P + 2), dict(n_tokens=P + 2)])
def test_product_routes(hl, change):
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_mx4, hl.make_route(**{**ROUTE, **change}), *PRODUCT.values())


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(dim=0), dict(dim=2 ** 25), dict(outputs=0), dict(outputs=2 ** 25), dict(x=None), dict(x=P + 1), dict(ld_x=63),
    dict(weights=None), dict(weights=P + 8), dict(y=None), dict(y=P + 1), dict(ld_y=31), dict(ws=None), dict(ws=P + 64)])
def test_products(hl, change):
    r = hl.make_route(**ROUTE)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_mx4, r, *_with(PRODUCT, **change))
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_mx4, None, *PRODUCT.values())
    need = hl.hl_expert_mx4_workspace_bytes(300, 8, 64)
    _refused(hl, hl.HL_ECAPACITY, hl.hl_expert_mx4, r, *_with(PRODUCT, ws_bytes=need - 1))
