"""What hl_expert_mx4_checked refuses on the host: all that hl_expert_mx4 does, and a status word out of place (no GPU needed)."""
import pytest

from tests.test_refusals_tokens_router_mx4 import P, PRODUCT, ROUTE, _refused, hl  # noqa: F401


@pytest.mark.parametrize("change", [
    dict(dtype=3), dict(dim=0), dict(outputs=0), dict(x=None), dict(ld_x=63), dict(weights=P + 8), dict(y=None), dict(ld_y=31), dict(ws=None),
    dict(status=P + 2), dict(status=P + 1)])
def test_products(hl, change):                                   # noqa: F811
    args = {k: v for k, v in PRODUCT.items() if k != "stream"}
    args.update(status=P, stream=None)
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_mx4_checked, hl.make_route(**ROUTE), *{**args, **change}.values())
    _refused(hl, hl.HL_EINVAL, hl.hl_expert_mx4_checked, None, *args.values())
    need = hl.hl_expert_mx4_workspace_bytes(300, 8, 64)
    _refused(hl, hl.HL_ECAPACITY, hl.hl_expert_mx4_checked, hl.make_route(**ROUTE), *{**args, "ws_bytes": need - 1}.values())
