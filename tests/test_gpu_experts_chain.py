"""Tokens to logits of a mixture of experts and back, with all calls as they are used together: embedding, router, plan, the
experts (in 4 bits when serving, the caller's when training), the weighted sums, and the gradients of all of it.

Tolerances: serving is compared step by step, each step's reference being computed from the device's result of the step before; training
goes through some thirty fp32 roundings between sums of at most 96 terms: 1e-4 of the largest value covers 1 600 of them, and
an error in a formula is far larger."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_mx4 import _definition                       # noqa: E402

S = 2.0 ** -24
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _near(a, b, rel):
    a, b = a.double(), b.double()
    return float((a - b).abs().max()) <= rel * max(float(b.abs().max()), 1e-30)


class _Model:
    def __init__(self, hl, V=500, D=96, E=16, K=4, H=160, T=200):
        g = torch.Generator(device="cuda").manual_seed(11)
        self.V, self.D, self.E, self.K, self.H, self.T = V, D, E, K, H, T
        self.table = (0.1 * torch.randn(V, D, generator=g, device="cuda"))
        self.gate = torch.randn(D, E, generator=g, device="cuda") / D ** 0.5
        self.bias = 0.05 * torch.randn(E, generator=g, device="cuda")
        self.up = torch.randn(E, H, D, generator=g, device="cuda").to(BF16) / D ** 0.5
        self.down = torch.randn(E, D, H, generator=g, device="cuda").to(BF16) / H ** 0.5
        self.emb = hl.TokenEmbedding(T, V, D)
        self.router = hl.ExpertRouter(K, E, score="sigmoid", n_groups=4, top_groups=2, group_score="top2", scale=1.5)
        self.route = hl.ExpertRoute(T, K, E, align=8)
        self.tokens = torch.randint(0, V, (T,), generator=g, device="cuda").int()
        self.count = torch.tensor([T - 13], dtype=torch.int32, device="cuda")


def test_serving(hl):
    m = _Model(hl)
    up, down, table = hl.Mx4Weights(m.up), hl.Mx4Weights(m.down), m.table.to(BF16)
    out = torch.zeros(m.T, m.D, dtype=BF16, device="cuda")
    keep = {}

    def step():
        x = m.emb.embed(table, m.tokens, m.D ** 0.5, m.count)
        logits = (x.float() @ m.gate).to(BF16)
        experts, weights = m.router.choose(logits, m.bias, m.count)
        m.route.sort(experts, m.count)
        y = up.product(m.route, x)
        z = torch.relu(y)
        w = down.product(m.route, z, by_token=False)
        m.route.combine(w, weights, out)
        keep.update(x=x, logits=logits, experts=experts, weights=weights, y=y, z=z, w=w)

    def check():
        assert m.emb.status() == m.router.status() == m.route.status() == up.status() == down.status() == hl.HL_OK
        n = int(m.count)
        x, source = keep["x"], m.route.source.long()
        assert torch.equal(x[:n], (table[m.tokens[:n].long()].float() * torch.tensor(m.D ** 0.5, device="cuda")).to(BF16)) and (x[n:] == 0).all()
        for e in range(m.E):
            a, b = int(m.route.offsets[e]), int(m.route.offsets[e] + m.route.counts[e])
            if a == b:
                continue
            for got, rows, weights in ((keep["y"], x[source[a:b] // m.K], m.up[e]), (keep["w"], keep["z"][a:b], m.down[e])):
                p, q = _definition(rows), _definition(weights)
                tol = 2 * p.shape[1] * S * (p.abs() @ q.abs().t()) + 2.0 ** -8 * (p @ q.t()).abs() + 1e-30
                assert ((got[a:b].double() - p @ q.t()).abs() <= tol).all()
        place = m.route.place[:n].long()
        v = torch.where((place >= 0).unsqueeze(2), keep["w"][place.clamp(min=0)].double(), 0.0) * keep["weights"][:n].double().unsqueeze(2)
        want, size = v.sum(dim=1), v.abs().sum(dim=1)
        assert ((out[:n].double() - want).abs() <= 2.0 ** -8 * want.abs() + m.K * 2 * S * size).all() and (out[n:] == 0).all()

    step()
    check()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed, n in ((1, 200), (2, 1), (3, 64)):
        m.tokens.copy_(torch.randint(0, m.V, (m.T,), generator=torch.Generator().manual_seed(seed)))
        m.count.fill_(n)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check()


@pytest.mark.parametrize("score,renorm", [("sigmoid", True), ("softmax", True), ("softmax", False)])
def test_training(hl, score, renorm):
    m = _Model(hl)
    m.router = hl.ExpertRouter(m.K, m.E, score=score, n_groups=4, top_groups=2, group_score="top2", renorm=renorm, scale=1.5)
    n, scale = int(m.count), m.D ** 0.5
    factor = torch.rand(m.E, m.D, generator=torch.Generator().manual_seed(1)).cuda() + 0.5      # the experts: tanh(row * factor)
    target = torch.randn(n, m.D, generator=torch.Generator().manual_seed(2)).cuda()

    x = m.emb.embed(m.table, m.tokens, scale, m.count)
    logits = x @ m.gate
    experts, weights = m.router.choose(logits, m.bias, m.count)
    m.route.sort(experts, m.count)
    y = m.route.dispatch(x)
    owner = torch.bucketize(torch.arange(m.route.cap_rows, device="cuda"), m.route.offsets[1:].long(), right=True).clamp(max=m.E - 1)
    z = torch.tanh(y * factor[owner])
    out = m.route.combine(z, weights)
    grad_out = torch.zeros(m.T, m.D, device="cuda")
    grad_out[:n] = 2 * (out[:n] - target)
    grad_z, grad_w = m.route.combine_backward(grad_out, z, weights)
    grad_logits = m.router.backward(logits, experts, grad_w, m.count)
    grad_x = m.route.dispatch_backward(grad_z * (1 - z * z) * factor[owner]) + grad_logits @ m.gate.t()
    m.emb.sort(m.tokens, m.count)
    grad_table = m.emb.backward(grad_x, scale)
    assert m.emb.status() == m.router.status() == m.route.status() == hl.HL_OK

    table = m.table.double().requires_grad_()
    gate = m.gate.double().requires_grad_()
    xs = table[m.tokens[:n].long()] * scale
    s = xs @ gate
    s.retain_grad()
    s_all = torch.sigmoid(s) if score == "sigmoid" else torch.softmax(s, dim=1)
    chosen = s_all.gather(1, experts[:n].long())
    w = 1.5 * (chosen / chosen.sum(dim=1, keepdim=True) if renorm else chosen)
    rows = torch.tanh(xs.unsqueeze(1) * factor.double()[experts[:n].long()])
    outs = (rows * w.unsqueeze(2)).sum(dim=1)
    ((outs - target.double()) ** 2).sum().backward()
    assert (experts[:n] >= 0).all() and _near(weights[:n], w.detach(), 1e-4) and _near(out[:n], outs.detach(), 1e-4)
    assert _near(grad_logits[:n], s.grad, 1e-4) and _near(x[:n].t() @ grad_logits[:n], gate.grad, 1e-4)
    assert _near(grad_table, table.grad, 1e-4)
    assert (grad_table[torch.bincount(m.tokens[:n].long(), minlength=m.V) == 0] == 0).all()
