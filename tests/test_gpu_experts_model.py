"""The operators together, as a training step uses them: a mini-batch fragmented and pooled, the popular inputs through a mixture of
experts and back (the number of them on the device), the gradients clipped by the norm of the tables' row gradients and the dense
model's, and one update per row -- against the same in 64 bits with torch's own differentiation.

Tolerances: values go through some twenty fp32 roundings between sums of at most 64 terms; 1e-4 of the largest value covers 800 of
them, and an error in a formula is far larger."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _near(a, b, rel=1e-4):
    a, b = a.double(), b.double()
    return float((a - b).abs().max()) <= rel * max(float(b.abs().max()), 1e-30)


class _Experts:
    """E experts on rows of width F: tanh(row * scale_e), elementwise, so that the products stay out of this."""

    def __init__(self, E, F):
        g = torch.Generator().manual_seed(5)
        self.scale = (torch.rand(E, F, generator=g) + 0.5).cuda()

    def __call__(self, y, owner, scale=None):
        scale = self.scale if scale is None else scale
        return torch.tanh(y * scale.to(y.dtype)[owner])


def _table_model(hl, seed, B=64, T=3, D=8, rows=40, per=2):
    rng = np.random.default_rng(seed)
    n = T * B
    lengths = rng.integers(0, 2 * per, n)
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    idx = rng.integers(0, rows, off[-1]).astype(np.int32)
    idx[rng.random(off[-1]) < 0.7] %= 7                                        # popular ones
    table = rng.standard_normal((T * rows, D)).astype(np.float32)
    host = torch.from_numpy(table.copy()).pin_memory()
    hot = np.concatenate([t * rows + np.arange(12) for t in range(T)])
    h = hl.Hotline([rows] * T, D, 1, B, max(1, len(idx)), len(hot), T * rows, host)
    return h, torch.from_numpy(idx).cuda(), torch.from_numpy(off).cuda(), table, hot, (B, T, D, rows)


@pytest.mark.parametrize("max_norm", [1e9, 0.05])
@pytest.mark.parametrize("seed", [1, 2])
def test_a_training_step(hl, seed, max_norm):
    h, idx, off, table, hot, (B, T, D, rows) = _table_model(hl, seed)
    E, K, F, lr = 5, 2, T * D, 0.25
    with h, torch.cuda.stream(h.main):
        h.set_hot_rows(torch.from_numpy(hot).cuda())
        h.build_remap()
        h.fragment(idx, off, B)
        h.gather_cold()
        h.fwd_pop()
        h.fwd_non()
        h.main.synchronize()
        n_pop, n_non = (int(x) for x in h.counts[:2].cpu())
        assert 3 < n_pop < B - 3
        experts = _Experts(E, F)
        g = torch.Generator().manual_seed(seed)
        choice = torch.randint(-1, E, (B, K), generator=g).to(torch.int32).cuda()
        weights = torch.rand(B, K, generator=g).cuda()
        dense = torch.randn(300, generator=g).cuda()
        target = torch.randn(B, F, generator=g).cuda()

        # the popular inputs' rows, padded to the batch; the number of inputs stays on the device
        def inputs(pooled, n):
            return pooled[:T * n].view(T, n, D).permute(1, 0, 2).reshape(n, F)

        x = torch.zeros(B, F, device="cuda")
        x[:n_pop] = inputs(h.pooled_pop, n_pop)
        x[n_pop:] = float("nan")
        route = hl.ExpertRoute(B, K, E, align=4)
        route.sort(choice, n_tokens=h.counts)
        y = route.dispatch(x)
        owner = torch.bucketize(torch.arange(route.cap_rows, device="cuda"), route.offsets[1:].long(), right=True).clamp(max=E - 1)
        z = experts(y, owner)
        out = route.combine(z, weights)
        grad_out = torch.zeros(B, F, device="cuda")
        grad_out[:n_pop] = 2 * (out[:n_pop] - target[:n_pop])
        grad_z, grad_w = route.combine_backward(grad_out, z, weights)
        grad_y = grad_z * (1 - z * z) * experts.scale[owner]
        grad_x = route.dispatch_backward(grad_y)
        assert route.status() == hl.HL_OK
        grad_non = 2 * (h.pooled_non[:T * n_non] - 1.0)
        grad_all = torch.cat([grad_x[:n_pop].view(n_pop, T, D).permute(1, 0, 2).reshape(T * n_pop, D), grad_non])
        dense_in = dense.clone()
        norm = h.update_clipped(grad_all, lr, max_norm, others=[(dense, dense)])
        h.scatter_cold()
        h.flush_hot()
        h.status()
        after = h.host_table.clone()

        # the same in 64 bits
        tab = torch.from_numpy(table).cuda().double().requires_grad_()
        w64 = weights.double().requires_grad_()
        o = off.long()
        bag = torch.repeat_interleave(torch.arange(T * B, device="cuda"), o[1:] - o[:-1])
        row = idx.long() + rows * (bag // B)
        pooled = torch.zeros(T * B, D, dtype=torch.float64, device="cuda").index_add(0, bag, tab[row]).view(T, B, D)
        perm = h.perm.long()
        xs = pooled[:, perm[:n_pop]].permute(1, 0, 2).reshape(n_pop, F)
        outs = 0
        for k in range(K):
            c = choice[:n_pop, k].long()
            v = torch.tanh(xs * experts.scale.double()[c.clamp(min=0)]) * w64[:n_pop, k:k + 1]
            outs = outs + torch.where((c >= 0).unsqueeze(1), v, 0.0)
        loss = ((outs - target[:n_pop].double()) ** 2).sum() + ((pooled[:, perm[n_pop:]] - 1.0) ** 2).sum()
        loss.backward()
        total = (tab.grad.square().sum() + dense_in.double().square().sum()).sqrt()
        f = torch.clamp(max_norm / (total + 1e-6), max=1.0)
        assert _near(out[:n_pop], outs.detach()) and _near(grad_w[:n_pop], w64.grad[:n_pop])
        assert _near(norm, total.detach().view(1))
        assert _near(dense, dense_in.double() * f)
        step = torch.from_numpy(table).cuda().double() - lr * f * tab.grad
        # (what a row changed by, which clipping makes small beside the row itself: fp32 rows round 2^-24 of it)
        assert float((after.cuda().double() - step).abs().max()) <= 1e-4 * lr * float(f) * float(tab.grad.abs().max()) + 2.0 ** -22
        assert (out[n_pop:] == 0).all()


def test_clipping_counts_a_row_once(hl):
    """All inputs look up one row: the row's gradient is the sum, its norm B times that of one."""
    B, D = 50, 16
    host = torch.zeros(4, D).pin_memory()
    h = hl.Hotline([4], D, 1, B, B, 4, 4, host)
    with h, torch.cuda.stream(h.main):
        h.set_hot_rows(torch.arange(4).cuda())
        h.build_remap()
        h.fragment(torch.full((B,), 2, dtype=torch.int32, device="cuda"), torch.arange(B + 1, dtype=torch.int32, device="cuda"), B)
        h.gather_cold()
        grad = torch.ones(B, D, device="cuda")
        norm = h.update_clipped(grad, 1.0, 1.0)
        h.status()
        e = B * D ** 0.5
        assert abs(norm.item() - e) <= 1e-6 * e
        assert _near(h.cache[2], torch.full((D,), -B / (e + 1e-6)).cuda(), 1e-6)
        assert (h.cache[[0, 1, 3]] == 0).all()
        for bad in (grad.double(), grad[:, :8], grad.cpu(), torch.ones(B + 1, D, device="cuda"), grad.view(-1)):
            with pytest.raises(ValueError):
                h.update_clipped(bad, 1.0, 1.0)
        with pytest.raises(hl.HotlineError):
            h.update_clipped(grad, 1.0, -1.0)


def test_clipping_needs_a_mini_batch_and_all_of_its_gradients(hl):
    B, D = 50, 16
    h = hl.Hotline([4], D, 1, B, B, 4, 4, torch.zeros(4, D).pin_memory())
    grad, dense = torch.ones(B, D, device="cuda"), torch.ones(7, device="cuda")
    torch.cuda.synchronize()
    with h:
        h.set_hot_rows(torch.arange(4).cuda())
        h.build_remap()
        with pytest.raises(ValueError):
            h.update_clipped(grad, 1.0, 1.0)
        idx, off = torch.full((B,), 2, dtype=torch.int32, device="cuda"), torch.arange(B + 1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        h.fragment(idx, off, B)
        h.gather_cold()
        for bad, others in [(grad[1:], ()), (grad, [(dense.cpu(), dense.cpu())]), (grad, [(dense, dense), (dense, dense)])]:
            with pytest.raises(ValueError):
                h.update_clipped(bad, 1.0, 1.0, others)
        # (called beside another stream than the main one, which the first call's buffers are not to be filled on)
        torch.cuda._sleep(20_000_000)
        norm = h.update_clipped(grad, 1.0, 1.0)
        h.main.synchronize()
        e = B * D ** 0.5
        assert abs(norm.item() - e) <= 1e-6 * e
        torch.cuda.synchronize()
        assert abs(norm.item() - e) <= 1e-6 * e


def test_what_a_route_refuses(hl):
    for bad in (dict(top_k=0), dict(top_k=65), dict(n_experts=0), dict(n_experts=1025), dict(align=0), dict(max_tokens=-1),
                dict(max_tokens=2 ** 30), dict(cap_rows=-1)):
        with pytest.raises(ValueError):
            hl.ExpertRoute(**{**dict(max_tokens=8, top_k=2, n_experts=4), **bad})
    r = hl.ExpertRoute(8, 2, 4)
    e = torch.zeros(8, 2, dtype=torch.int32, device="cuda")
    for bad in (e.long(), e.cpu(), e[:, :1], torch.zeros(9, 2, dtype=torch.int32, device="cuda"), e.t().contiguous().t()):
        with pytest.raises(ValueError):
            r.sort(bad)
    with pytest.raises(ValueError):
        r.sort(e, expert_cap=-1)
    with pytest.raises(ValueError):
        r.sort(e, n_tokens=torch.zeros(1, dtype=torch.int32))
    r.sort(e)
    x = torch.zeros(8, 16, device="cuda")
    y, w = r.dispatch(x), torch.ones(8, 2, device="cuda")
    for bad in (x[:7], x.cpu(), x.t().contiguous().t(), x.view(-1), x[:, :1].expand(8, 16)):
        with pytest.raises(ValueError):
            r.dispatch(bad)
    for bad in (x.double(), x.int()):
        with pytest.raises(TypeError):
            r.dispatch(bad)
    for bad in (w.half(), w[:, :1], w.t().contiguous().t()):
        with pytest.raises(ValueError):
            r.combine(y, bad)
    with pytest.raises(ValueError):
        r.combine(y, w, out=torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        r.combine(y, w, out=y[:8])
    with pytest.raises(ValueError):
        r.combine_backward(x, y, w, grad_y=y)
    with pytest.raises(ValueError):
        r.combine_backward(x, None, w, grad_weights=w)
    with pytest.raises(ValueError):
        r.combine_backward(x, y[:, :8], w)


def test_a_route_again_with_fewer_tokens_and_none(hl):
    r = hl.ExpertRoute(20, 2, 3, align=2)
    x = torch.randn(20, 12, device="cuda")
    for n in (20, 7, 0, 1):
        e = torch.randint(0, 3, (n, 2), dtype=torch.int32, device="cuda")
        r.sort(e)
        out = r.dispatch_backward(r.dispatch(x[:n]))
        assert r.status() == hl.HL_OK and out.shape == (n, 12)
        assert torch.equal(out, 2 * x[:n])
    e[:] = 7
    r.sort(e)
    assert r.status(False) == hl.HL_EBOUNDS
    with pytest.raises(hl.HotlineError):
        r.status()
    small = hl.ExpertRoute(20, 2, 3, cap_rows=10)
    small.sort(torch.zeros(20, 2, dtype=torch.int32, device="cuda"))
    assert small.status(False) == hl.HL_ECAPACITY and int((small.place >= 0).sum()) == 10


def test_another_stream_than_the_tensors_own(hl):
    """Work queued on a side stream behind an event; nothing of it on the default stream."""
    r = hl.ExpertRoute(300, 2, 6, align=8)
    e = torch.randint(0, 6, (300, 2), dtype=torch.int32, device="cuda")
    x = torch.randn(300, 64, device="cuda").bfloat16()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        r.sort(e)
        y = r.dispatch(x)
        out = r.combine(y, None)
    s.synchronize()
    assert torch.equal(out, (2 * x.float()).bfloat16())
