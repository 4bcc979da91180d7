"""Rows of tokens (hl_token_embed) and the gradient of their table (hl_token_sort, hl_token_embed_bwd).

Tolerances, with s = 2^-24 (a rounding of fp32) and u = eps / 2 of the result's type: a row is one product in fp32, rounded once: it
is compared bit by bit with torch's.  A gradient of m tokens is a sum of fp32 numbers, in some order: off by at most m s sum|g|
before the scale, whose product adds s, and rounding adds u of the result (2^-25 more for fp16 below its normal range)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

S = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _rows(n, dim, dtype, pad=0, at=0, seed=0):
    """A view of n rows with values around them that are no part of it."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(n + 1, dim + pad, generator=g, device="cuda").to(dtype)
    return t[:n, at:at + dim]


def _tokens(n, V, seed, kind="power"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "power":
        u = torch.rand(n, generator=g, device="cuda")
        t = ((V + 1.0) ** u - 1).long().clamp(max=V - 1)        # log-uniform: some rows very often
    elif kind == "same":
        t = torch.full((n,), V // 2, device="cuda")
    elif kind == "distinct":
        t = torch.randperm(V, generator=g, device="cuda")[:n]
    elif kind == "last":
        t = torch.full((n,), V - 1, device="cuda")
    else:
        t = torch.full((n,), -1, device="cuda")
    return t.int()


def _embed(hl, table, tokens, scale, out, n_tokens=None, status=None):
    hl.hl_token_embed(hl.dtype_of(table), table.shape[0], table.shape[1], table, table.stride(0), tokens, tokens.numel(), n_tokens, scale,
                      hl.dtype_of(out), out, out.stride(0), status, torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 9, 24, 37, 64, 337, 1000, 2050, 4096])
@pytest.mark.parametrize("table_type,out_type", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32), (F16, F16), (F16, BF16)])
def test_rows(hl, dim, table_type, out_type):
    for n, V, pad, at in ((1, 1, 0, 0), (5, 100, 8, 0), (33, 50, 3, 1), (700, 1000, 5, 2)):
        table = _rows(V, dim, table_type, pad, at, dim)
        tokens = _tokens(n, V, n)
        tokens[n // 2] = -1
        wide = torch.full((n + 2, dim + 9), -7.0, dtype=out_type, device="cuda")
        for o in (0, 1, 8):
            for live in (None, n // 2, n, 0):
                wide[:] = -7.0
                out = wide[:n, o:o + dim]
                count = None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda")
                _embed(hl, table, tokens, 3.7, out, count)
                rows = n if live is None else live
                t = tokens[:rows].long()
                want = torch.where((t >= 0).unsqueeze(1), table[t.clamp(min=0)].float() * torch.tensor(3.7, device="cuda"), 0.0).to(out_type)
                assert torch.equal(out[:rows], want)
                assert (wide[:rows, :o] == -7).all() and (wide[:rows, o + dim:] == -7).all() and (wide[rows:] == -7).all()


def test_tokens_that_are_no_rows(hl):
    table = _rows(10, 16, F32)
    tokens = torch.tensor([0, 10, -1, -2, 9, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    status, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((7, 16), 5.0, device="cuda")
    for dim in (16, 13):
        status.zero_()
        _embed(hl, table[:, :dim], tokens[:1], 1.0, out[:, :dim], status=status)
        _embed(hl, table[:, :dim], tokens[2:3], 1.0, out[:, :dim], status=status)
        assert int(status) == hl.HL_OK
        _embed(hl, table[:, :dim], tokens, 1.0, out[:, :dim], status=status)
        assert int(status) == hl.HL_EBOUNDS
        assert torch.equal(out[0, :dim], table[0, :dim]) and torch.equal(out[4, :dim], table[9, :dim])
        assert (out[[1, 2, 3, 5, 6], :dim] == 0).all()
    # infinities and NaN in a row that is there, and none in one that is not
    table[3] = float("inf")
    table[4] = float("nan")
    _embed(hl, table, torch.tensor([3, 4, -1], dtype=torch.int32, device="cuda"), 0.5, out[:3])
    assert torch.isinf(out[0]).all() and torch.isnan(out[1]).all() and (out[2] == 0).all()


class _Backward:
    def __init__(self, hl, tokens, V, dim, live=None, most=None):
        self.hl, self.tokens, self.V, self.dim = hl, tokens, V, dim
        n = tokens.numel()
        self.n_tokens = None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda")
        self.sorted = torch.full((n + 4,), -7, dtype=torch.int32, device="cuda")
        self.order = torch.full((n + 4,), -7, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws_bytes = hl.hl_token_workspace_bytes(max(n, most or 0), dim)
        self.ws = torch.full((self.ws_bytes + 256,), 0xA5, dtype=torch.uint8, device="cuda")
        hl.hl_token_sort(tokens, n, self.n_tokens, V, self.sorted, self.order, self.status, self.ws, self.ws_bytes,
                         torch.cuda.current_stream().cuda_stream)
        live = n if live is None else live
        t = tokens[:live]
        key = torch.where((t >= 0) & (t < V), t, V)
        want, order = torch.sort(key.long(), stable=True)
        assert torch.equal(self.sorted[:live].long(), want) and torch.equal(self.order[:live].long(), order)
        assert (self.sorted[n:] == -7).all() and (self.order[n:] == -7).all()
        self.live = live

    def __call__(self, grad_out, scale, table, accumulate=False):
        self.ws[: self.ws_bytes] = 0xA5
        self.hl.hl_token_embed_bwd(self.V, self.dim, self.sorted, self.order, self.tokens.numel(), self.n_tokens, self.hl.dtype_of(grad_out),
                                   grad_out, grad_out.stride(0), scale, self.hl.dtype_of(table), table, table.stride(0), accumulate,
                                   self.ws, self.ws_bytes, torch.cuda.current_stream().cuda_stream)
        assert (self.ws[self.ws_bytes:] == 0xA5).all()

    def check(self, grad_out, scale, table, accumulate=False):
        before = table.clone()
        self(grad_out, scale, table, accumulate)
        t = self.tokens[: self.live].long()
        there = (t >= 0) & (t < self.V)
        g = grad_out[: self.live][there].double()
        want = torch.zeros(self.V, self.dim, dtype=torch.float64, device="cuda").index_put_((t[there],), g, accumulate=True)
        size = torch.zeros_like(want).index_put_((t[there],), g.abs(), accumulate=True)
        many = torch.bincount(t[there], minlength=self.V).unsqueeze(1)
        tol = (many * size + want.abs()) * S * abs(scale)
        want *= scale
        if accumulate:
            want += before.double()
            tol = tol + S * want.abs()
        tol = tol + torch.finfo(table.dtype).eps / 2 * want.abs() + (2.0 ** -25 if table.dtype == F16 else 1e-40)
        err = (table.double() - want).abs()
        assert (err <= tol).all(), float((err - tol).max())
        untouched = (many == 0).squeeze(1)
        assert torch.equal(table[untouched], before[untouched] if accumulate else torch.zeros_like(before[untouched]))


@pytest.mark.parametrize("dim", [1, 3, 8, 20, 37, 64, 255, 337, 512, 1030, 2048])
@pytest.mark.parametrize("grad_type,table_type", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16), (F32, BF16)])
def test_gradients(hl, dim, grad_type, table_type):
    for n, V, pad, at, live in ((1, 1, 0, 0, None), (40, 7, 8, 0, None), (555, 300, 3, 1, 400), (3001, 5000, 5, 2, None)):
        b = _Backward(hl, _tokens(n, V, n), V, dim, live)
        grad_out = _rows(n, dim, grad_type, pad, at, n)
        wide = torch.full((V + 2, dim + 9), -7.0, dtype=table_type, device="cuda")
        for o in (0, 8, 1):
            wide[:] = -7.0
            b.check(grad_out, 1.7, wide[:V, o:o + dim])
            assert (wide[:V, :o] == -7).all() and (wide[:V, o + dim:] == -7).all() and (wide[V:] == -7).all()


@pytest.mark.parametrize("kind", ["same", "last", "distinct", "power", "none"])
@pytest.mark.parametrize("n,V,dim", [(31, 64, 24), (33, 40, 24), (1000, 1000, 337), (5000, 20_000, 8), (70_001, 100_000, 12),
                                     (70_000, 80_000, 37)])
def test_runs(hl, kind, n, V, dim):
    """Runs inside a window, over the next one's border, and over all windows; one row, one token, none."""
    if kind == "distinct" and n > V:
        n = V
    b = _Backward(hl, _tokens(n, V, 3, kind), V, dim)
    grad_out = _rows(n, dim, F32, seed=1)
    table = torch.full((V, dim), 3.0, device="cuda")
    b.check(grad_out, -0.5, table)
    again = torch.full((V, dim), 4.0, device="cuda")
    b(grad_out, -0.5, again)
    assert torch.equal(table, again)
    b.check(grad_out, 2.0, table, accumulate=True)


@pytest.mark.parametrize("n", [2047, 2048, 2049, 4095, 16_384, 16_385, 32_767, 32_768, 32_769, 33_000])
@pytest.mark.parametrize("V", [1, 200, 255, 256, 70_000, 20_000_000])
def test_orders_around_the_sorts_sizes(hl, n, V):
    """Tokens in all numbers of digits, also fewer than there is room for: _Backward compares the order with a stable sort's."""
    for live in (None, n - 1, 2049, 1, 0):
        live = live if live is None else min(live, n)
        tokens = _tokens(n, V, n + V, "power")
        tokens[::7] = -1
        assert int(_Backward(hl, tokens, V, 4, live).status) == hl.HL_OK
        if live is None or live > 5:
            tokens[5] = V
            assert int(_Backward(hl, tokens, V, 4, live).status) == hl.HL_EBOUNDS


def test_runs_of_every_length_around_the_windows(hl):
    """Rows of 1, 2, 3 ... 70 and of 15, 16, 17 times 16, 32 and 64 tokens, one behind the other."""
    lengths = list(range(1, 71)) + [w * k + d for w in (16, 32, 64) for k in (1, 15, 16, 17) for d in (-1, 0, 1)]
    tokens = torch.repeat_interleave(torch.arange(len(lengths)), torch.tensor(lengths))
    tokens = tokens[torch.randperm(tokens.numel(), generator=torch.Generator().manual_seed(4))].int().cuda()
    for dim in (16, 300, 301):
        for dtype in (F32, BF16):
            _Backward(hl, tokens, len(lengths) + 3, dim).check(_rows(tokens.numel(), dim, dtype), 1.0,
                                                               torch.zeros(len(lengths) + 3, dim, dtype=dtype, device="cuda"))


def test_no_tokens_and_bad_ones(hl):
    V, dim = 50, 24
    none = _Backward(hl, torch.zeros(0, dtype=torch.int32, device="cuda"), V, dim)
    table = torch.full((V, dim), 3.0, device="cuda")
    none.check(torch.zeros(0, dim, device="cuda"), 1.0, table, accumulate=True)
    none.check(torch.zeros(0, dim, device="cuda"), 1.0, table)
    b = _Backward(hl, torch.tensor([3, 50, -1, 49, -9, 3, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), V, dim)
    assert int(b.status) == hl.HL_EBOUNDS
    b.check(_rows(7, dim, F32), 1.0, table)
    dead = _Backward(hl, _tokens(100, V, 1), V, dim, live=0)
    dead.check(_rows(100, dim, F32), 1.0, table)
    assert int(dead.status) == hl.HL_OK


def test_masked_infinities_stay_out(hl):
    """Gradients of skipped tokens, and of those behind the last, may be anything."""
    V, dim, n = 30, 40, 200
    tokens = _tokens(n, V, 1)
    tokens[::3] = -1
    grad_out = _rows(n, dim, F32)
    grad_out[::3] = float("nan")
    grad_out[150:] = float("inf")
    b = _Backward(hl, tokens, V, dim, live=150)
    clean = torch.where(torch.isfinite(grad_out), grad_out, 0.0)
    a, c = torch.zeros(V, dim, device="cuda"), torch.zeros(V, dim, device="cuda")
    b(grad_out, 1.0, a)
    b(clean, 1.0, c)
    assert torch.equal(a, c)


def test_against_differences(hl):
    """The gradient of sum(grad_out * embed(table)) by differences: it is linear in the table."""
    V, dim, n, scale = 9, 5, 40, 1.25
    table, tokens, grad_out = _rows(V, dim, F32).contiguous(), _tokens(n, V, 2), _rows(n, dim, F32, seed=3)
    got = torch.zeros(V, dim, device="cuda")
    _Backward(hl, tokens, V, dim)(grad_out, scale, got)
    out, h = torch.zeros(n, dim, device="cuda"), 0.5
    for v in (0, 3, 8):
        for d in range(dim):
            values = []
            for sign in (1, -1):
                moved = table.clone()
                moved[v, d] += sign * h
                _embed(hl, moved, tokens, scale, out)
                values.append(float((out.double() * grad_out.double()).sum()))
            # (each row of the products is rounded twice: 2 n s of sum|grad * out|)
            assert abs((values[0] - values[1]) / (2 * h) - float(got[v, d])) < 4 * n * S * 50


def test_a_table_beyond_31_bits(hl):
    """Offsets of more than 2^31 values, in the table and in its gradient."""
    V, dim = 530_000, 4096
    table = torch.zeros(V, dim, dtype=BF16, device="cuda")
    rows = torch.tensor([0, 1, V // 2, V - 2, V - 1], device="cuda")
    table[rows] = _rows(5, dim, BF16)
    tokens = rows[torch.tensor([4, 3, 0, 4, 2, 1, 4], device="cuda")].int()
    out = torch.zeros(7, dim, dtype=BF16, device="cuda")
    _embed(hl, table, tokens, 1.0, out)
    assert torch.equal(out, table[tokens.long()])
    table.fill_(1.0)
    b = _Backward(hl, tokens, V, dim)
    grad_out = _rows(7, dim, BF16, seed=1)
    b(grad_out, 1.0, table)
    want = torch.zeros(5, dim, dtype=torch.float64, device="cuda")
    want.index_add_(0, torch.tensor([4, 3, 0, 4, 2, 1, 4], device="cuda"), grad_out.double())
    assert ((table[rows].double() - want).abs() <= 2.0 ** -8 * want.abs() + 8 * S * 20).all()
    assert int(torch.count_nonzero(table.view(-1)[: 2 ** 31])) <= 4 * dim          # (in pieces: what is zero otherwise)
    assert float(table[5000:5100].abs().max()) == 0 and float(table[V - 100:V - 2].abs().max()) == 0


def test_class(hl):
    V, dim, n = 300, 64, 500
    emb = hl.TokenEmbedding(1000, V, dim)
    table, tokens = _rows(V, dim, BF16).contiguous(), _tokens(n, V, 5)
    count = torch.tensor([450], dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        x = emb.embed(table, tokens, 8.0, count, dtype=F32)
        emb.sort(tokens, count)
        grad = emb.backward(x, 8.0)
    assert emb.status() == hl.HL_OK
    t = tokens.long()
    assert torch.equal(x[:450], table[t[:450]].float() * 8.0) and (x[450:] == 0).all()
    want = torch.zeros(V, dim, dtype=torch.float64, device="cuda").index_add_(0, t[:450], x[:450].double()) * 8.0
    assert (grad.double() - want).abs().max() <= 500 * S * want.abs().max()
    # fewer tokens than before, and none
    for m in (999, 77, 1, 0):
        emb.sort(_tokens(m, V, m))
        assert emb.backward(torch.ones(m, dim, device="cuda")).double().sum() == m * dim
    emb.sort(torch.tensor([V], dtype=torch.int32, device="cuda"))
    assert emb.status(raise_on_error=False) == hl.HL_EBOUNDS
    for f in (lambda: emb.embed(table.t(), tokens), lambda: emb.embed(table, t), lambda: emb.embed(table[:10], tokens),
              lambda: emb.embed(table, tokens, out=table[:n]), lambda: emb.sort(_tokens(1001, V, 1)), lambda: emb.sort(emb.order[:10]),
              lambda: emb.backward(x), lambda: emb.backward(torch.ones(1, dim, device="cuda"), accumulate=True),
              lambda: emb.embed(table.double(), tokens)):
        with pytest.raises((ValueError, TypeError)):
            f()


def test_captured_and_replayed(hl):
    """One embedding's calls in a graph, another's beside it, with other tokens each time."""
    V, dim, n = 1000, 96, 3000
    table = _rows(V, dim, BF16).contiguous()
    embs = [hl.TokenEmbedding(n, V, dim) for _ in range(2)]
    state = []
    for emb in embs:
        tokens, x, grad = _tokens(n, V, 1), torch.zeros(n, dim, dtype=BF16, device="cuda"), torch.zeros(V, dim, device="cuda")

        def step(emb=emb, tokens=tokens, x=x, grad=grad):
            emb.embed(table, tokens, 2.0, out=x)
            emb.sort(tokens)
            emb.backward(x, 2.0, grad)

        step()
        torch.cuda.synchronize()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            step()
        state.append((graph, stream, tokens, x, grad))
    for round_ in range(3):
        for i, (graph, stream, tokens, x, grad) in enumerate(state):
            tokens.copy_(_tokens(n, V, 10 * round_ + i))
        torch.cuda.synchronize()
        for graph, stream, *_ in state:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for graph, stream, tokens, x, grad in state:
            t = tokens.long()
            assert torch.equal(x, (table[t].float() * 2.0).to(BF16))
            want = torch.zeros(V, dim, dtype=torch.float64, device="cuda").index_add_(0, t, x.double()) * 2.0
            many = torch.bincount(t, minlength=V).unsqueeze(1)
            size = torch.zeros(V, dim, dtype=torch.float64, device="cuda").index_add_(0, t, x.double().abs()) * 2.0
            assert ((grad.double() - want).abs() <= (many + 2) * S * size).all()
