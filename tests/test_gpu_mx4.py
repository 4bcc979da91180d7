"""Matrices in 4 bits (hl_mx4_*) and the experts' product with them (hl_expert_mx4).

Quantisation is exact by its definition: the values that come back are compared for equality with those of the definition in 64
bits, rounded once to the type they come back in.  A product adds dim exact products (of values of two significant bits each, times powers of two) in
fp32, in some order: off by at most dim s sum|x w| with s = 2^-24 for each addition's rounding (doubled here, as the order and width in which the tensor cores add up a block's
products is theirs to choose, and they may cut where others round), and by half a step of the result's type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

S = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _power(n):
    return ((n.long() + 1023) << 52).view(torch.float64)


def _definition(x):
    """fp64 values of a matrix in 4 bits."""
    rows, dim = x.shape
    v = torch.zeros(rows, -(-dim // 32) * 32, dtype=torch.float64, device=x.device)
    v[:, :dim] = x.double()
    v = v.view(rows, -1, 32)
    top = v.abs().amax(dim=2, keepdim=True)
    bad = ~torch.isfinite(v).all(dim=2, keepdim=True)
    top = torch.where(bad | (top == 0), 1.0, top)
    e = torch.frexp(top).exponent.long() - 1                     # floor of the logarithm
    unit = _power((e - 2).clamp(min=-127))
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    a = torch.where(bad, 0.0, v.abs() / unit)
    low = (torch.bucketize(a, grid, right=True) - 1).clamp(0, 7)
    high = (low + 1).clamp(max=7)
    middle = (grid[low] + grid[high]) / 2
    up = (a > middle) | ((a == middle) & (high % 2 == 0) & (high != low))
    q = torch.where(up, grid[high], grid[low]) * torch.sign(v) * unit
    q = torch.where(bad, float("nan"), q)
    return q.reshape(rows, -1)[:, :dim]


def _there_and_back(hl, x, out_type, n=1, stride=None):
    """x: [n * rows, dim] rows (a view); the matrices' rows lie one behind the other."""
    rows, dim, ld = x.shape[0] // n, x.shape[1], x.stride(0)
    need = n * hl.hl_mx4_bytes(rows, dim)
    q = torch.full((need + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    hl.hl_mx4_quantise(hl.dtype_of(x), n, rows, dim, x, ld, rows * ld if stride is None else stride, q, _stream())
    wide = torch.full((n * rows + 1, dim + 9), -7.0, dtype=out_type, device="cuda")
    for o in (0, 8, 3):
        wide[:] = -7.0
        out = wide[: n * rows, o:o + dim]
        hl.hl_mx4_dequantise(n, rows, dim, q, hl.dtype_of(out), out, out.stride(0), rows * out.stride(0), _stream())
        assert (wide[: n * rows, :o] == -7).all() and (wide[: n * rows, o + dim:] == -7).all() and (wide[n * rows:] == -7).all()
    assert (q[need:] == 0x5A).all()
    return q[:need], out.contiguous()


def _same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 31, 32, 33, 64, 255, 256, 257, 512, 600, 768, 1024, 1030, 2048, 2500])
@pytest.mark.parametrize("dtype", TYPES)
def test_values(hl, dim, dtype):
    for n, rows, pad, at in ((1, 1, 0, 0), (1, 127, 8, 0), (3, 129, 0, 0), (2, 40, 5, 1)):
        g = torch.Generator(device="cuda").manual_seed(dim + rows)
        wide = torch.randn(n * rows, dim + pad, generator=g, device="cuda") * torch.exp(2 * torch.randn(n * rows, 1, generator=g, device="cuda"))
        x = wide.to(dtype)[:, at:at + dim]
        for out_type in (F32, dtype):
            _, got = _there_and_back(hl, x, out_type, n)
            assert _same(got, _definition(x).to(out_type))


@pytest.mark.parametrize("dtype", TYPES)
def test_every_value_of_16_bits_and_ties(hl, dtype):
    if dtype == F32:
        base = torch.arange(2 ** 16, dtype=torch.int32).view(-1, 1) << 16
        x = (base | torch.tensor([0, 1, 0x7fff, 0x8000, 0x8001, 0xffff], dtype=torch.int32)).view(F32).reshape(-1)
    else:
        x = torch.arange(2 ** 16, dtype=torch.int32).to(torch.int16).view(dtype)
    # each with a block of its own, next to a power of two that decides the exponent, and next to nothing
    x = x.cuda()
    lone = torch.zeros(x.numel(), 32, dtype=dtype, device="cuda")
    lone[torch.arange(x.numel()), torch.arange(x.numel()) % 32] = x
    _, got = _there_and_back(hl, lone, F32)
    assert _same(got, _definition(lone).float())
    beside = lone.clone()
    beside[:, 5] = 4.0
    beside[torch.arange(x.numel()), (torch.arange(x.numel()) % 16) + 8] = x
    _, got = _there_and_back(hl, beside, F32)
    assert _same(got, _definition(beside).float())
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, 7.0, 7.75, 0.2490234375, 0.2509765625, 4.0], device="cuda")
    t = torch.zeros(8, 32, device="cuda")
    t[:, : ties.numel()] = ties * (2.0 ** torch.arange(-6, 2, device="cuda")).view(-1, 1)
    t = torch.cat([t, -t]).to(dtype)
    _, got = _there_and_back(hl, t, F32)
    assert _same(got, _definition(t).float())


def test_blocks_with_infinities_and_nan(hl):
    x = torch.randn(6, 100, device="cuda")
    x[0, 40] = float("inf")
    x[1, 99] = float("-inf")
    x[2, 0] = float("nan")
    x[3] = 0.0
    x[4] = torch.finfo(F32).max
    x[5] = torch.finfo(F32).tiny / 4
    for dtype in TYPES:
        _, got = _there_and_back(hl, x.to(dtype), F32)
        want = _definition(x.to(dtype)).float()
        assert _same(got, want)
        assert torch.isnan(got[0, 32:64]).all() and not torch.isnan(got[0, :32]).any() and torch.isnan(got[1, 96:]).all()


def test_matrices_beyond_31_bits(hl):
    rows, dim = 1_100_000, 2048
    x = torch.zeros(rows, dim, dtype=BF16, device="cuda")
    at = torch.tensor([0, 1, 524_288, 1_048_577, rows - 1], device="cuda")
    x[at] = torch.randn(5, dim, device="cuda").to(BF16)
    q = torch.empty(hl.hl_mx4_bytes(rows, dim), dtype=torch.uint8, device="cuda")
    hl.hl_mx4_quantise(hl.HL_BF16, 1, rows, dim, x, dim, 0, q, _stream())
    want = _definition(x[at]).to(BF16)
    x.fill_(1.0)
    hl.hl_mx4_dequantise(1, rows, dim, q, hl.HL_BF16, x, dim, 0, _stream())
    assert torch.equal(x[at], want) and float(x[2:1000].abs().max()) == 0 and float(x[-1000:-1].abs().max()) == 0


# ---- the product --------------------------------------------------------------------------------------------------------------
class _Case:
    def __init__(self, hl, T, K, E, dim, F, dtype=BF16, align=1, live=None, pad=0, at=0, cap_rows=None, seed=0, choices=None, none=0.1):
        self.hl, self.E, self.dim, self.F, self.K, self.T = hl, E, dim, F, K, T
        g = torch.Generator(device="cuda").manual_seed(seed + 1000 * dim + F)
        if choices is None:
            choices = torch.randint(0, E, (T, K), generator=g, device="cuda")
            choices = torch.where(torch.rand(T, K, generator=g, device="cuda") < none, -1, choices)
        self.route = hl.ExpertRoute(T, K, E, align=align, cap_rows=cap_rows)
        n_tokens = None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda")
        self.route.sort(choices.int().contiguous(), n_tokens)
        self.cap = self.route.cap_rows
        self.counts, self.offsets = self.route.counts.tolist(), self.route.offsets.tolist()
        self.x = torch.randn(T + 1, dim + pad, generator=g, device="cuda").to(dtype)[:T, at:at + dim]
        self.rows = torch.randn(self.cap + 1, dim + pad, generator=g, device="cuda").to(dtype)[: self.cap, at:at + dim]
        self.w = (torch.randn(E * F, dim, generator=g, device="cuda") / dim ** 0.5).to(dtype)
        self.q = torch.empty(E * hl.hl_mx4_bytes(F, dim), dtype=torch.uint8, device="cuda")
        hl.hl_mx4_quantise(hl.dtype_of(self.w), E, F, dim, self.w, dim, F * dim, self.q, _stream())
        self.wide = torch.full((self.cap + 2, F + pad + 3), -7.0, dtype=dtype, device="cuda")
        self.y = self.wide[: self.cap, at:at + F]
        self.at = at
        self.ws_bytes = hl.hl_expert_mx4_workspace_bytes(self.cap, E, dim)
        self.ws = torch.full((self.ws_bytes + 256,), 0xFF, dtype=torch.uint8, device="cuda")

    def run(self, by_token):
        x = self.x if by_token else self.rows
        self.wide.fill_(-7.0)
        self.ws[: self.ws_bytes] = 0xFF                          # (whatever lies in it)
        ld_x, ld_y = max(x.stride(0), self.dim), max(self.wide.stride(0), self.F)
        self.hl.hl_expert_mx4(self.route._route, self.hl.dtype_of(x), self.dim, self.F, x, ld_x, by_token, self.q, self.y, ld_y, self.ws,
                              self.ws_bytes, _stream())
        torch.cuda.synchronize()
        assert int(self.ws[:4].view(torch.int32)) == self.hl.HL_OK and (self.ws[self.ws_bytes:] == 0xFF).all()

    def check(self, by_token):
        self.run(by_token)
        source = self.route.source.long()
        for e in range(self.E):
            n, a, b = self.counts[e], self.offsets[e], self.offsets[e + 1]
            if n:
                rows = self.x[source[a:a + n] // self.K] if by_token else self.rows[a:a + n]
                x, w = _definition(rows), _definition(self.w[e * self.F:(e + 1) * self.F])
                want, size = x @ w.t(), x.abs() @ w.abs().t()
                tol = 2 * self.dim * S * size + torch.finfo(self.y.dtype).eps / 2 * want.abs() + 2.0 ** -25
                err = (self.y[a:a + n].double() - want).abs()
                assert (err <= tol).all(), (e, float((err - tol).max()))
            assert (self.y[a + n:b] == 0).all()
        end = self.offsets[-1]
        assert (self.wide[end:] == -7).all()
        assert (self.wide[:end, : self.at] == -7).all() and (self.wide[:end, self.at + self.F:] == -7).all()


@pytest.mark.parametrize("dim,F", [(1, 1), (31, 5), (32, 128), (64, 130), (256, 127), (257, 256), (600, 64), (1024, 300), (2500, 129),
                                   (4096, 512)])
@pytest.mark.parametrize("dtype", TYPES)
def test_product(hl, dim, F, dtype):
    for T, K, E, align, pad, at in ((1, 1, 1, 1, 0, 0), (1, 2, 8, 1, 8, 0), (7, 3, 4, 16, 5, 1), (150, 2, 5, 1, 0, 0)):
        c = _Case(hl, T, K, E, dim, F, dtype, align, pad=pad, at=at)
        c.check(True)
        c.check(False)


@pytest.mark.parametrize("T,K,E,align", [(1, 8, 256, 1), (3, 2, 64, 128), (16, 1, 1, 1), (17, 1, 1, 1), (128, 1, 1, 1), (129, 1, 1, 1),
                                         (239, 1, 1, 7), (240, 1, 1, 1), (241, 1, 1, 1), (480, 1, 2, 1), (481, 1, 1, 1), (2000, 4, 7, 16),
                                         (3000, 2, 40, 128), (900, 40, 64, 1), (64, 64, 1024, 3), (5000, 1, 3, 100)])
def test_rows_of_experts(hl, T, K, E, align):
    """Tiles that are full, one over, nearly empty; more choices of a token than a warp has lanes; many experts without rows."""
    c = _Case(hl, T, K, E, 320, 200, align=align, seed=T)
    c.check(True)
    c.check(False)


def test_tokens_on_the_device_and_none(hl):
    for live in (0, 1, 50, 99, 100):
        c = _Case(hl, 100, 2, 6, 96, 64, align=8, live=live)
        c.check(True)
        c.check(False)
    c = _Case(hl, 100, 2, 6, 96, 64, none=1.1)                   # no choice names an expert
    c.check(True)
    c = _Case(hl, 0, 2, 6, 96, 64)
    c.check(True)
    one = torch.full((300, 2), 3, device="cuda")                 # all of them, and twice, the same one
    _Case(hl, 300, 2, 6, 96, 64, choices=one).check(True)


def test_rows_that_did_not_fit(hl):
    for cap in (1, 63, 100, 255):
        c = _Case(hl, 200, 2, 4, 64, 48, align=16, cap_rows=cap)
        assert c.route.status(raise_on_error=False) == hl.HL_ECAPACITY
        c.check(True)
        c.check(False)


def test_nan_stays_in_its_row(hl):
    c = _Case(hl, 300, 2, 3, 128, 100, none=0.0)
    c.x[5, 7] = float("nan")
    c.x[6, 70] = float("inf")
    c.run(True)
    token = c.route.source[: c.offsets[-1]].long() // 2
    bad = (token == 5) | (token == 6)
    assert torch.isnan(c.y[: c.offsets[-1]][bad]).all() and torch.isfinite(c.y[: c.offsets[-1]][~bad]).all()
    w = c.w.clone()
    w[100 + 9, 3] = float("nan")                                 # a row of expert 1's
    hl.hl_mx4_quantise(hl.HL_BF16, 3, 100, 128, w, 128, 12800, c.q, _stream())
    c.x[5:7] = 0.0
    c.run(True)
    y = c.y[: c.offsets[-1]]
    a, b = c.offsets[1], c.offsets[2]
    assert torch.isnan(y[a:b, 9]).all() and int(torch.isnan(y).sum()) == b - a


def test_the_same_each_time(hl):
    c = _Case(hl, 1500, 2, 9, 1000, 700)
    c.run(True)
    first = c.y.clone()
    for _ in range(5):
        c.run(True)
        assert torch.equal(c.y, first)


def test_plans_from_elsewhere_stay_inside_the_buffers(hl):
    """Counts and offsets that no sort made: rows outside the buffer are not touched, whatever else comes out."""
    c = _Case(hl, 40, 2, 4, 64, 32)
    for counts, offsets in (([2 ** 31 - 1] * 4, [0, 10, 20, 30, 40]), ([80, 80, 80, 80], [0, 0, 0, 0, 0]), ([-5, 3, -2 ** 31, 9], [5, 4, 3, 2, 1]),
                            ([10, 10, 10, 10], [-7, 2 ** 31 - 1, 70, 79, 2 ** 31 - 1])):
        c.route.counts.copy_(torch.tensor(counts, dtype=torch.int32))
        c.route.offsets.copy_(torch.tensor(offsets, dtype=torch.int32))
        for by_token in (True, False):
            c.run(by_token)
            assert (c.wide[c.cap:] == -7).all() and (c.wide[:, c.F:] == -7).all()


def test_no_tokens_and_a_plan_of_some(hl):
    """Tokens' rows of which there are none, whatever counts the plan has."""
    c = _Case(hl, 3, 2, 4, 64, 32)
    place, counts, offsets = c.route.place, c.route.counts, c.route.offsets
    counts.fill_(2)
    offsets.copy_(torch.arange(5, dtype=torch.int32) * 2)
    route = hl.make_route(0, None, 2, 4, 1, 6, None, None, counts, offsets)
    c.wide.fill_(-7.0)
    c.ws[: c.ws_bytes] = 0xFF
    hl.hl_expert_mx4(route, hl.HL_BF16, 64, 32, None, 64, True, c.q, c.y, c.wide.stride(0), c.ws, c.ws_bytes, _stream())
    torch.cuda.synchronize()
    assert int(c.ws[:4].view(torch.int32)) == hl.HL_OK and (c.wide == -7).all()
    # some, of which the device says there are none: no row of x is read
    route = hl.make_route(3, torch.zeros(1, dtype=torch.int32, device="cuda"), 2, 4, 1, 6, place, None, counts, offsets)
    c.x.fill_(float("nan"))
    hl.hl_expert_mx4(route, hl.HL_BF16, 64, 32, c.x, c.x.stride(0), True, c.q, c.y, c.wide.stride(0), c.ws, c.ws_bytes, _stream())
    torch.cuda.synchronize()
    assert int(c.ws[:4].view(torch.int32)) == hl.HL_OK and (c.wide[6:] == -7).all()


def test_class(hl):
    E, F, dim, T, K = 6, 96, 160, 70, 2
    w = torch.randn(E, F, dim, device="cuda").to(BF16)
    weights = hl.Mx4Weights(w)
    assert torch.equal(weights.dequantise(BF16).view(-1, dim), _definition(w.view(-1, dim)).to(BF16))
    route = hl.ExpertRoute(T, K, E, align=4)
    route.sort(torch.randint(0, E, (T, K), device="cuda").int())
    x = torch.randn(T, dim, device="cuda").to(BF16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        y = weights.product(route, x)
        z = weights.product(route, route.dispatch(x), by_token=False)
    assert weights.status() == hl.HL_OK and torch.equal(y, z)
    bigger = hl.ExpertRoute(3000, K, E)
    bigger.sort(torch.randint(0, E, (3000, K), device="cuda").int())
    weights.product(bigger, torch.randn(3000, dim, device="cuda").to(BF16))
    assert torch.equal(weights.product(route, x), y) and weights.status() == hl.HL_OK
    other = hl.ExpertRoute(T, K, E + 1)
    for f in (lambda: weights.product(other, x), lambda: weights.product(route, x[1:]), lambda: weights.product(route, x[:, 1:]),
              lambda: weights.product(route, x, by_token=False), lambda: weights.product(route, x, out=y.float()),
              lambda: hl.Mx4Weights(w[0]), lambda: hl.Mx4Weights(w.cpu()), lambda: hl.Mx4Weights(w.transpose(1, 2)),
              lambda: hl.Mx4Weights(w.double()), lambda: weights.product(route, x.double())):
        with pytest.raises((ValueError, TypeError)):
            f()
