"""Tokens sorted by expert and back (hl_expert_*), against the definitions computed choice by choice in 64 bits.

Tolerances, with u = eps / 2 of the rows' type and s = 2^-24 (a rounding of fp32), from the arithmetic alone: a weighted sum of K
products in fp32 is off by at most K s sum|w y|, and rounding it once adds u of the result; a product that is rounded to fp32 and
then to the rows' type is off by s + u of itself; a dot product of D terms in fp32, in any order, by at most (D + 8) s sum|g y|;
fp16 results below 2^-14 are off by up to 2^-25 more."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

S = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def hl():
    import paper_2204_05436_b200 as hl
    return hl


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _u(dtype):
    return torch.finfo(dtype).eps / 2


def _tiny(dtype):
    return 2.0 ** -25 if dtype == torch.float16 else 0.0


class _Route:
    """The plan's buffers, behind and in front of which nothing may be written."""

    def __init__(self, hl, T, K, E, align=1, live=None, cap_rows=None, source=True):
        n = T * K
        self.hl, self.T, self.K, self.E, self.align = hl, T, K, E, align
        self.live = T if live is None else live
        self.rows = n + min(E, n) * (align - 1) if cap_rows is None else cap_rows
        d = "cuda"
        self.n_tokens = None if live is None else torch.tensor([live], dtype=torch.int32, device=d)
        self.place = torch.full((n + 8,), -7, dtype=torch.int32, device=d)
        self.source = torch.full((self.rows + 8,), -7, dtype=torch.int32, device=d) if source else None
        self.counts = torch.full((E + 8,), -7, dtype=torch.int32, device=d)
        self.offsets = torch.full((E + 9,), -7, dtype=torch.int32, device=d)
        self.status = torch.full((1,), 99, dtype=torch.int32, device=d)
        self.ws_bytes = hl.hl_expert_workspace_bytes(T, K, E)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=d)
        self.route = hl.make_route(T, self.n_tokens, K, E, align, self.rows, self.place, self.source, self.counts, self.offsets)

    def sort(self, experts, cap=0):
        self.hl.hl_expert_sort(self.route, experts, cap, self.status, self.ws, self.ws_bytes, _stream())


def _expected(experts, live, E, align, cap, rows):
    """place, source, counts, offsets, status by a loop over the choices (-7: untouched)."""
    T, K = experts.shape
    e = experts[:live].reshape(-1)
    ok = (e >= 0) & (e < E)
    status = -2 if np.any(~ok & (e != -1)) else 0
    place, source = np.full(T * K, -7), np.full(rows, -7)
    place[: live * K] = -1
    counts, offsets, at = np.zeros(E, int), np.zeros(E + 1, int), 0
    for x in range(E):
        choices = np.flatnonzero(ok & (e == x))
        choices = choices[:cap] if cap else choices
        offsets[x] = min(at, rows)
        if at + len(choices) > rows:
            status = status or -3
        fit = choices[: max(0, rows - at)]
        counts[x] = len(fit)
        place[fit] = at + np.arange(len(fit))
        source[at:at + len(fit)] = fit
        up = at + -(-len(choices) // align) * align
        source[min(at + len(fit), rows):min(up, rows)] = -1
        at = up
    offsets[E] = min(at, rows)
    return place, source, counts, offsets, status


def _choices(T, K, E, seed, skew=0.0, none=0.0, bad=0):
    r = np.random.RandomState(seed)
    load = (np.arange(E) + 1.0) ** -skew
    e = r.choice(E, size=(T, K), p=load[r.permutation(E)] / load.sum())
    e[r.rand(T, K) < none] = -1
    if bad:
        at = r.randint(0, T * K, bad)
        e.reshape(-1)[at] = r.choice([-2, E, 2 ** 31 - 1, -2 ** 31], bad)
    return e.astype(np.int32)


def _check_sort(hl, experts, E, align=1, live=None, cap=0, cap_rows=None, source=True):
    T, K = experts.shape
    p = _Route(hl, T, K, E, align, live, cap_rows, source)
    p.sort(torch.from_numpy(experts).cuda(), cap)
    torch.cuda.synchronize()
    place, src, counts, offsets, status = _expected(experts, min(max(p.live, 0), T), E, align, cap, p.rows)
    pad = [-7] * 8
    assert p.status.item() == status
    np.testing.assert_array_equal(p.offsets.cpu().numpy(), [*offsets, *pad])
    np.testing.assert_array_equal(p.counts.cpu().numpy(), [*counts, *pad])
    np.testing.assert_array_equal(p.place.cpu().numpy(), [*place, *pad])
    if source:
        np.testing.assert_array_equal(p.source.cpu().numpy(), [*src, *pad])
    return p


@pytest.mark.parametrize("T,K,E", [(1, 1, 1), (1, 2, 8), (3, 64, 5), (31, 1, 2), (33, 4, 8), (257, 3, 37), (1000, 8, 1024),
                                   (4096, 2, 64), (4097, 2, 64), (8191, 1, 3), (8193, 1, 1000), (16384, 4, 64), (16385, 4, 257),
                                   (70001, 1, 1024), (40000, 8, 256), (300_000, 1, 2), (1_000_003, 1, 128),
                                   (512, 1, 16), (513, 1, 17), (8192, 1, 500), (8193, 1, 64), (32768, 1, 1024), (32769, 1, 65),
                                   (65536, 1, 16), (65537, 1, 300), (98304, 1, 256), (98305, 1, 257)])
def test_sort_sizes(hl, T, K, E):
    _check_sort(hl, _choices(T, K, E, T + K, skew=0.8, none=0.05), E)


@pytest.mark.parametrize("T,K,E", [(5, 2, 4), (3000, 3, 37), (9000, 4, 64), (50_001, 3, 300)])
@pytest.mark.parametrize("align", [2, 16, 100, 128, 65536])
def test_sort_fills_experts_up(hl, T, K, E, align):
    if align == 65536 and E > 64:
        E = 9
    _check_sort(hl, _choices(T, K, E, align, skew=1.0), E, align)


@pytest.mark.parametrize("T,K,E", [(40, 2, 8), (9000, 3, 37), (60_000, 2, 100)])
def test_sort_live_tokens_capacity_and_strange_ids(hl, T, K, E):
    e = _choices(T, K, E, 5, skew=0.7, none=0.1)
    for live in (0, 1, T // 3, T, T + 5, -4):
        _check_sort(hl, e, E, align=4, live=live)
    for cap in (1, T * K // (2 * E) + 1, T * K):
        _check_sort(hl, e, E, align=3, cap=cap)
    p = _check_sort(hl, _choices(T, K, E, 6, bad=5), E)                        # HL_EBOUNDS
    assert p.status.item() == hl.HL_EBOUNDS
    p = _check_sort(hl, e, E, align=2, cap_rows=T * K // 2)                    # HL_ECAPACITY
    assert p.status.item() == hl.HL_ECAPACITY
    _check_sort(hl, e, E, cap_rows=0)
    _check_sort(hl, e, E, source=False)
    _check_sort(hl, np.full_like(e, -1), E, align=8)                           # nobody goes anywhere
    _check_sort(hl, np.full_like(e, E - 1), E, align=8)                        # all to one


def test_sort_of_a_huge_capacity_limit(hl):
    e = _choices(50, 2, 4, 1)
    p = _Route(hl, 50, 2, 4)
    p.sort(torch.from_numpy(e).cuda(), 2 ** 40)
    assert p.counts[:4].sum().item() == 100


def _rows(n, D, dtype, pad, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = (torch.randn(n, D + pad, generator=g, device="cuda") * scale).to(dtype)
    return t[:, :D]


def _filled(n, D, dtype, pad):
    return torch.full((n, D + pad), 5.0, dtype=dtype, device="cuda")


SHAPES = [  # T, K, E, D, pad, align, live, none
    (1, 1, 1, 1, 0, 1, None, 0.0), (1, 2, 8, 1664, 0, 1, None, 0.0), (4, 2, 8, 64, 0, 16, None, 0.0), (5, 3, 4, 7, 2, 4, 3, 0.3),
    (33, 8, 16, 2048, 0, 128, None, 0.1), (100, 4, 37, 337, 2, 1, 77, 0.2), (65, 2, 5, 1001, 7, 8, 64, 0.0),
    (64, 6, 64, 4096, 8, 3, None, 0.5), (17, 64, 3, 40, 0, 2, None, 0.1), (300, 2, 300, 36, 4, 2, 299, 0.0),
    (9, 2, 4, 20_000, 0, 2, None, 0.0), (2, 5, 4, 33_000, 1, 2, None, 0.2), (2000, 3, 16, 130, 0, 64, 1500, 1.0),
    (20, 2, 4, 260, 2, 4, 0, 0.0),
]


def _case(hl, shape, seed=3):
    T, K, E, D, pad, align, live, none = shape
    p = _Route(hl, T, K, E, align, live)
    p.sort(torch.from_numpy(_choices(T, K, E, seed, skew=0.5, none=none)).cuda())
    place = p.place[:T * K].view(T, K).long()
    live = T if live is None else live
    return p, place[:live], live, int(p.offsets[E].item())


def _sum_expected(y, place, w):
    v = y[place.clamp(min=0)].double()
    v = torch.where((place >= 0).unsqueeze(2), v, 0.0)
    if w is not None:
        v = v * w.double().unsqueeze(2)
    return v.sum(1), v.abs().sum(1)


def _rows_expected(x, place, w, end):
    out = torch.zeros(end, x.shape[1], dtype=torch.float64, device="cuda")
    t, k = torch.nonzero(place >= 0, as_tuple=True)
    v = x[t].double()
    out[place[t, k]] = v if w is None else v * w[t, k].double().unsqueeze(1)
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_dispatch_and_its_gradient(hl, shape, dtype):
    p, place, live, end = _case(hl, shape)
    T, K, E, D, pad = shape[:5]
    x, y = _rows(T, D, dtype, pad, 1), _filled(p.rows, D, dtype, pad)
    x[live:] = float("nan")
    hl.hl_expert_dispatch(p.route, hl.dtype_of(x), D, x, D + pad, y, D + pad, _stream())
    assert torch.equal(y[:end, :D].double(), _rows_expected(x, place, None, end))
    assert (y[end:] == 5).all() and (y[:, D:] == 5).all()
    gy, gx = _rows(p.rows, D, dtype, pad, 2), _filled(T, D, dtype, pad)
    gy[end:] = float("nan")                                                    # rows that no choice has are not read
    hl.hl_expert_combine(p.route, hl.dtype_of(x), D, gy, D + pad, None, gx, D + pad, _stream())
    e, size = _sum_expected(gy, place, None)
    off = (gx[:live, :D].double() - e).abs()
    assert (off <= K * S * size + _u(dtype) * (e.abs() + K * S * size) + _tiny(dtype)).all()
    assert (gx[live:] == 5).all() and (gx[:, D:] == 5).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_combine_and_its_gradients(hl, shape, dtype):
    p, place, live, end = _case(hl, shape)
    T, K, E, D, pad = shape[:5]
    ty, ld = hl.dtype_of(torch.empty(0, dtype=dtype)), D + pad
    y, out = _rows(p.rows, D, dtype, pad, 1), _filled(T, D, dtype, pad)
    y[end:] = float("inf")
    w = torch.rand(T, K, device="cuda")
    w[:live][place < 0] = float("nan")                                         # weights of choices without a row: not used
    hl.hl_expert_combine(p.route, ty, D, y, ld, w, out, ld, _stream())
    wz = torch.nan_to_num(w)[:live]
    e, size = _sum_expected(y, place, wz)
    assert ((out[:live, :D].double() - e).abs() <= K * S * size + _u(dtype) * (e.abs() + K * S * size) + _tiny(dtype)).all()
    assert (out[live:] == 5).all() and (out[:, D:] == 5).all()

    go = _rows(T, D, dtype, pad, 2)
    go[live:] = float("nan")
    gy, gw = _filled(p.rows, D, dtype, pad), torch.full((T * K + 8,), 5.0, device="cuda")
    hl.hl_expert_combine_bwd(p.route, ty, D, go, ld, y, ld, w, gy, ld, gw, _stream())
    e = _rows_expected(go, place, wz, end)
    assert ((gy[:end, :D].double() - e).abs() <= (S + _u(dtype) * (1 + S)) * e.abs() + _tiny(dtype)).all()
    assert (gy[end:] == 5).all() and (gy[:, D:] == 5).all()
    prod = go[:live].double().unsqueeze(1) * torch.where((place >= 0).unsqueeze(2), y[place.clamp(min=0)].double(), 0.0)
    off = (gw[:live * K].view(live, K).double() - prod.sum(2)).abs()
    assert (off <= (D + 8) * S * prod.abs().sum(2)).all()
    assert (gw[live * K:] == 5).all()
    # without weights, and without a gradient of them (y is then not looked at)
    gy2 = _filled(p.rows, D, dtype, pad)
    hl.hl_expert_combine_bwd(p.route, ty, D, go, ld, None, 0, None, gy2, ld, None, _stream())
    assert torch.equal(gy2[:end, :D].double(), _rows_expected(go, place, None, end))


def test_gradients_agree_with_differences(hl):
    """<grad, direction> against the change of a linear function of the outputs, which is exact to rounding: out is linear in y
    and in w."""
    T, K, E, D = 50, 3, 7, 96
    p, place, live, end = _case(hl, (T, K, E, D, 0, 4, None, 0.2))
    y, w, go = _rows(p.rows, D, torch.float32, 0, 1), torch.rand(T, K, device="cuda"), _rows(T, D, torch.float32, 0, 2)
    dy, dw = _rows(p.rows, D, torch.float32, 0, 3), torch.randn(T, K, device="cuda")

    def f(y, w):
        out = torch.empty(T, D, device="cuda")
        hl.hl_expert_combine(p.route, hl.HL_F32, D, y, D, w, out, D, _stream())
        return (out.double() * go.double()).sum().item()

    gy, gw = torch.zeros(p.rows, D, device="cuda"), torch.zeros(T, K, device="cuda")
    hl.hl_expert_combine_bwd(p.route, hl.HL_F32, D, go, D, y, D, w, gy, D, gw, _stream())
    # the differences of step 1: rounding of f at both ends, K s of sum|g||w||y| each, and of the gradient, likewise
    place0 = torch.where((place >= 0).unsqueeze(2), y[place.clamp(min=0)].double(), 0.0)
    size = (go.double().abs().unsqueeze(1) * (place0.abs() + 6) * (w.abs() + dw.abs()).double().unsqueeze(2)).sum().item()
    bound = 4 * (K + D + 8) * S * size
    assert abs(f(y + dy, w) - f(y, w) - (gy.double() * dy.double())[:end].sum().item()) <= bound
    assert abs(f(y, w + dw) - f(y, w) - (gw.double() * dw.double()).sum().item()) <= bound


@pytest.mark.parametrize("shift", [0, 1, 2, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_begin_anywhere(hl, dtype, shift):
    """Buffers that begin `shift` values behind a multiple of 16 bytes, with row strides of their own."""
    T, K, E, D = 40, 2, 5, 128
    p, place, live, end = _case(hl, (T, K, E, D, 0, 4, None, 0.1))
    ty = hl.dtype_of(torch.empty(0, dtype=dtype))

    def buffer(n, ld, fill=None):
        flat = torch.randn(shift + n * ld, device="cuda").to(dtype)
        return flat[shift:].view(n, ld)

    x, y, out, gy = buffer(T, 128), buffer(p.rows, 136), buffer(T, 132), buffer(p.rows, 129)
    w, gw = torch.rand(T, K, device="cuda"), torch.empty(T, K, device="cuda")
    hl.hl_expert_dispatch(p.route, ty, D, x, 128, y, 136, _stream())
    assert torch.equal(y[:end, :D].double(), _rows_expected(x, place, None, end))
    hl.hl_expert_combine(p.route, ty, D, y, 136, w, out, 132, _stream())
    e, size = _sum_expected(y[:, :D], place, w)
    assert ((out[:, :D].double() - e).abs() <= K * S * size + _u(dtype) * (e.abs() + K * S * size) + _tiny(dtype)).all()
    hl.hl_expert_combine_bwd(p.route, ty, D, x, 128, y, 136, w, gy, 129, gw, _stream())
    e = _rows_expected(x, place, w, end)
    assert ((gy[:end, :D].double() - e).abs() <= (S + _u(dtype) * (1 + S)) * e.abs() + _tiny(dtype)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,ld,ld_y", [(1, 1, 1), (3, 4, 5), (7, 9, 9), (8, 11, 9), (9, 9, 10), (23, 25, 25), (41, 43, 41)])
def test_gradients_of_many_short_rows_that_begin_anywhere(hl, D, ld, ld_y, dtype):
    """Rows of less than a line to a few, a thread or a few of them each: values before and behind the whole lines, y alike or not."""
    T, K, E = 60_001, 3, 16
    p, place, live, end = _case(hl, (T, K, E, D, 0, 4, 60_000, 0.1))
    ty = hl.dtype_of(torch.empty(0, dtype=dtype))
    y, go, gy = _rows(p.rows, D, dtype, ld_y - D, 1), _rows(T, D, dtype, ld - D, 2), _filled(p.rows, D, dtype, ld - D)
    w, gw = torch.rand(T, K, device="cuda"), torch.full((T, K), 5.0, device="cuda")
    hl.hl_expert_combine_bwd(p.route, ty, D, go, ld, y, ld_y, w, gy, ld, gw, _stream())
    e = _rows_expected(go, place, w[:live], end)
    assert ((gy[:end, :D].double() - e).abs() <= (S + _u(dtype) * (1 + S)) * e.abs() + _tiny(dtype)).all()
    assert (gy[end:] == 5).all() and (gy[:, D:] == 5).all()
    y0 = torch.where((place >= 0).unsqueeze(2), y[place.clamp(min=0)].double(), 0.0)
    prod = go[:live].double().unsqueeze(1) * y0
    assert ((gw[:live].double() - prod.sum(2)).abs() <= (D + 8) * S * prod.abs().sum(2)).all()
    assert (gw[live:] == 5).all()


@pytest.mark.parametrize("T", [600, 60_000])
def test_a_captured_run_replayed_with_other_choices(hl, T):
    """Sort, there, back and the gradients as one graph, beside eager calls with another workspace."""
    K, E, D = 2, 16, 256 if T < 1000 else 24
    p, q = _Route(hl, T, K, E, 8), _Route(hl, T, K, E, 8)
    e = torch.from_numpy(_choices(T, K, E, 1)).cuda()
    x, w = _rows(T, D, torch.bfloat16, 0, 1), torch.rand(T, K, device="cuda")

    def run(r, y, out, gy, gw):
        r.sort(e)
        hl.hl_expert_dispatch(r.route, hl.HL_BF16, D, x, D, y, D, _stream())
        hl.hl_expert_combine(r.route, hl.HL_BF16, D, y, D, w, out, D, _stream())
        hl.hl_expert_combine_bwd(r.route, hl.HL_BF16, D, out, D, y, D, w, gy, D, gw, _stream())

    def buffers(r):
        return (_filled(r.rows, D, torch.bfloat16, 0), _filled(T, D, torch.bfloat16, 0), _filled(r.rows, D, torch.bfloat16, 0),
                torch.zeros(T, K, device="cuda"))

    a, b = buffers(p), buffers(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run(p, *a)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        run(p, *a)
    for seed in (2, 3):
        e.copy_(torch.from_numpy(_choices(T, K, E, seed, skew=0.5, none=0.1)))
        x.copy_(_rows(T, D, torch.bfloat16, 0, seed))
        for t in (*a, *b):
            t.fill_(0)
        torch.cuda.synchronize()
        g.replay()
        run(q, *b)
        torch.cuda.synchronize()
        end = int(q.offsets[E].item())
        assert torch.equal(p.place, q.place) and torch.equal(p.offsets, q.offsets)
        for u, v in zip(a, b):
            assert torch.equal(u[:end], v[:end])


def test_two_calls_at_once_and_the_same_call_twice(hl):
    """Two routes on two streams at the same time, several times: every result is that of the call alone."""
    T, K, E, D = 20_000, 4, 64, 512
    e = torch.from_numpy(_choices(T, K, E, 1, skew=0.9)).cuda()
    x, w = _rows(T, D, torch.bfloat16, 0, 1), torch.rand(T, K, device="cuda")
    p = [_Route(hl, T, K, E, 16) for _ in range(3)]
    outs = [(_filled(r.rows, D, torch.bfloat16, 0), _filled(T, D, torch.bfloat16, 0), _filled(r.rows, D, torch.bfloat16, 0),
             torch.zeros(T, K, device="cuda")) for r in p]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        for r, (y, out, gy, gw), s in zip(p, outs, streams):
            with torch.cuda.stream(s):
                r.sort(e)
                hl.hl_expert_dispatch(r.route, hl.HL_BF16, D, x, D, y, D, _stream())
                hl.hl_expert_combine(r.route, hl.HL_BF16, D, y, D, w, out, D, _stream())
                hl.hl_expert_combine_bwd(r.route, hl.HL_BF16, D, x, D, y, D, w, gy, D, gw, _stream())
    torch.cuda.synchronize()
    for r, o in zip(p[1:], outs[1:]):
        assert torch.equal(r.place, p[0].place) and torch.equal(r.source, p[0].source)
        for u, v in zip(o, outs[0]):
            assert torch.equal(u, v)


def test_offsets_beyond_32_bits(hl):
    """Rows whose values lie more than 2^31 values into their buffer."""
    T, K, E, D = 3, 2, 2, 64
    ld = 2 ** 29                                       # five rows: 2^31 + 2^29 values, 5 GB of fp16
    p, place, live, end = _case(hl, (T, K, E, D, 0, 1, None, 0.0))
    assert end == 6
    y = torch.empty(5 * ld + D, dtype=torch.float16, device="cuda")
    x = _rows(T, D, torch.float16, 0, 1)
    hl.hl_expert_dispatch(p.route, hl.HL_F16, D, x, D, y, ld, _stream())
    rows = torch.stack([y[r * ld:r * ld + D] for r in range(6)])
    assert torch.equal(rows.double(), _rows_expected(x, place, None, end))
    out = _filled(T, D, torch.float16, 0)
    hl.hl_expert_combine(p.route, hl.HL_F16, D, y, ld, None, out, D, _stream())
    e, size = _sum_expected(rows, place, None)
    assert ((out.double() - e).abs() <= K * S * size + _u(torch.float16) * (e.abs() + K * S * size) + 2.0 ** -25).all()


def test_values_that_are_not_finite_stay_where_they_are(hl):
    T, K, E, D = 8, 2, 4, 40
    p, place, live, end = _case(hl, (T, K, E, D, 0, 2, None, 0.0))
    x = _rows(T, D, torch.bfloat16, 0, 1)
    x[3, 5], x[4, 6] = float("inf"), float("nan")
    y = _filled(p.rows, D, torch.bfloat16, 0)
    hl.hl_expert_dispatch(p.route, hl.HL_BF16, D, x, D, y, D, _stream())
    out = _filled(T, D, torch.bfloat16, 0)
    hl.hl_expert_combine(p.route, hl.HL_BF16, D, y, D, None, out, D, _stream())
    bad = ~torch.isfinite(out)
    assert bad.sum().item() == 2 and torch.isinf(out[3, 5]) and torch.isnan(out[4, 6])


def test_the_first_call_of_all_can_be_captured():
    """In a process of its own, in which no kernel has been loaded."""
    import os
    import subprocess
    import sys
    code = """
import torch, paper_2204_05436_b200 as hl
T, K, E, D = 20000, 2, 8, 64
r = hl.ExpertRoute(T, K, E, align=8)
e = torch.randint(0, E, (T, K), dtype=torch.int32, device="cuda")
x = torch.randn(T, D, device="cuda")
y, out = torch.zeros(r.cap_rows, D, device="cuda"), torch.zeros(T, D, device="cuda")
ts = hl.make_tensors([(out, out)])
ws, norm = torch.empty(hl.hl_grad_workspace_bytes(), dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")
s = torch.cuda.Stream()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=s):
    r.sort(e)
    r.combine(r.dispatch(x, y), None, out)
    hl.hl_grad_clip(ts, None, 0, 1.0, norm, ws, ws.numel(), torch.cuda.current_stream().cuda_stream)
g.replay()
torch.cuda.synchronize()
n = (2 * x).double().norm()
assert abs(norm.item() - n.item()) <= 1e-6 * n.item()
assert (out.double() - 2 * x.double() / (n + 1e-6)).abs().max() <= 1e-6 * (2 * x).abs().max() / n
print("ok")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip().endswith("ok"), out.stderr[-2000:]


def test_places_outside_the_buffer_are_skipped(hl):
    """A plan that a caller made: rows beyond cap_rows are neither read nor written."""
    T, K, E, D = 4, 2, 2, 16
    p = _Route(hl, T, K, E, cap_rows=6)
    p.place[:8] = torch.tensor([0, 6, 1, 2 ** 31 - 1, 2, -2 ** 31, 3, -9], dtype=torch.int32, device="cuda")
    x, y = _rows(T, D, torch.float32, 0, 1), _filled(8, D, torch.float32, 0)
    hl.hl_expert_dispatch(p.route, hl.HL_F32, D, x, D, y, D, _stream())
    assert torch.equal(y[:4], x) and (y[4:] == 5).all()
    out, gw = _filled(T, D, torch.float32, 0), torch.empty(T, K, device="cuda")
    hl.hl_expert_combine(p.route, hl.HL_F32, D, y, D, None, out, D, _stream())
    assert torch.equal(out, x)
    gy = _filled(8, D, torch.float32, 0)
    hl.hl_expert_combine_bwd(p.route, hl.HL_F32, D, x, D, y, D, None, gy, D, gw, _stream())
    assert torch.equal(gy[:4], x) and (gy[4:] == 5).all() and (gw[:, 1] == 0).all()
