"""The global gradient norm, clipping and the row gradients' squared norm (hl_grad_*, hl_embbag_grad_sumsq), against 64 bits.

Tolerances: sums of squares are fp64 (10^7 terms: 1e-9 of the result at most), the norm is rounded to fp32 once (2^-24); the
factor is rounded to fp32, the product with it too, and then to the tensor's type: 2 * 2^-24 + u of the value, u = eps / 2, and
half a step of fp16's values below 2^-14, 2^-25."""
import math

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


class _Work:
    def __init__(self, hl):
        self.bytes = hl.hl_grad_workspace_bytes()
        self.ws = torch.full((self.bytes,), 255, dtype=torch.uint8, device="cuda")       # (NaNs)
        self.norm = torch.full((1,), -1.0, device="cuda")


def _norm(hl, pairs, further=None):
    w = _Work(hl)
    hl.hl_grad_norm(hl.make_tensors(pairs), further, 0 if further is None else further.numel(), w.norm, w.ws, w.bytes, _stream())
    return w.norm.item()


def _clip(hl, pairs, max_norm, further=None):
    w = _Work(hl)
    hl.hl_grad_clip(hl.make_tensors(pairs), further, 0 if further is None else further.numel(), max_norm, w.norm, w.ws, w.bytes,
                    _stream())
    return w.norm.item()


def _squares(tensors):
    return sum(float(t.double().square().sum()) for t in tensors)


def _values(n, dtype, seed, shift=0, scale=1e-2):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(n + shift, generator=g, device="cuda") * scale).to(dtype)[shift:]


def _check_scaled(dst, src, f):
    e = src.double() * f
    u = torch.finfo(dst.dtype).eps / 2
    tiny = 2.0 ** -25 if dst.dtype == torch.float16 else 0.0
    assert ((dst.double() - e).abs() <= (2 * S * 1.01 + u) * e.abs() + tiny).all()


def _factor(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6))


SIZES = [[], [0], [1], [3, 0, 8], [7, 8191], [8192], [8193, 1, 1, 5], [100_000, 17, 65_536], [3] * 33, [1, 4099] * 700,
         [5_000_001]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
def test_norm_and_clip(hl, sizes, dtype):
    ts = [_values(n, dtype, i) for i, n in enumerate(sizes)]
    norm = math.sqrt(_squares(ts))
    assert abs(_norm(hl, [(t, None) for t in ts]) - norm) <= 1.01 * S * norm
    for max_norm in (0.3 * norm, 2 * norm + 1, 0.0):
        src = [t.clone() for t in ts]
        dst = [torch.full_like(t, 7, dtype=torch.float32) for t in ts]
        said = _clip(hl, list(zip(src, dst)), max_norm)
        assert abs(said - norm) <= 1.01 * S * norm
        f = _factor(norm, max_norm)
        for s, d, t in zip(src, dst, ts):
            assert torch.equal(s, t)
            _check_scaled(d, t, f)
        _clip(hl, [(s, s) for s in src], max_norm)                             # in place
        for s, t in zip(src, ts):
            if f == 1.0:
                assert torch.equal(s, t)
            else:
                _check_scaled(s, t, f)


@pytest.mark.parametrize("src", TYPES)
@pytest.mark.parametrize("dst", TYPES)
def test_every_pair_of_types_at_every_alignment(hl, src, dst):
    pairs, want = [], []
    for i, (n, a, b) in enumerate([(1, 1, 3), (2, 3, 0), (15, 1, 1), (16, 0, 0), (1000, 5, 7), (20_000, 1, 0), (8192, 0, 1), (8200, 7, 6)]):
        s, d = _values(n, src, i, a), torch.full((n + b + 9,), 7.0, dtype=dst, device="cuda")
        pairs.append((s, d[b:b + n]))
        want.append((s, d, n, b))
    norm = math.sqrt(_squares([s for s, *_ in want]))
    _clip(hl, pairs, 0.5 * norm)
    for s, d, n, b in want:
        _check_scaled(d[b:b + n], s, _factor(norm, 0.5 * norm))
        assert (d[:b] == 7).all() and (d[b + n:] == 7).all()


def test_mixed_tensors_further_sums_and_flags(hl):
    a, b, c = _values(5000, torch.float32, 1), _values(777, torch.bfloat16, 2), _values(64, torch.float16, 3)
    further = torch.tensor([2.5, 0.25], dtype=torch.float64, device="cuda")
    norm = math.sqrt(_squares([a, c]) + 2.75)
    da, db = torch.empty_like(a), torch.empty(777, device="cuda")
    got = _clip(hl, [(a, da), (b, db, hl.HL_TENSOR_NOT_IN_NORM), (c, None)], 0.7, further)
    assert abs(got - norm) <= 1.01 * S * norm
    _check_scaled(da, a, _factor(norm, 0.7))
    _check_scaled(db, b, _factor(norm, 0.7))
    assert abs(_norm(hl, [], further) - math.sqrt(2.75)) <= 1.01 * S * 2
    # only tensors outside the norm; a norm of nothing
    assert _clip(hl, [(b, db, hl.HL_TENSOR_NOT_IN_NORM)], 1.0) == 0.0
    assert torch.equal(db, b.float())


@pytest.mark.parametrize("which", ["all", "one not in the norm", "one not written", "one empty"])
@pytest.mark.parametrize("n", [32, 33, 128, 129, 256, 257, 512, 513, 1000, 1001, 2003])
def test_as_many_tensors_as_a_list_holds_and_one_more(hl, n, which):
    """(One launch takes 32, 128, 256, 512 or 1 000 of them; norm and scaling share a list where all tensors count in both.)"""
    sizes = [1 + (i * 37) % 300 for i in range(n)]
    odd = n // 2
    if which == "one empty":
        sizes[odd] = 0
    src = [_values(m, torch.float32, i) for i, m in enumerate(sizes)]
    dst = [torch.full((m,), 7.0, device="cuda") for m in sizes]
    pairs = [(s, d) for s, d in zip(src, dst)]
    squares = _squares(src)
    if which == "one not in the norm":
        pairs[odd] = (src[odd], dst[odd], hl.HL_TENSOR_NOT_IN_NORM)
        squares = _squares(src[:odd] + src[odd + 1:])
    if which == "one not written":
        pairs[odd] = (src[odd], None)
    norm = math.sqrt(squares)
    assert abs(_clip(hl, pairs, 0.5 * norm) - norm) <= 1.01 * S * norm
    f = _factor(norm, 0.5 * norm)
    if which == "one not written":
        assert (dst[odd] == 7).all()
        del src[odd], dst[odd]
    _check_scaled(torch.cat(dst), torch.cat(src), f)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_range_of_the_types(hl, dtype):
    """Squares beyond fp32's range on either side."""
    top = torch.finfo(dtype).max
    for v in (top, 2.0 ** -24 if dtype == torch.float16 else 1e-37, 1e-45 if dtype == torch.float32 else 2.0 ** -24, 1e-20, 1e25):
        t = torch.full((1000,), v, device="cuda", dtype=torch.float64).clamp(max=top).to(dtype)
        e = math.sqrt(_squares([t]))
        got = _norm(hl, [(t, None)])
        if e > 3.4e38:
            assert got == float("inf")
        else:
            assert abs(got - e) <= 1.01 * S * e + 2.0 ** -149
    mixed = torch.cat([torch.full((500,), 1e-30, device="cuda"), torch.full((3,), 1e20, device="cuda")]).clamp(max=top).to(dtype)
    e = math.sqrt(_squares([mixed]))
    assert abs(_norm(hl, [(mixed, None)]) - e) <= 1.01 * S * e


@pytest.mark.parametrize("at", [0, 8195, 99_999])
def test_not_finite(hl, at):
    t = _values(100_000, torch.bfloat16, 1)
    t[at] = float("inf")
    d = torch.empty(100_000, device="cuda")
    assert _clip(hl, [(t, d)], 1.0) == float("inf")
    finite = torch.isfinite(t)
    assert (d[finite] == 0).all() and torch.isnan(d[at])
    t[at] = float("nan")
    assert math.isnan(_clip(hl, [(t, d)], 1.0)) and torch.isnan(d).all()


def test_many_more_tensors_than_a_launch_takes(hl):
    sizes = [1 + (i * 37) % 500 for i in range(2305)]
    flat = _values(sum(sizes), torch.float32, 1)
    out = torch.zeros_like(flat)
    at = np.concatenate([[0], np.cumsum(sizes)])
    norm = math.sqrt(_squares([flat]))
    got = _clip(hl, [(flat[a:b], out[a:b]) for a, b in zip(at[:-1], at[1:])], 0.5 * norm)
    assert abs(got - norm) <= 1.01 * S * norm
    _check_scaled(out, flat, _factor(norm, 0.5 * norm))


def test_the_same_bits_every_time_and_in_a_graph(hl):
    ts = [_values(n, torch.float32, n) for n in (1_000_003, 4099, 70_000)]
    ds = [torch.zeros_like(t) for t in ts]
    w = _Work(hl)
    tensors = hl.make_tensors(list(zip(ts, ds)))

    def run():
        hl.hl_grad_clip(tensors, None, 0, 0.5, w.norm, w.ws, w.bytes, _stream())

    run()
    first = [d.clone() for d in ds] + [w.norm.clone()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        run()
    for i in range(3):
        for d in ds:
            d.zero_()
        w.norm.zero_()
        g.replay() if i else run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, ds + [w.norm]))
    ts[0].mul_(3)                                                              # other values, the same graph
    g.replay()
    torch.cuda.synchronize()
    norm = math.sqrt(_squares(ts))
    assert abs(w.norm.item() - norm) <= 1.01 * S * norm
    _check_scaled(ds[0], ts[0], _factor(norm, 0.5))


# ---- row gradients ------------------------------------------------------------------------------------------------------
class _Model:
    def __init__(self, hl, rows, D, batch, max_nnz, S=1):
        self.hl, self.rows, self.D, self.max_nnz = hl, rows, D, max_nnz
        geom = hl.make_geometry([rows], D, S)
        n = hl.hl_workspace_bytes(geom, batch, max_nnz, rows, 0)
        self.ws = torch.full((n,), 0, dtype=torch.uint8, device="cuda")
        self.ctx = hl.hl_create(geom, batch, max_nnz, rows, 0, self.ws, n)

    def __del__(self):
        torch.cuda.synchronize()
        self.hl.hl_destroy(self.ctx)


def _check_rows(hl, slots, D, bags=None, batch=None, rows=None, room=1):
    """slots: sorted, one per lookup"""
    n = len(slots)
    batch = batch or max(1, n)
    rows = rows or int(max(slots, default=0)) + 1
    m = _Model(hl, rows, D, batch, max(1, n) * room)
    bags = np.random.RandomState(n).permutation(n) if bags is None else bags
    # (arrays as long as the context's mini-batches may be, as prepare takes them)
    s, b = (torch.from_numpy(np.append(np.asarray(x, np.int32), np.full(m.max_nnz - n, 5, np.int32))).cuda() for x in (slots, bags))
    grad = _values(batch * D, torch.float32, 9).view(batch, D)
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    got = torch.full((2,), -1.0, dtype=torch.float64, device="cuda")
    hl.hl_embbag_grad_sumsq(m.ctx, s, b, count, grad, got, _stream())
    s, b = s[:n], b[:n]
    ok = (s >= 0) & (s < rows) & (b >= 0) & (b < batch)
    G = torch.zeros(rows, D, dtype=torch.float64, device="cuda")
    G.index_add_(0, s[ok].long(), grad[b[ok].long()].double())
    e = float(G.square().sum())
    assert abs(got[0].item() - e) <= 1e-11 * e, (got[0].item(), e)
    assert got[1].item() == -1
    return m


DIMS = [4, 16, 20, 36, 64, 100, 128, 260, 1024]


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 127, 128, 129, 255, 257, 1023, 1025, 5000])
def test_runs_of_every_length(hl, n, D):
    r = np.random.RandomState(n + D)
    lengths = r.choice([1, 1, 2, 3, 15, 16, 17, 40, 130, 600], size=n + 1)
    slots = np.repeat(np.arange(n + 1) * 3, lengths)[:n]
    _check_rows(hl, slots, D, room=1 + (n % 2) * 3)


@pytest.mark.parametrize("D", [4, 16, 64, 128, 512])
def test_long_runs_and_their_borders(hl, D):
    window = {4: 1024, 16: 1024, 64: 256, 128: 128, 512: 128}[D]
    for lengths in ([5000], [1, 9000, 1], [window, window], [window - 1, window + 1, 1], [window + 1, 2 * window, window - 1],
                    [3 * window, 1, 3 * window - 1, 5], [16] * 100, [17] * 100, [1] * (2 * window) + [7000]):
        _check_rows(hl, np.repeat(np.arange(len(lengths)), lengths), D)
    _check_rows(hl, np.repeat([0, 1, 2], [window * 300, 5, window * 20]), D, bags=np.zeros(window * 320 + 5, int), batch=3)


def test_skipped_lookups_and_bags_outside(hl):
    slots = np.repeat([0, 3, 9, 10], [20, 300, 5, 400])                        # 10: behind the cache, where skipped lookups sort
    bags = np.arange(725) % 50
    bags[[3, 30, 400]] = [-1, 50, 2 ** 31 - 1]
    m = _check_rows(hl, slots, 64, bags=bags, batch=50, rows=10)
    assert hl.hl_status(m.ctx, False) in (hl.HL_OK, hl.HL_EBOUNDS)


@pytest.mark.parametrize("kind", ["one", "many"])
def test_on_what_prepare_makes(hl, kind):
    """hl_embbag_bwd_prepare, the norm, clipping, hl_embbag_bwd_apply: one step of clipped SGD."""
    r = np.random.RandomState(4)
    B, T, rows, D = 300, 1, 500, 32
    per = np.ones(B, int) if kind == "one" else r.randint(0, 9, B)
    off = np.concatenate([[0], np.cumsum(per)])
    ids = np.minimum((r.pareto(0.8, off[-1]) * 3).astype(int), rows - 1)
    m = _Model(hl, rows, D, B, int(off[-1]) + 5)
    i32 = dict(dtype=torch.int32, device="cuda")
    ub = hl.make_ubatch(o := torch.tensor(off, **i32), i := torch.tensor(ids, **i32), len(ids))
    n = torch.tensor([B], **i32)
    slots, bags, count = torch.zeros(len(ids) + 5, **i32), torch.zeros(len(ids) + 5, **i32), torch.zeros(1, **i32)
    hl.hl_embbag_bwd_prepare(m.ctx, ub, n, slots, bags, count, _stream())
    grad = _values(B * D, torch.float32, 1).view(B, D)
    dense = _values(1000, torch.float32, 2)
    sumsq = torch.zeros(1, dtype=torch.float64, device="cuda")
    hl.hl_embbag_grad_sumsq(m.ctx, slots, bags, count, grad, sumsq, _stream())
    G = torch.zeros(rows, D, dtype=torch.float64, device="cuda")
    bag = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(per, device="cuda"))
    G.index_add_(0, i.long(), grad[bag].double())
    norm = math.sqrt(float(G.square().sum()) + _squares([dense]))
    cache = torch.zeros(rows, D, device="cuda")
    g2 = grad.clone()
    got = _clip(hl, [(g2, g2, hl.HL_TENSOR_NOT_IN_NORM), (dense, dense)], 0.25 * norm, sumsq)
    assert abs(got - norm) <= 1.01 * S * norm
    hl.hl_embbag_bwd_apply(m.ctx, cache, slots, bags, count, g2, 1.0, _stream())
    e = -G * _factor(norm, 0.25 * norm)
    assert torch.allclose(cache.double(), e, rtol=1e-5, atol=1e-6)
    assert hl.hl_status(m.ctx) == hl.HL_OK
