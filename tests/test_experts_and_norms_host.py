"""What ExpertRoute and Hotline check and allocate before anything is queued, on tensors in host memory with the library's calls
taken out (no GPU needed)."""
import pytest
import torch


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


@pytest.fixture
def route(hl):
    """A route of 8 tokens, two of four experts each, whose calls go to `calls`."""
    r = hl.ExpertRoute.__new__(hl.ExpertRoute)
    r.device = torch.device("cpu")
    r.max_tokens, r.top_k, r.n_experts, r.align, r.cap_rows = 8, 2, 4, 1, 16
    i32 = dict(dtype=torch.int32)
    r.place, r.source = torch.full((8, 2), -1, **i32), torch.full((16,), -1, **i32)
    r.counts, r.offsets = torch.zeros(4, **i32), torch.zeros(5, **i32)
    r.calls = []
    r._call = lambda f, *a: r.calls.append((f, a))
    r._set(8, None)
    return r


@pytest.mark.parametrize("default", [torch.float32, torch.bfloat16, torch.float16, torch.float64])
@pytest.mark.parametrize("rows", [torch.float32, torch.bfloat16, torch.float16])
def test_gradients_of_weights_are_fp32_whatever_torchs_default(route, rows, default):
    x, y, w = torch.zeros(8, 6, dtype=rows), torch.zeros(16, 6, dtype=rows), torch.zeros(8, 2, dtype=torch.float32)
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        grad_y, grad_w = route.combine_backward(x, y, w)
        others = route.dispatch(x), route.combine(y, w), route.dispatch_backward(y)
    finally:
        torch.set_default_dtype(before)
    assert grad_w.dtype == torch.float32 and grad_w.shape == (8, 2)
    assert grad_y.dtype == rows and all(t.dtype == rows for t in others)
    assert len(route.calls) == 4


@pytest.fixture
def hotline(hl, monkeypatch):
    """A Hotline of 3 tables with rows of 8, at most 64 inputs, whose calls go to `calls`."""
    from types import SimpleNamespace

    from paper_2204_05436_b200 import pipeline
    h = hl.Hotline.__new__(hl.Hotline)
    h.ctx, h.calls = None, []
    for name in ("hl_fragment", "hl_step", "hl_embbag_bwd_prepare_merged", "hl_embbag_grad_sumsq", "hl_grad_clip", "hl_embbag_bwd_apply"):
        monkeypatch.setattr(pipeline.B, name, lambda *a, name=name: h.calls.append(name))
    h._batch = lambda indices, offsets, batch: batch
    h.device = torch.device("cpu")
    h.T, h.S, h.D, h.max_batch, h.max_nnz, h.n_dense, h.bags = 3, 1, 8, 64, 64 * 3, 0, 0
    h.max_bags = 64 * 3
    h.cache, h.host_table = torch.zeros(4, 8), None
    h.perm = h.counts = h.counts_non = h.pop = h.non = h.dense_out = h.step_buffers = None
    h.main = h.side = SimpleNamespace(cuda_stream=0)
    h.clip_sorted = tuple(torch.zeros(192, dtype=torch.int32) for _ in range(3))
    h.clip_sumsq, h.clip_norm, h.clip_ws = torch.zeros(1, dtype=torch.float64), torch.zeros(1), torch.zeros(256, dtype=torch.uint8)
    return h


def test_clipping_goes_by_the_mini_batch_that_step_put_in_the_buffers(hotline):
    """step() fills the buffers that fragment() fills: gradients of fewer bags than its mini-batch has are refused."""
    h = hotline
    h.fragment(None, None, 16)
    h.update_clipped(torch.zeros(16 * 3, 8), 0.1, 1.0)
    h.step(None, None, 50, None, None, 0.1)
    done = len(h.calls)
    with pytest.raises(ValueError):
        h.update_clipped(torch.zeros(16 * 3, 8), 0.1, 1.0)
    assert len(h.calls) == done
    h.update_clipped(torch.zeros(50 * 3, 8), 0.1, 1.0)
    assert len(h.calls) > done


def test_clipping_needs_a_mini_batch_after_a_step_that_failed(hotline, monkeypatch):
    """What the buffers hold then is not known."""
    from paper_2204_05436_b200 import pipeline

    def failing(*a):
        raise RuntimeError
    h = hotline
    h.fragment(None, None, 16)
    monkeypatch.setattr(pipeline.B, "hl_step", failing)
    with pytest.raises(RuntimeError):
        h.step(None, None, 50, None, None, 0.1)
    with pytest.raises(ValueError):
        h.update_clipped(torch.zeros(64 * 3, 8), 0.1, 1.0)


def test_clipping_is_refused_while_mini_batches_are_in_a_pipeline(hl, hotline):
    """Their sorts, ahead on other streams, and their updates use the scratch that the call takes."""
    h = hotline
    grad = torch.zeros(16 * 3, 8)
    for cls, in_flight, idle in [(hl.PipelinedHotline, dict(j_submitted=3, j_done=2), dict(j_submitted=3, j_done=3)),
                                 (hl.NativePipelinedHotline, dict(in_flight=2, pipe=None), dict(in_flight=0, pipe=None))]:
        p = cls.__new__(cls)
        p.__dict__.update(h.__dict__, **in_flight)
        p.fragment(None, None, 16)
        h.calls.clear()
        with pytest.raises(ValueError, match="pipeline"):
            p.update_clipped(grad, 0.1, 1.0)
        assert not h.calls
        p.__dict__.update(idle)
        p.update_clipped(grad, 0.1, 1.0)
        assert len(h.calls) == 4
        p.bags = 0                                   # a mini-batch of start() and step() is not one to clip
        with pytest.raises(ValueError, match="start"):
            p.update_clipped(grad, 0.1, 1.0)


def test_gradient_lists_of_views_that_overlap(hl):
    """What is written shares no byte with what else is read or written, wherever the two begin; what is only read may."""
    flat, out = torch.zeros(200), torch.zeros(400)
    half = torch.zeros(400, dtype=torch.bfloat16)
    a, b, c = flat[:100], flat[50:150], flat[100:]
    for bad in ([(a, a), (b, b)],                    # scaled in place, both
                [(b, b), (a, a)],
                [(a, out[:100]), (b, out[99:199])],  # written twice
                [(a, out[10:110]), (out[:11], None)],  # read, and another's dst
                [(out[109:200], None), (a, out[10:110])],
                [(a, a), (c, None), (flat[99:101], None)],
                [(a, b)], [(b, a)],                  # its own src, shifted
                [(a, half[:100]), (half[99:], None)],
                [(half[:100], half.view(torch.float32)[:100])],
                [(half[:100], half.view(torch.float16)[:100])],
                [(flat, None), (out[:1], flat[199:])],
                [(flat[:1], flat[:1]), (flat, None)]):
        with pytest.raises(ValueError):
            hl.make_tensors(bad)
    for good in ([(a, a), (c, c)],                   # side by side
                 [(a, None), (b, None), (flat, out[:200]), (a, out[200:300]), (b, out[300:])],
                 [(a, c)], [(flat[i:i + 1], flat[i:i + 1]) for i in range(199, -1, -1)],
                 [(half[:100], half.view(torch.float32)[50:150])],
                 [(a, a), (flat[50:50], None), (flat[50:50], flat[60:60])]):       # (empty ones, inside)
        assert len(hl.make_tensors(good)) == len(good)


def test_a_tensor_written_over_a_part_of_itself_is_refused_by_the_library(hl):
    """(Addresses that nothing is read from or written to; a list made by hand.)"""
    P, need = 0x7000_0000_0000, hl.hl_grad_workspace_bytes()
    F32, BF16 = hl.HL_F32, hl.HL_BF16
    for src, dst, n, s, d in [(P, P + 4, 10, F32, F32), (P + 4, P, 10, F32, F32), (P, P + 36, 10, F32, F32), (P, P + 16, 10, BF16, F32),
                              (P + 36, P, 10, BF16, F32), (P, P + 36, 10, F32, BF16), (P, P, 10, BF16, F32)]:
        ts = (hl.hl_tensor * 1)(hl.hl_tensor(src, dst, n, s, d, 0, 0))
        with pytest.raises(hl.HotlineError) as e:
            hl.hl_grad_clip(ts, None, 0, 1.0, P, P + (1 << 20), need, None)
        assert e.value.status == hl.HL_EINVAL


def _values_of(t):
    """Where a matrix's values lie in its storage."""
    return {t.storage_offset() + r * t.stride(0) + c for r in range(t.shape[0]) for c in range(t.shape[1])}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_a_route_writes_shares_nothing_with_the_rows_it_reads(route, dtype):
    """Views of one buffer: columns side by side and rows between rows are taken, wherever they begin; any value in common is not."""
    import random
    r, rng = route, random.Random(1)
    flat, w = torch.zeros(2000, dtype=dtype), torch.zeros(8, 2)

    def view(rows, begin, ld):
        return flat[begin:].as_strided((rows, 6), (ld, 1))

    pairs = [((0, 6), (48, 6)), ((0, 6), (47, 6)), ((96, 6), (0, 6)), ((95, 6), (0, 6)), ((0, 20), (6, 20)), ((0, 20), (5, 20)),
             ((0, 20), (14, 20)), ((0, 20), (15, 20)), ((12, 24), (0, 12)), ((6, 24), (0, 12)), ((0, 6), (0, 6))]
    pairs += [((rng.randint(0, 150), rng.randint(6, 40)), (rng.randint(0, 150), rng.choice([6, 7, 12, 20, 24, 40]))) for _ in range(600)]
    pairs += [((rng.randint(0, 60), 12 * rng.randint(1, 4)), (rng.randint(0, 60), 12 * rng.randint(1, 4))) for _ in range(300)]
    seen = set()
    for few, many in pairs:
        a, b = view(8, *few), view(16, *many)
        shared = bool(_values_of(a) & _values_of(b))
        seen.add(shared)
        for call in (lambda: r.dispatch(a, b), lambda: r.combine(b, w, a), lambda: r.combine_backward(a, None, w, b),
                     lambda: r.dispatch_backward(b, a)):
            r.calls.clear()
            if shared:
                with pytest.raises(ValueError, match="written"):
                    call()
                assert not r.calls
            else:
                call()
                assert len(r.calls) == 1
    assert seen == {True, False}


def test_what_a_route_writes_shares_nothing_with_weights_and_choices(route):
    r = route
    flat = torch.zeros(400)
    x, y, w = torch.zeros(8, 6), torch.zeros(16, 6), flat[:16].view(8, 2)
    grad_w = flat[16:32].view(8, 2)
    rows = lambda begin, n: flat[begin:begin + 6 * n].view(n, 6)              # noqa: E731
    r.combine(y, w, rows(16, 8))
    r.combine_backward(x, y, w, rows(32, 16), grad_w)
    r.combine_backward(x, y, None, rows(0, 16), flat[96:112].view(8, 2))
    e = torch.zeros(8, 2, dtype=torch.int32)
    r._status, r._ws, r._ws_bytes = torch.zeros(1, dtype=torch.int32), None, 0
    r.sort(e)
    n = len(r.calls)
    for bad in (lambda: r.combine(y, w, rows(15, 8)),                          # out, weights
                lambda: r.combine_backward(x, y, w, rows(15, 16), flat[300:316].view(8, 2)),     # grad_y, weights
                lambda: r.combine_backward(x, y, w, rows(31, 16), grad_w),     # grad_y, grad_weights
                lambda: r.combine_backward(x, y, w, rows(32, 16), w),          # grad_weights, weights
                lambda: r.combine_backward(x, y, w, rows(32, 16), flat[15:31].view(8, 2)),
                lambda: r.combine_backward(rows(31, 8), y, w, rows(100, 16), grad_w),            # grad_weights, grad_out
                lambda: r.combine_backward(x, rows(31, 16), w, rows(200, 16), grad_w),           # grad_weights, y
                lambda: r.sort(r.place), lambda: r.sort(r.source.view(8, 2))):
        with pytest.raises(ValueError, match="written"):
            bad()
    assert len(r.calls) == n
