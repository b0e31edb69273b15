"""Attention with sliding windows and sinks, decode steps and prefill chunks, against 64 bits (tolerances: masked_ops.attention)."""
import numpy as np
import pytest
import torch

import masked_ops as M
import plain_ops as P
from test_gpu_prefix import BF16, E4M3, SHAPES, Rows, gpu  # noqa: F401  (gpu: fixture)
from workloads import gen

pytestmark = pytest.mark.gpu

WINDOWS = [(1, 0), (1, 1), (16, 0), (17, 4), (5, 40), (100, 4), (64, 16), (130, 33), (1000, 0), (1 << 30, 3), (2147483647, 2147483647)]


@pytest.fixture(params=[0, 1, 2], ids=["units of 16", "groups of 128", "units of 32"])
def form(gpu, request):  # noqa: F811
    """The ways in which chunks and trees fall into work-groups."""
    assert gpu.set_mask_form(request.param) == 0
    yield request.param
    gpu.set_mask_form(-1)


def decode(gpu, rows, q, ctx, window, sinks):  # noqa: F811
    c = rows.c
    out = torch.full((len(ctx), c.hq, c.d), float("nan"), device="cuda")
    assert gpu.decode_attention_window_dev(c.m, P.dev(q), P.i32(ctx), window, sinks, out) == 0
    M.check(out.cpu().double().numpy(), q, lambda s: rows.kv[s], [1] * len(ctx), lambda s: M.window_seen(ctx[s], 1, window, sinks))


def prefill(gpu, rows, q, n, ctx, window, sinks):  # noqa: F811
    c = rows.c
    out = torch.full((sum(n), c.hq, c.d), float("nan"), device="cuda")
    assert gpu.prefill_attention_window_dev(c.m, P.dev(q), n, P.i32(ctx), window, sinks, out) == 0
    M.check(out.cpu().double().numpy(), q, lambda s: rows.kv[s], n, lambda s: M.window_seen(ctx[s], n[s], window, sinks))


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_decode(gpu, hq, hkv, d, dtype):  # noqa: F811
    """Contexts of no token, of one, around the ends of pages and windows, and of many windows; windows and sinks that meet, overlap or leave a gap."""
    lens = [0, 1, 2, 15, 16, 17, 31, 33, 64, 100, 101, 130, 163, 250, 700, 1500]
    rows = Rows(gpu, hq, hkv, d, dtype, lens, frames=100)
    for i, (window, sinks) in enumerate(WINDOWS):
        decode(gpu, rows, gen.queries((31, d, i), len(lens), hq, d), lens, window, sinks)
    # fewer tokens than the rows hold, and one sequence
    decode(gpu, rows, gen.queries((32, d), len(lens), hq, d), [x // 2 for x in lens], 40, 5)
    decode(gpu, rows, gen.queries((33, d), 3, hq, d), lens[:3], 2, 1)
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 1, 128, BF16), (4, 4, 64, E4M3)])
def test_decode_wide_windows_of_few_rows(gpu, hq, hkv, d, dtype):  # noqa: F811
    """Rows whose windows are cut into parts; among them rows without tokens, and short ones."""
    lens = [20000, 3, 0, 9000]
    rows = Rows(gpu, hq, hkv, d, dtype, lens, frames=100)
    for window, sinks in ((8000, 4), (4001, 500), (12345, 0), (20000, 1), (33, 9000)):
        decode(gpu, rows, gen.queries((34, window), 4, hq, d), lens, window, sinks)
        decode(gpu, rows, gen.queries((35, window), 1, hq, d), lens[:1], window, sinks)
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_prefill(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Ragged chunks: none, one, around tiles, several windows long, behind nothing and behind long contexts; queries before their row."""
    n = [1, 0, 7, 33, 64, 150, 5, 300, 40, 16]
    ctx = [1, 20, 7, 50, 1000, 150, 999, 301, 25, 16]                    # row 8: 15 queries stand before position 0
    rows = Rows(gpu, hq, hkv, d, dtype, [max(x, 1) for x in ctx], frames=100)
    for i, (window, sinks) in enumerate(WINDOWS):
        q = gen.queries((36, d, i), sum(n), hq, d)
        out = torch.full((sum(n), hq, d), float("nan"), device="cuda")
        assert gpu.prefill_attention_window_dev(rows.c.m, P.dev(q), n, P.i32(ctx), window, sinks, out) == 0
        got = out.cpu().double().numpy()
        seen = lambda s: np.concatenate([np.zeros((max(n[s] - ctx[s], 0), ctx[s]), dtype=bool), M.window_seen(ctx[s], min(n[s], ctx[s]), window, sinks)])
        M.check(got, q, lambda s: rows.kv[s], n, seen)
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, BF16), (8, 1, 64, BF16), (16, 2, 128, E4M3)])
def test_prefill_long(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Prompts of many groups, and few queries whose wide window is cut into parts."""
    rows = Rows(gpu, hq, hkv, d, dtype, [1200, 9000, 700], frames=200)
    q = gen.queries((37, d), 1200 + 3 + 650, hq, d)
    for window, sinks in ((256, 4), (1000, 0), (8500, 20)):
        prefill(gpu, rows, q, [1200, 3, 650], [1200, 9000, 700], window, sinks)
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_seen_may_hold_anything(gpu, form, d, value):  # noqa: F811
    """NaN and infinities in tokens between the sinks and the window, and (the pool is all NaN) behind the context."""
    hq, hkv, lens, window, sinks = 8, 2, [300, 77, 1000], 50, 5
    rows = Rows(gpu, hq, hkv, d, BF16, lens)
    for s, n in enumerate(lens):
        k, v = (P.bits(x) for x in rows.kv[s])
        k, v = k.copy(), v.copy()
        bad = int(P.bits(np.array([value]))[0])
        k[sinks:n - window - 3], v[sinks:n - window - 3] = bad, bad
        rows.c.fill(s, {"k": k, "v": v})
    q = gen.queries((38, d), 3, hq, d)
    decode(gpu, rows, q, lens, window, sinks)
    q = gen.queries((39, d), 12, hq, d)
    prefill(gpu, rows, q, [4, 4, 4], lens, window, sinks)
    rows.c.close()


def test_as_the_calls_without_windows(gpu, form):  # noqa: F811
    """A window that covers everything: the rows of decode_attention and prefill_attention, up to the order of sums."""
    hq, hkv, d, lens = 32, 8, 128, [0, 5, 600, 2000, 31]
    rows = Rows(gpu, hq, hkv, d, BF16, lens, frames=60)
    ctx, n = P.i32(lens), [0, 5, 20, 100, 31]
    q = gen.queries((40,), 5, hq, d)
    a, b = (torch.empty((5, hq, d), device="cuda") for _ in range(2))
    assert gpu.decode_attention_dev(rows.c.m, P.dev(q), ctx, a) == 0 and gpu.decode_attention_window_dev(rows.c.m, P.dev(q), ctx, 1 << 29, 0, b) == 0
    M.same(a, b, q, lambda s: rows.kv[s], [1] * 5, lambda s: M.window_seen(lens[s], 1, 1 << 29, 0))
    q = gen.queries((41,), sum(n), hq, d)
    a, b = (torch.empty((sum(n), hq, d), device="cuda") for _ in range(2))
    assert gpu.prefill_attention_dev(rows.c.m, P.dev(q), n, ctx, a) == 0 and gpu.prefill_attention_window_dev(rows.c.m, P.dev(q), n, ctx, 2000, 0, b) == 0
    M.same(a, b, q, lambda s: rows.kv[s], n, lambda s: M.window_seen(lens[s], n[s], 2000, 0))
    rows.c.close()


def test_many_sequences(gpu, form):  # noqa: F811
    """More sequences than a launch's plan holds."""
    hq, hkv, d, n = 4, 1, 64, 1000
    rng = np.random.default_rng(6)
    lens = [int(x) for x in rng.integers(1, 60, n)]
    rows = Rows(gpu, hq, hkv, d, BF16, lens, frames=40)
    decode(gpu, rows, gen.queries((42,), n, hq, d), lens, 20, 3)
    new = [int(min(x, y)) for x, y in zip(rng.integers(0, 9, n), lens)]
    prefill(gpu, rows, gen.queries((43,), sum(new), hq, d), new, lens, 20, 3)
    assert gpu.device_errors() == 0
    rows.c.close()


def test_refusals(gpu):  # noqa: F811
    hq, hkv, d = 8, 2, 64
    rows = Rows(gpu, hq, hkv, d, BF16, [40, 20])
    m, q, ctx, out = rows.c.m, P.dev(gen.queries((44,), 4, hq, d)), P.i32([40, 20]), torch.zeros((4, hq, d), device="cuda")
    dec = lambda model=m, q=q, ctx=ctx, window=8, sinks=2, out=out: gpu.decode_attention_window_dev(model, q, ctx, window, sinks, out)
    pre = lambda model=m, q=q, n=(2, 2), ctx=ctx, window=8, sinks=2, out=out: gpu.prefill_attention_window_dev(model, q, n, ctx, window, sinks, out)
    for call in (dec, pre):
        assert call(model=63) == -2 and call(window=0) == -1 and call(window=-5) == -1 and call(sinks=-1) == -1
        assert call(q=None) == -1 and call(out=None) == -1 and call(out=out.flatten()[1:]) == -1 and call(q=q.flatten()[1:]) == -1
    three = P.i32([1, 1, 1])
    assert dec(ctx=three) == -6 and pre(ctx=three, n=(1, 1, 1)) == -6 and pre(n=(-1, 2)) == -1 and pre(n=(1 << 24, 1)) == -6
    assert dec(ctx=P.i32([])) == 0 and pre(ctx=P.i32([]), n=()) == 0 and pre(n=(0, 0)) == 0
    torch.cuda.synchronize()
    assert not out.any() and gpu.device_errors() == 0
    rows.c.close()


def test_captured_and_replayed(gpu):  # noqa: F811
    """A decode step captured while rows are short, replayed when they have grown out of their windows; eager calls between."""
    hq, hkv, d, n = 16, 2, 128, 6
    rows = Rows(gpu, hq, hkv, d, BF16, [1500] * n, frames=60)
    c, q, ctx = rows.c, P.dev(gen.queries((45,), n, hq, d)), P.i32([3] * n)
    out, eager = (torch.zeros((n, hq, d), device="cuda") for _ in range(2))
    call = lambda o: gpu.decode_attention_window_dev(c.m, q, ctx, 700, 4, o)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        gpu.use_current_stream()
        assert call(out) == 0
    gpu.use_current_stream()
    for step, lens in enumerate(([3, 0, 1, 16, 700, 703], [800, 1500, 1499, 704, 705, 17], [900] * 6)):
        ctx.copy_(P.i32(lens))
        q.copy_(P.dev(gen.queries((46, step), n, hq, d)))
        graph.replay()
        torch.cuda.synchronize()
        M.check(out.cpu().double().numpy(), P.host(q), lambda s: rows.kv[s], [1] * n, lambda s: M.window_seen(lens[s], 1, 700, 4))
        assert call(eager) == 0
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        out.zero_()
    assert gpu.device_errors() == 0
    del graph
    c.close()
