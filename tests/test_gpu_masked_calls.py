"""Windows and drafted trees as a program calls them: layers of a model on an elastic pool and another stream than the default; graphs captured while rows
are short and replayed when they are long; a workspace that is refused to a capture and grows behind it; which form a call takes.  Tolerances:
masked_ops.attention."""
import numpy as np
import pytest
import torch

import masked_ops as M
import plain_ops as P
from test_gpu_prefix import BF16, E4M3, Rows, gpu, values  # noqa: F401  (gpu: fixture)
from test_gpu_windows import form  # noqa: F401  (fixture)
from workloads import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_layers_of_an_elastic_pool_on_another_stream(gpu, dtype):  # noqa: F811
    hq, hkv, d, layers, lens, n = 8, 2, 64, 3, [300, 17, 900], [5, 3, 20]
    c = P.Cache(gpu, hq, hkv, d, dtype, lens, frames=4, n_layers=layers, elastic=True)
    rng = np.random.default_rng(4)
    masks = [M.random_tree(rng, x, 0.6) for x in n]
    kv = []
    for layer in range(layers):
        assert gpu.set_layer(c.m, layer) == 0
        raw = [gen.seq_kv((80, layer, s), x, hkv, d, dtype, 16) for s, x in enumerate(lens)]
        for s, x in enumerate(raw):
            c.fill(s, x)
        kv.append([values(x, dtype) for x in raw])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        gpu.use_current_stream()
        ctx, sees = P.i32(lens), M.words_of(sum(masks, []), 1)
        for layer in (2, 0, 1):
            assert gpu.set_layer(c.m, layer) == 0
            row = lambda s: kv[layer][s]
            q = gen.queries((81, layer), sum(n), hq, d)
            out = [torch.empty((x, hq, d), device="cuda") for x in (len(lens), sum(n), sum(n))]
            assert gpu.decode_attention_window_dev(c.m, P.dev(q[:len(lens)]), ctx, 100, 4, out[0]) == 0
            assert gpu.prefill_attention_window_dev(c.m, P.dev(q), n, ctx, 30, 0, out[1]) == 0
            assert gpu.tree_attention_dev(c.m, P.dev(q), n, ctx, sees, out[2]) == 0
            stream.synchronize()
            M.check(out[0].cpu().double().numpy(), q, row, [1] * len(lens), lambda s: M.window_seen(lens[s], 1, 100, 4))
            M.check(out[1].cpu().double().numpy(), q, row, n, lambda s: M.window_seen(lens[s], n[s], 30, 0))
            M.check(out[2].cpu().double().numpy(), q, row, n, lambda s: M.tree_seen(lens[s], masks[s], 0, 0))
    gpu.use_current_stream()
    assert gpu.set_layer(c.m, 0) == 0 and gpu.device_errors() == 0
    c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, BF16), (16, 8, 64, E4M3)])
def test_rows_grown_since_the_capture(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Captured with the parts that short rows come in, replayed when they are many times as long, and when they are short again."""
    n, start = [4, 30, 1], [600, 40, 16]
    grown = [[3000, 2900, 17], [1, 30, 3000], [2999, 31, 385], start]
    rows = Rows(gpu, hq, hkv, d, dtype, [3000] * 3, frames=100)
    c = rows.c
    for s in range(3):
        gpu.seq_release(c.m, s)
    assert gpu.seq_reserve_batch(c.m, [0, 1, 2], start) >= 0
    rng = np.random.default_rng(5)
    masks = [M.random_tree(rng, x, 0.5) for x in n]
    sees, ctx, q = M.words_of(sum(masks, []), 1), P.i32(start), gen.queries((82, d), sum(n), hq, d)
    out = [torch.zeros((x, hq, d), device="cuda") for x in (3, sum(n), sum(n))]
    q3, qn = P.dev(q[:3]), P.dev(q)

    def calls():
        assert gpu.decode_attention_window_dev(c.m, q3, ctx, 2000, 4, out[0]) == 0
        assert gpu.prefill_attention_window_dev(c.m, qn, n, ctx, 2500, 5, out[1]) == 0
        assert gpu.tree_attention_dev(c.m, qn, n, ctx, sees, out[2]) == 0

    calls()
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        gpu.use_current_stream()
        calls()
    gpu.use_current_stream()
    for upto in range(48, 3048, 48):
        assert gpu.seq_reserve_batch(c.m, [0, 1, 2], [min(upto, 3000)] * 3) >= 0
    for s in range(3):
        c.fill(s, gen.seq_kv((7, s), 3000, hkv, d, dtype, 16, peak_frac=0.02), 3000)
    for lens in [start] + grown:
        ctx.copy_(P.i32(lens))
        for x in out:
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got, row = [x.cpu().double().numpy() for x in out], lambda s: rows.kv[s]
        before = lambda s: max(n[s] - lens[s], 0)                        # queries that stand before their row
        M.check(got[0], q, row, [1] * 3, lambda s: M.window_seen(lens[s], 1, 2000, 4))
        M.check(got[1], q, row, n, lambda s: np.concatenate([np.zeros((before(s), lens[s]), dtype=bool), M.window_seen(lens[s], n[s] - before(s), 2500, 5)]))
        M.check(got[2], q, row, n, lambda s: M.tree_seen(lens[s], masks[s], 0, 0))
    assert gpu.device_errors() == 0
    del graph
    c.close()


def test_groups_in_parts_captured_and_replayed(gpu):  # noqa: F811
    """Refused to a capture while there is no workspace, then captured; a larger eager call between replays makes a larger workspace, and the graph goes on
    with its own."""
    hq, hkv, d, n, lens = 16, 2, 64, [40, 40, 40], [6000, 5000, 4000]
    rows = Rows(gpu, hq, hkv, d, BF16, lens, frames=60)
    c, rng = rows.c, np.random.default_rng(6)
    masks = [M.random_tree(rng, 40, 0.5) for _ in n]
    sees, ctx, q = M.words_of(sum(masks, []), 1), P.i32(lens[:1]), P.dev(gen.queries((83,), 120, hq, d))
    out, eager = (torch.zeros((120, hq, d), device="cuda") for _ in range(2))
    call = lambda o, k=1, x=ctx: gpu.tree_attention_dev(c.m, q, n[:k], x, sees, o)
    stream, graph, refused = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    assert gpu.set_mask_form(1) == 0
    torch.cuda.synchronize()
    with torch.cuda.graph(refused, stream=stream):
        gpu.use_current_stream()
        assert call(out) == -3 and "capture" in gpu.last_error()
    gpu.use_current_stream()
    assert call(out) == 0
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        gpu.use_current_stream()
        assert call(out) == 0
    gpu.use_current_stream()
    for step, x in enumerate((6000, 5999, 2000, 41)):
        ctx.copy_(P.i32([x]))
        q.copy_(P.dev(gen.queries((84, step), 120, hq, d)))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        M.check(out[:40].cpu().double().numpy(), P.host(q), lambda s: rows.kv[s], n[:1], lambda s: M.tree_seen(x, masks[0], 0, 0))
        if step == 1:
            assert call(eager, 3, P.i32(lens)) == 0
            torch.cuda.synchronize()
            M.check(eager.cpu().double().numpy(), P.host(q), lambda s: rows.kv[s], n, lambda s: M.tree_seen(lens[s], masks[s], 0, 0))
    gpu.set_mask_form(-1)
    assert gpu.device_errors() == 0
    del graph, refused
    c.close()


def test_which_form(gpu):  # noqa: F811
    """Up to 16 columns units of 16, beyond 128 groups; between by what is read: few short rows as units, many long ones as groups."""
    for hq, hkv, d, batch, held, nodes, want in ((32, 8, 128, 4, 500, 4, 0), (4, 4, 64, 2, 300, 16, 0), (16, 4, 128, 2, 500, 33, 1), (16, 8, 128, 16, 500, 20, 0),
                                                 (16, 4, 128, 64, 3000, 16, 1)):
        c = P.Cache(gpu, hq, hkv, d, E4M3 if want == 0 else BF16, [held] * batch, frames=500)
        q, out = torch.zeros((batch * nodes, hq, d), dtype=torch.int16, device="cuda"), torch.full((batch * nodes, hq, d), float("nan"), device="cuda")
        # (what is held decides, not what is seen: contexts of no token)
        assert gpu.tree_attention_dev(c.m, q, [nodes] * batch, P.i32([0] * batch), M.words_of([0] * batch * nodes, 1), out) == 0
        assert gpu.last_mask_form() == want, (hq, hkv, batch, held, nodes)
        assert not out.any()
        c.close()


def test_largest_and_smallest(gpu, form):  # noqa: F811
    """One token of one row; as many drafts as a mask takes, in one row behind nothing; windows of one token; 16 heads a kv head."""
    hq, hkv, d = 16, 1, 128
    rows = Rows(gpu, hq, hkv, d, BF16, [256, 1, 30])
    rng = np.random.default_rng(7)
    for masks, lens in (([[1]], [1]), ([M.random_tree(rng, 256, 0.3)], [256]), ([M.random_tree(rng, 1, 0.3), [1], [1] * 2], [256, 1, 30])):
        n = [len(x) for x in masks]
        q, out = gen.queries((85, sum(n)), sum(n), hq, d), torch.full((sum(n), hq, d), float("nan"), device="cuda")
        for window in (0, 256):
            assert gpu.tree_attention_dev(rows.c.m, P.dev(q), n, P.i32(lens), M.words_of(sum(masks, []), 4), out, window, 0) == 0
            M.check(out.cpu().double().numpy(), q, lambda s: rows.kv[s], n, lambda s: M.tree_seen(lens[s], masks[s], window, 0))
        assert gpu.prefill_attention_window_dev(rows.c.m, P.dev(q), n, P.i32(lens), 1, 0, out) == 0
        M.check(out.cpu().double().numpy(), q, lambda s: rows.kv[s], n, lambda s: M.window_seen(lens[s], n[s], 1, 0))
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("n", [200, 1000])
def test_many_sequences(gpu, n):  # noqa: F811
    """More sequences than a launch's shorter and longer plan hold: drafts appended, attended to, kept; no rotation, so that keys are what came in."""
    hq, hkv, d = 4, 1, 64
    rng = np.random.default_rng(n)
    base, new = rng.integers(0, 40, n).tolist(), rng.integers(0, 7, n).tolist()
    c = P.Cache(gpu, hq, hkv, d, BF16, [x + 7 for x in base], frames=40)
    masks = [M.random_tree(rng, x, 0.5) for x in new]
    total, ctx = sum(new), [a + b for a, b in zip(base, new)]
    kv = []
    for s, x in enumerate(base):
        raw = gen.seq_kv((86, s), max(x, 1), hkv, d, BF16, 16)
        c.fill(s, raw, x)
        kv.append([P.f64(raw[y][:x]) for y in ("k", "v")])
    q, k, v = (gen.queries((87, i), total, h, d) for i, h in enumerate((hq, hkv, hkv)))
    at = np.cumsum([0] + new)
    for s in range(n):
        kv[s] = [np.concatenate([old, P.f64(x[at[s]:at[s + 1]])]) for old, x in zip(kv[s], (k, v))]
    sees, lens = M.words_of(sum(masks, []), 1), P.i32(ctx)
    q_out, out = torch.zeros((total, hq, d), dtype=torch.int16, device="cuda"), torch.full((total, hq, d), float("nan"), device="cuda")
    assert gpu.qkv_append_tree_dev(c.m, P.dev(q), P.dev(k), P.dev(v), new, lens, sees, q_out) == total
    assert gpu.tree_attention_dev(c.m, q_out, new, lens, sees, out) == 0
    torch.cuda.synchronize()
    assert np.array_equal(P.host(q_out).view(np.int16), q.view(np.int16))
    M.check(out.cpu().double().numpy(), q, lambda s: kv[s], new, lambda s: M.tree_seen(ctx[s], masks[s], 0, 0))
    paths = [M.path_of(x[int(rng.integers(len(x)))]) if x else [] for x in masks]
    packed = sum([p + [0] * (m - len(p)) for p, m in zip(paths, new)], [])
    left = P.i32([0] * n)
    assert gpu.kv_keep_dev(c.m, new, lens, P.i32(packed), P.i32([len(p) for p in paths]), left) == n
    torch.cuda.synchronize()
    assert left.tolist() == [b + len(p) for b, p in zip(base, paths)]
    for s in rng.choice(n, 60, replace=False).tolist() + [0, n - 1]:
        rows = list(range(base[s])) + [base[s] + j for j in paths[s]]
        if rows:
            for got, want in zip(c.read(s, 0, len(rows)), kv[s]):
                assert np.array_equal(got, want[rows]), s
    assert gpu.device_errors() == 0
    c.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_blocks_beyond_4_gib(gpu, form, dtype):  # noqa: F811
    """Rows whose blocks lie all over a pool of 5 GiB: read under windows and masks, moved together."""
    hq, hkv, d, n, lens = 16, 4, 128, [5, 20], [400, 300]
    rows = Rows(gpu, hq, hkv, d, dtype, lens, frames=5120)
    c, rng = rows.c, np.random.default_rng(8)
    masks = [M.random_tree(rng, x, 0.5) for x in n]
    ctx, q = P.i32(lens), gen.queries((88,), sum(n), hq, d)
    out = [torch.full((x, hq, d), float("nan"), device="cuda") for x in (2, sum(n), sum(n))]
    assert gpu.decode_attention_window_dev(c.m, P.dev(q[:2]), ctx, 150, 4, out[0]) == 0
    assert gpu.prefill_attention_window_dev(c.m, P.dev(q), n, ctx, 150, 4, out[1]) == 0
    assert gpu.tree_attention_dev(c.m, P.dev(q), n, ctx, M.words_of(sum(masks, []), 1), out[2]) == 0
    got, row = [x.cpu().double().numpy() for x in out], lambda s: rows.kv[s]
    M.check(got[0], q, row, [1, 1], lambda s: M.window_seen(lens[s], 1, 150, 4))
    M.check(got[1], q, row, n, lambda s: M.window_seen(lens[s], n[s], 150, 4))
    M.check(got[2], q, row, n, lambda s: M.tree_seen(lens[s], masks[s], 0, 0))
    before = [c.read(s, 0, x) for s, x in enumerate(lens)]
    assert gpu.kv_keep_dev(c.m, n, ctx, P.i32([0, 3, 0, 0, 0] + [2, 19] + [0] * 18), P.i32([2, 2])) == 2
    for s, stay in enumerate(([395, 398], [282, 299])):
        # (moved into an e4m3 block: within half a step of its values, and of bf16 on the way, under a scale that may have grown: e4m3 2^-4, bf16 2^-8 relative, or
        # half the lowest step, 2^-10, of the scale, which no value here has above 2^-3)
        for x, y in zip(c.read(s, lens[s] - n[s], 2), before[s]):
            assert np.all(np.abs(x - y[stay]) <= (0.0 if dtype == BF16 else 1.0) * (np.abs(y[stay]) * (2.0 ** -4 + 2.0 ** -7) + 2.0 ** -13)), s
    assert gpu.device_errors() == 0
    c.close()


@pytest.mark.parametrize("items", [1, 64, 700, 100000])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(16, 4, 128, BF16), (4, 4, 64, E4M3)])
def test_cut_as_asked(gpu, form, hq, hkv, d, dtype, items):  # noqa: F811
    """Any number of parts: one, a few, more than the workspace has room for."""
    n, lens = [3, 50, 1, 8], [5000, 1200, 40, 8]
    rows = Rows(gpu, hq, hkv, d, dtype, lens, frames=100)
    rng, ctx = np.random.default_rng(items), P.i32(lens)
    masks = [M.random_tree(rng, x, 0.5) for x in n]
    q, row = gen.queries((89, d), sum(n), hq, d), lambda s: rows.kv[s]
    out = [torch.full((x, hq, d), float("nan"), device="cuda") for x in (4, sum(n), sum(n))]
    assert gpu.set_split(items, 0) == 0
    try:
        assert gpu.decode_attention_window_dev(rows.c.m, P.dev(q[:4]), ctx, 3000, 20, out[0]) == 0
        assert gpu.prefill_attention_window_dev(rows.c.m, P.dev(q), n, ctx, 3000, 20, out[1]) == 0
        assert gpu.tree_attention_dev(rows.c.m, P.dev(q), n, ctx, M.words_of(sum(masks, []), 1), out[2]) == 0
    finally:
        gpu.set_split(0, 0)
    got = [x.cpu().double().numpy() for x in out]
    M.check(got[0], q, row, [1] * 4, lambda s: M.window_seen(lens[s], 1, 3000, 20))
    M.check(got[1], q, row, n, lambda s: M.window_seen(lens[s], n[s], 3000, 20))
    M.check(got[2], q, row, n, lambda s: M.tree_seen(lens[s], masks[s], 0, 0))
    assert gpu.device_errors() == 0
    rows.c.close()
