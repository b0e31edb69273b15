"""Drafted trees: their attention over the cache, against 64 bits (tolerances: masked_ops.attention); their way into the cache at the positions of their
depths; the accepted tokens moved together."""
import numpy as np
import pytest
import torch

import masked_ops as M
import plain_ops as P
from test_gpu_prefix import BF16, E4M3, SHAPES, Rows, gpu  # noqa: F401  (gpu: fixture)
from test_gpu_qkv_append import close, inputs, weights
from test_gpu_windows import form  # noqa: F401  (fixture)
from workloads import gen

pytestmark = pytest.mark.gpu


def attend(gpu, rows, q, masks, ctx, window=0, sinks=0, words=None):  # noqa: F811
    c, n = rows.c, [len(x) for x in masks]
    words = words or max(1, (max(n) + 63) // 64)
    out = torch.full((sum(n), c.hq, c.d), float("nan"), device="cuda")
    assert gpu.tree_attention_dev(c.m, P.dev(q), n, P.i32(ctx), M.words_of(sum(masks, []), words), out, window, sinks) == 0
    M.check(out.cpu().double().numpy(), q, lambda s: rows.kv[s], n, lambda s: M.tree_seen(ctx[s], masks[s], window, sinks))


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_trees(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Trees of no token, of one, of odd numbers and across the ends of pages and mask words, behind no context, short and long ones."""
    n = [1, 0, 5, 26, 60, 7, 64, 2, 33, 16]
    base = [0, 50, 0, 300, 1000, 31, 17, 16, 0, 700]
    rng = np.random.default_rng(hq + d)
    ctx = [a + b for a, b in zip(base, n)]
    rows = Rows(gpu, hq, hkv, d, dtype, [max(x, 1) for x in ctx], frames=100)
    for i, (branch, window, sinks) in enumerate(((0.0, 0, 0), (0.4, 0, 7), (0.8, 64, 0), (0.5, 100, 4), (1.0, 250, 33))):
        masks = [M.random_tree(rng, x, branch) for x in n]
        attend(gpu, rows, gen.queries((51, d, i), sum(n), hq, d), masks, ctx, window, sinks, 1 + i % 4)
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(16, 4, 128, BF16), (3, 3, 64, E4M3)])
def test_any_mask(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Masks that are no trees: any bits, none, all; bits behind the drafts, which are not looked at; up to 256 drafted tokens; a context length below
    the number of drafts, and one beyond the row's blocks."""
    rng = np.random.default_rng(d)
    n, base = [256, 100, 9, 65, 20, 4], [40, 0, 200, 33, -6, 60]
    any_bits = lambda k: int.from_bytes(rng.bytes(32), "little") >> int(rng.integers(0, 250)) if k % 3 else 0
    masks = [[any_bits(k) for k in range(x)] for x in n]
    masks[1][0] = (1 << 256) - 1
    ctx = [a + b for a, b in zip(base, n)]
    rows = Rows(gpu, hq, hkv, d, dtype, [max(x, 1) for x in ctx], frames=100)
    q = gen.queries((52, d), sum(n), hq, d)
    attend(gpu, rows, q, masks, ctx, 0, 0, 4)
    attend(gpu, rows, q, masks, ctx, 256, 3, 4)
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, BF16), (8, 1, 64, BF16), (64, 8, 128, BF16), (16, 2, 128, E4M3), (4, 1, 64, E4M3)])
def test_trees_behind_long_contexts(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Few drafted tokens and many in front of contexts that are cut into parts."""
    n, base = [3, 40, 1], [9000, 5000, 12000]
    rng = np.random.default_rng(9)
    ctx = [a + b for a, b in zip(base, n)]
    rows = Rows(gpu, hq, hkv, d, dtype, ctx, frames=240)
    masks = [M.random_tree(rng, x, 0.5) for x in n]
    q = gen.queries((53, d), sum(n), hq, d)
    attend(gpu, rows, q, masks, ctx)
    attend(gpu, rows, q, masks, ctx, 7000, 5)
    attend(gpu, rows, q[:3], masks[:1], ctx[:1])
    assert gpu.device_errors() == 0
    rows.c.close()


def test_chain_is_a_chunk(gpu, form):  # noqa: F811
    """A tree without branches sees what a chunk's queries see."""
    hq, hkv, d, n, base = 32, 8, 128, [7, 30, 1], [100, 0, 515]
    ctx = [a + b for a, b in zip(base, n)]
    rows = Rows(gpu, hq, hkv, d, BF16, ctx)
    q = gen.queries((54,), sum(n), hq, d)
    a, b = (torch.empty((sum(n), hq, d), device="cuda") for _ in range(2))
    masks = sum([[(2 << i) - 1 for i in range(x)] for x in n], [])
    assert gpu.prefill_attention_dev(rows.c.m, P.dev(q), n, P.i32(ctx), a) == 0
    assert gpu.tree_attention_dev(rows.c.m, P.dev(q), n, P.i32(ctx), M.words_of(masks, 1), b) == 0
    M.same(a, b, q, lambda s: rows.kv[s], n, lambda s: M.window_seen(ctx[s], n[s], ctx[s], 0))
    rows.c.close()


# rot, pairs, norm, pad, shift
@pytest.mark.parametrize("form", [("all", False, True, 0, 0), ("all", True, False, 8, 0), (20, False, True, 5, 1), (0, False, True, 0, 0)], ids=str)
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (5, 5, 64)])
def test_append(gpu, hq, hkv, d, form):  # noqa: F811
    """Queries and keys at the positions of their depths; an e4m3 cache bit for bit what kv_append_chunk makes of those keys; a chain bit for bit
    what qkv_append_chunk makes of it."""
    rot, pairs, norm, pad, shift = form
    rot = d if rot == "all" else rot
    freq = P.frequencies(rot) if rot else None
    rid = gpu.rotary_create(rot, int(pairs), freq, 1.25) if rot else -1
    n, base, before = [1, 0, 33, 16, 70, 5], [0, 9, 5, 32, 31, 16], [0, 7, 100, 1 << 20, 12345, 2000000000]
    rng = np.random.default_rng(d)
    masks = [M.random_tree(rng, x, 0.5) for x in n]
    masks[2][3] = 0                                                      # sees nothing: at its base
    ctx, rows = [a + b for a, b in zip(base, n)], sum(n)
    caches = {name: P.Cache(gpu, hq, hkv, d, dt, [x + 1 for x in ctx], frame_bytes=4 << 20, frames=8) for name, dt in
              (("bf16", BF16), ("e4m3", E4M3), ("again", E4M3), ("chain", BF16), ("chunk", BF16))}
    for s, x in enumerate(base):
        if x:
            for name, c in caches.items():
                c.fill(s, gen.seq_kv((61, s), x, hkv, d, c.dtype, 16))
    (wq, wk), (wq64, wk64) = weights((62, d), d) if norm else ((None, None), (None, None))
    (q, k, v), (q_b, k_b, v_b) = inputs((63, d), rows, hq, hkv, d, pad, shift)
    out = {name: torch.full((rows, hq, d), -1, dtype=torch.int16, device="cuda") for name in caches}
    tail = (wq, wk, 1e-6, rid, P.i32(before))
    sees, chain = M.words_of(sum(masks, []), 2), M.words_of(sum([[(2 << i) - 1 for i in range(x)] for x in n], []), 2)
    for name, bits in (("bf16", sees), ("e4m3", sees), ("chain", chain)):
        assert gpu.qkv_append_tree_dev(caches[name].m, q, k, v, n, P.i32(ctx), bits, out[name], *tail) == rows
    assert gpu.qkv_append_chunk_dev(caches["chunk"].m, q, k, v, n, P.i32(ctx), out["chunk"], *tail) == rows
    torch.cuda.synchronize()
    assert torch.equal(out["bf16"], out["e4m3"]) and torch.equal(out["chain"], out["chunk"])
    depth = np.array(sum([M.positions(x) for x in masks], []))
    pos = np.repeat(np.array(before, dtype=np.int64) + base, n) + depth
    want, size = P.turned(P.f64(q_b), pos, wq64, 1e-6, rot, pairs, freq, 1.25)
    assert close(P.f64(P.host(out["bf16"])), want, size)
    read = {name: [gpu.kv_read(c.m, s, 0, x)[1:] if x else None for s, x in enumerate(ctx)] for name, c in caches.items() if name != "again"}
    kb, vb = (np.concatenate([r[i][b:] for r, b in zip(read["bf16"], base) if r]) for i in (0, 1))
    want, size = P.turned(P.f64(k_b), pos, wk64, 1e-6, rot, pairs, freq, 1.25)
    assert close(P.f64(kb), want, size) and np.array_equal(vb, v_b)
    assert gpu.kv_append_chunk_dev(caches["again"].m, P.dev(kb), P.dev(vb), n, P.i32(ctx)) == rows
    for s, x in enumerate(ctx):
        if x:
            for a, b in zip(read["e4m3"][s], gpu.kv_read(caches["again"].m, s, 0, x)[1:]):
                assert np.array_equal(a, b), s
            for a, b in zip(read["chain"][s], read["chunk"][s]):
                assert np.array_equal(a, b), s
    assert gpu.device_errors() == 0
    if rot:
        assert gpu.rotary_destroy(rid) == 0
    for c in caches.values():
        c.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("hkv,d,layers", [(8, 128, 1), (3, 64, 4)])
def test_keep(gpu, dtype, hkv, d, layers):  # noqa: F811
    """Every layer of every row against kv_gather of the tokens that move and kv_append_chunk of them on a copy whose drafts were never there: bit for
    bit.  Paths of none, of one, all in place, the last alone, across pages; values that raise the scales."""
    hq = hkv
    n = [1, 0, 26, 40, 100, 16, 33, 64, 5]
    base = [0, 20, 16, 31, 7, 0, 45, 1, 100]
    rng = np.random.default_rng(d + dtype)
    kept = [[0], [], [0, 1, 2], [0, 1, 5, 6, 20, 39], sorted(rng.choice(100, 50, replace=False).tolist()), list(range(16)), [32], [], [1, 2, 4]]
    ctx, tokens = [a + b for a, b in zip(base, n)], sum(n)
    a, b = (P.Cache(gpu, hq, hkv, d, dtype, [x + 1 for x in ctx], frame_bytes=4 << 20, frames=8, n_layers=layers) for _ in range(2))
    g = gen.generator(64, d)
    first = np.cumsum([0] + n)
    drafts = []
    for layer in range(layers):
        gpu.set_layer(a.m, layer), gpu.set_layer(b.m, layer)
        for s, x in enumerate(base):
            if x:
                kv = gen.seq_kv((65, s, layer), x, hkv, d, dtype, 16)
                a.fill(s, kv), b.fill(s, kv)
        size = torch.exp(1.5 * torch.randn((tokens, 1, 1), generator=g))
        k, v = (P.dev(gen.to_bf16_bits(torch.randn((tokens, hkv, d), generator=g) * size)) for _ in range(2))
        assert gpu.kv_append_chunk_dev(a.m, k, v, n, P.i32(ctx)) == tokens
        assert gpu.kv_append_chunk_dev(b.m, k, v, n, P.i32(ctx)) == tokens
        drafts.append([gpu.kv_read(a.m, s, 0, x) for s, x in enumerate(ctx)])
    # the copy: what moves is gathered token by token, then appended behind those that are in their place
    for layer in range(layers):
        gpu.set_layer(b.m, layer)
        stay = [next((j for j, x in enumerate(p) if x != j), len(p)) for p in kept]
        moved = [p[j:] for p, j in zip(kept, stay)]
        rows = sum(len(x) for x in moved)
        kb, vb = (torch.empty((rows, hkv, d), dtype=torch.int16, device="cuda") for _ in range(2))
        seqs = [s for s, p in enumerate(moved) for _ in p]
        assert gpu.kv_gather_dev(b.m, seqs, [base[s] + x for s, p in enumerate(moved) for x in p], [1] * rows, kb, vb) == rows
        assert gpu.kv_append_chunk_dev(b.m, kb, vb, [len(p) for p in moved], P.i32([x + j + len(p) for x, j, p in zip(base, stay, moved)])) == rows
    packed = np.full(tokens, -7, dtype=np.int32)
    for s, p in enumerate(kept):
        packed[first[s]:first[s] + len(p)] = p
    lens = torch.full((len(n),), -1, dtype=torch.int32, device="cuda")
    gpu.set_layer(a.m, layers - 1)                                        # (all layers, whichever is set)
    assert gpu.kv_keep_dev(a.m, n, P.i32(ctx), P.i32(packed), P.i32([len(p) for p in kept]), lens) == len(n)
    torch.cuda.synchronize()
    assert lens.tolist() == [x + len(p) for x, p in zip(base, kept)]
    for layer in range(layers):
        gpu.set_layer(a.m, layer), gpu.set_layer(b.m, layer)
        for s, p in enumerate(kept):
            if base[s] + len(p):
                got, want = (gpu.kv_read(c.m, s, 0, base[s] + len(p))[1:] for c in (a, b))
                for x, y in zip(got, want):
                    assert x is None and y is None or np.array_equal(x, y), (layer, s)
            if dtype == BF16 and base[s]:                                  # what is in front is not touched
                assert np.array_equal(gpu.kv_read(a.m, s, 0, base[s])[1], drafts[layer][s][1][:base[s]])
    assert gpu.device_errors() == 0
    a.close(), b.close()


def test_keep_refuses_rows(gpu):  # noqa: F811
    """Entries out of order or of range, counts and context lengths that do not fit: the row stays as it is, others go on."""
    hkv, d, n = 2, 64, 8
    cases = [([0, 2], 2, 20), ([2, 2], 2, 20), ([3, 1], 2, 20), ([7, 8], 2, 20), ([-1, 3], 2, 20), ([1], -1, 20), ([1], 9, 20), ([1], 1, 7), ([1], 1, 49), ([1, 3], 2, 20)]
    c = P.Cache(gpu, hkv, hkv, d, BF16, [48] * len(cases))
    kvs = [gen.seq_kv((66, s), 48, hkv, d, BF16, 16) for s in range(len(cases))]
    for s, kv in enumerate(kvs):
        c.fill(s, kv)
    packed = np.zeros((len(cases), n), dtype=np.int32)
    for s, (p, _, _) in enumerate(cases):
        packed[s, :len(p)] = p
    lens = P.i32([0] * len(cases))
    assert gpu.kv_keep_dev(c.m, [n] * len(cases), P.i32([x for _, _, x in cases]), P.i32(packed.ravel()), P.i32([x for _, x, _ in cases]), lens) == len(cases)
    assert gpu.device_errors() == 2
    for s, (p, m, ctx) in enumerate(cases):
        want = kvs[s]["k"].copy()
        good = s in (0, 9)
        if good:
            want[12:14] = kvs[s]["k"][[12 + x for x in p]]
        assert np.array_equal(gpu.kv_read(c.m, s, 0, 48)[1], want), s
        assert int(lens[s]) == (14 if good else ctx)
    c.close()


def test_refusals(gpu):  # noqa: F811
    hq, hkv, d = 8, 2, 64
    rows = Rows(gpu, hq, hkv, d, BF16, [100, 90])
    m, n, total = rows.c.m, [3, 2], 5
    q, ctx, out = P.dev(gen.queries((55,), 70, hq, d)), P.i32([100, 90]), torch.zeros((70, hq, d), device="cuda")
    sees = M.words_of([1] * 70, 1)
    tree = lambda model=m, q=q, n=n, ctx=ctx, sees=sees, out=out, window=0, sinks=0: gpu.tree_attention_dev(model, q, n, ctx, sees, out, window, sinks)
    assert tree(model=63) == -2 and tree(q=None) == -1 and tree(out=None) == -1 and tree(window=-1) == -1 and tree(sinks=-1) == -1 and tree(n=[-1, 2]) == -1
    assert tree(window=2) == -1 and tree(window=3) == 0 and tree(n=[65, 2]) == -6 and tree(sees=sees[:4]) == -1 and tree(sees=sees.int()) == -1
    assert tree(sees=M.words_of([1] * 70, 5)) == -1 and tree(sees=sees.expand(-1, 2)) == -1 and tree(n=[1, 1, 1], ctx=P.i32([1, 1, 1])) == -6 and tree(n=[0, 0]) == 0
    out.zero_()
    (a, k, v), _ = inputs((67,), 70, hq, hkv, d)
    q_out = torch.zeros((70, hq, d), dtype=torch.int16, device="cuda")
    app = lambda model=m, n=n, ctx=ctx, sees=sees, q_out=q_out, k=k: gpu.qkv_append_tree_dev(model, a, k, v, n, ctx, sees, q_out)
    assert app(model=63) == -2 and app(q_out=None) == -1 and app(n=[65, 2]) == -6 and app(sees=sees[:4]) == -1 and app(k=k[:4]) == -1 and app(n=[-1, 1]) == -1
    assert app(n=[0, 0]) == 0 and app(n=[1, 1, 1], ctx=P.i32([1, 1, 1])) == -6
    kept, count, lens = P.i32([0] * total), P.i32([0, 0]), P.i32([0, 0])
    keep = lambda model=m, n=n, ctx=ctx, kept=kept, count=count, lens=lens: gpu.kv_keep_dev(model, n, ctx, kept, count, lens)
    assert keep(model=63) == -2 and keep(kept=kept[:4]) == -1 and keep(count=count[:1]) == -1 and keep(lens=lens[:1]) == -1 and keep(n=[-1, 2]) == -1
    assert keep(lens=ctx) == -1 and keep(lens=count) == -1 and keep(lens=kept[2:4]) == -1 and keep(n=[1, 1, 1]) == -6 and keep(n=[]) == 0
    torch.cuda.synchronize()
    assert not out.any() and not q_out.any() and not lens.any() and gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_drafted_and_verified(gpu, form, dtype, window, sinks):  # noqa: F811
    """Steps of speculative decoding as a layer goes through them: drafts appended, attended to, the accepted path kept, on and on.  In a bf16 cache the
    accepted tokens end up bit for bit as if they had been appended one by one, and their outputs are those of a decode step."""
    hq, hkv, d, batch, room = 8, 2, 128, 5, 200
    a, b = (P.Cache(gpu, hq, hkv, d, dtype, [room] * batch) for _ in range(2))
    rid = gpu.rotary_create(d, 0, P.frequencies(d))
    rng = np.random.default_rng(11)
    before = P.i32([0, 5, 1000, 77, 3])
    have = [0, 3, 16, 20, 33]
    for s, x in enumerate(have):
        if x:
            kv = gen.seq_kv((68, s), x, hkv, d, dtype, 16)
            a.fill(s, kv), b.fill(s, kv)
    for step in range(6):
        n = [int(x) for x in rng.integers(1, 14, batch)]
        masks = [M.random_tree(rng, x, 0.4) for x in n]
        paths = [M.path_of(x[int(rng.integers(0, len(x)))]) for x in masks]
        paths[step % batch] = paths[step % batch][:int(rng.integers(0, 2))]
        ctx, tokens, first = [x + y for x, y in zip(have, n)], sum(n), np.cumsum([0] + n)
        (q, k, v), _ = inputs((69, step), tokens, hq, hkv, d)
        q_out, out = torch.empty((tokens, hq, d), dtype=torch.int16, device="cuda"), torch.empty((tokens, hq, d), device="cuda")
        sees = M.words_of(sum(masks, []), 1)
        assert gpu.qkv_append_tree_dev(a.m, q, k, v, n, P.i32(ctx), sees, q_out, rotary=rid, before=before) == tokens
        assert gpu.tree_attention_dev(a.m, q_out, n, P.i32(ctx), sees, out, window, sinks) == 0
        got, rows = out.cpu().double().numpy(), [a.read(s, 0, x) for s, x in enumerate(ctx)]
        M.check(got, P.host(q_out), lambda s: rows[s], n, lambda s: M.tree_seen(ctx[s], masks[s], window, sinks))
        packed = np.zeros(tokens, dtype=np.int32)
        for s, p in enumerate(paths):
            packed[first[s]:first[s] + len(p)] = p
        lens = P.i32([0] * batch)
        assert gpu.kv_keep_dev(a.m, n, P.i32(ctx), P.i32(packed), P.i32([len(p) for p in paths]), lens) == batch
        # the same tokens one by one
        for j in range(max(len(p) for p in paths)):
            live = [s for s in range(batch) if j < len(paths[s])]
            at = [int(first[s]) + paths[s][j] for s in live]
            ql, cl = [int(s in live) for s in range(batch)], [have[s] + j + 1 for s in range(batch)]
            one, row = torch.empty((len(live), hq, d), dtype=torch.int16, device="cuda"), torch.empty((len(live), hq, d), device="cuda")
            assert gpu.qkv_append_chunk_dev(b.m, q[at], k[at], v[at], ql, P.i32(cl), one, rotary=rid, before=before) == len(live)
            assert torch.equal(one, q_out[at])
            if window:
                assert gpu.prefill_attention_window_dev(b.m, one, ql, P.i32(cl), window, sinks, row) == 0
            else:
                assert gpu.prefill_attention_dev(b.m, one, ql, P.i32(cl), row) == 0
            if dtype == BF16:
                held = [b.read(s, 0, have[s] + j + 1) for s in live]
                M.same(row, out[at], P.host(one), lambda i: held[i], [1] * len(live), lambda i: M.window_seen(have[live[i]] + j + 1, 1, window or room, sinks))
        have = [x + len(p) for x, p in zip(have, paths)]
        torch.cuda.synchronize()
        assert lens.tolist() == have
        if dtype == BF16:
            for s, x in enumerate(have):
                if x:
                    for y, z in zip(gpu.kv_read(a.m, s, 0, x)[1:3], gpu.kv_read(b.m, s, 0, x)[1:3]):
                        assert np.array_equal(y, z), (step, s)
    assert gpu.device_errors() == 0 and gpu.rotary_destroy(rid) == 0
    a.close(), b.close()


def test_captured_and_replayed(gpu):  # noqa: F811
    """A verification step as a graph: appended, attended to, kept; other trees, paths and lengths in every replay, eager calls on another cache beside it."""
    hq, hkv, d, batch, n = 8, 2, 64, 4, 9
    a, b = (P.Cache(gpu, hq, hkv, d, BF16, [400] * batch) for _ in range(2))
    for s in range(batch):
        kv = gen.seq_kv((70, s), 300, hkv, d, BF16, 16)
        a.fill(s, kv), b.fill(s, kv)
    rid, rng = gpu.rotary_create(d, 0, P.frequencies(d)), np.random.default_rng(3)
    (q, k, v), _ = inputs((71,), batch * n, hq, hkv, d)
    ctx, sees, kept, count = P.i32([n] * batch), M.words_of([0] * batch * n, 1), P.i32([0] * batch * n), P.i32([0] * batch)
    results = [[torch.zeros((batch * n, hq, d), dtype=torch.int16, device="cuda"), torch.zeros((batch * n, hq, d), device="cuda"), P.i32([0] * batch)] for _ in range(2)]

    def call(c, r):
        assert gpu.qkv_append_tree_dev(c.m, q, k, v, [n] * batch, ctx, sees, r[0], rotary=rid) == batch * n
        assert gpu.tree_attention_dev(c.m, r[0], [n] * batch, ctx, sees, r[1], 64, 2) == 0
        assert gpu.kv_keep_dev(c.m, [n] * batch, ctx, kept, count, r[2]) == batch

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        gpu.use_current_stream()
        call(a, results[0])
    gpu.use_current_stream()
    for lens in ([0, 1, 17, 100], [40, 300, 33, 16], [250, 30, 64, 5], [10, 10, 10, 10]):
        masks = [M.random_tree(rng, n, 0.5) for _ in range(batch)]
        paths = [M.path_of(x[int(rng.integers(0, n))]) for x in masks]
        ctx.copy_(P.i32([x + n for x in lens]))
        sees.copy_(M.words_of(sum(masks, []), 1))
        kept.copy_(P.i32(np.array([p + [0] * (n - len(p)) for p in paths]).ravel()))
        count.copy_(P.i32([len(p) for p in paths]))
        graph.replay()
        torch.cuda.synchronize()
        call(b, results[1])
        torch.cuda.synchronize()
        for x, y in zip(*results):
            assert torch.equal(x, y)
        for s in range(batch):
            for x, y in zip(gpu.kv_read(a.m, s, 0, 400)[1:3], gpu.kv_read(b.m, s, 0, 400)[1:3]):
                assert np.array_equal(x, y)
    assert gpu.device_errors() == 0 and gpu.rotary_destroy(rid) == 0
    del graph
    a.close(), b.close()
