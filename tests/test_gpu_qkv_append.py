"""Queries and keys normed, rotated and appended in one launch, against 64 bits; the cache bit for bit what kv_append would make of the keys.

Tolerance of an element: one rounding to bf16 (2^-8 of the result) and what fp32 loses before it: products and sums of a and b (the pair,
normed) are off by at most some ten steps of 2^-24 of |a| + |b|, sin and cos of the hardware by 2^-20 absolute: 2^-18 (|a| + |b|) covers both."""
import numpy as np
import pytest
import torch

import plain_ops as P
from workloads import gen

pytestmark = pytest.mark.gpu

BF16, E4M3 = 0, 1


@pytest.fixture(scope="module")
def gpu():
    from paper_2505_04021_amd import PrismKV
    return PrismKV()


def close(got, want, size):
    return np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size + 1e-38)


def inputs(key, rows, hq, hkv, d, pad=0, shift=0):
    """Fused rows [rows][(Hq + 2 Hkv) D + pad] from element `shift` of a buffer on, their three parts as views, and the bits of those."""
    g = gen.generator(*key)
    n = (hq + 2 * hkv) * d
    x = gen.randn_bf16((rows, n), g)
    buf = torch.zeros(rows * (n + pad) + 16, dtype=torch.int16, device="cuda")
    view = buf[shift:shift + rows * (n + pad)].view(rows, n + pad)
    view[:, :n] = P.dev(x)
    parts = [view[:, a * d:b * d].unflatten(1, (-1, d)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]
    raw = [x[:, a * d:b * d].reshape(rows, -1, d) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]
    return parts, raw


def weights(key, d):
    w = [P.bits(1.0 + 0.3 * torch.randn(d, generator=gen.generator(*key, i), dtype=torch.float64).numpy()) for i in range(2)]
    return [P.dev(x) for x in w], [P.f64(x) for x in w]


# rot, pairs, norm, pad, shift
FORMS = [(0, False, True, 0, 0), ("all", False, True, 0, 0), ("all", True, True, 24, 0), ("all", False, False, 8, 8), (16, False, True, 0, 0),
         (16, True, False, 0, 3), (20, False, True, 5, 1), (2, False, True, 0, 0), (48, False, True, 0, 0), (34, True, True, 3, 0), (0, False, False, 0, 0)]


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 2, 64), (5, 5, 128), (12, 1, 64)])
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_step_and_chunk(gpu, oracle, hq, hkv, d, form):
    rot, pairs, norm, pad, shift = form
    rot = d if rot == "all" else rot
    q_lens = np.array([1, 0, 33, 16, 7, 50], dtype=np.int32)
    start = np.array([0, 9, 5, 32, 31, 16], dtype=np.int32)
    before = np.array([0, 7, 100, 1 << 20, 12345, 2000000000], dtype=np.int32)
    freq, magnitude = P.frequencies(rot) if rot else None, 1.25
    rid = gpu.rotary_create(rot, int(pairs), freq, magnitude) if rot else -1
    lens = [int(a + b + 1) for a, b in zip(start, q_lens)]
    c = {dt: P.Cache(gpu, hq, hkv, d, dt, lens, frame_bytes=4 << 20, frames=8) for dt in (BF16, E4M3)}
    o_pool = oracle.pool_create(32 << 20, 16, 4 << 20)
    o_m = oracle.model_register(o_pool, hq, hkv, d, E4M3, len(lens), 64)
    assert oracle.balloon_resize(o_m, 8) == 8 and oracle.seq_reserve_batch(o_m, list(range(len(lens))), lens) >= 0
    for s, n in enumerate(start):
        kv = gen.seq_kv((71, s), int(n), hkv, d, E4M3, 16) if n else None
        if n:
            c[E4M3].fill(s, kv)
            assert oracle.kv_write(o_m, s, 0, kv["k"], kv["v"], kv["k_scale"], kv["v_scale"]) == n
            c[BF16].fill(s, gen.seq_kv((72, s), int(n), hkv, d, BF16, 16))
    (wq, wk), (wq64, wk64) = weights((73, d), d) if norm else ((None, None), (None, None))
    ctx = start.copy()
    for step, ql in enumerate((q_lens, None)):
        ql_ = np.ones(len(lens), dtype=np.int32) if ql is None else ql
        ctx = ctx + ql_
        rows = int(ql_.sum())
        (q, k, v), (q_b, k_b, v_b) = inputs((74, step, d), rows, hq, hkv, d, pad, shift)
        seq = np.repeat(np.arange(len(lens)), ql_)
        idx = np.concatenate([np.arange(a - n, a) for a, n in zip(ctx, ql_)])
        pos = before.astype(np.int64)[seq] + idx
        out = torch.full((rows, hq, d), -1, dtype=torch.int16, device="cuda")
        read = {}
        for dt in (BF16, E4M3):
            args = (c[dt].m, q, k, v) + (() if ql is None else (ql_,)) + (P.i32(ctx), out, wq, wk, 1e-6, rid, P.i32(before))
            assert (gpu.qkv_append_dev if ql is None else gpu.qkv_append_chunk_dev)(*args) == (len(lens) if ql is None else rows)
            torch.cuda.synchronize()
            want, size = P.turned(P.f64(q_b), pos, wq64, 1e-6, rot, pairs, freq, magnitude)
            assert close(P.f64(P.host(out)), want, size), dt
            if rot < d and not norm:
                assert np.array_equal(P.host(out)[..., rot:], q_b[..., rot:])        # elements that nothing is done to
            read[dt] = [gpu.kv_read(c[dt].m, s, 0, int(n)) for s, n in enumerate(ctx)]
        # bf16: keys near 64 bits, values as they were
        kb, vb = (np.concatenate([r[i][n - m:] for r, n, m in zip(read[BF16], ctx, ql_)]) for i in (1, 2))
        want, size = P.turned(P.f64(k_b), pos, wk64, 1e-6, rot, pairs, freq, magnitude)
        assert close(P.f64(kb), want, size) and np.array_equal(vb, v_b)
        # e4m3: codes and scales, earlier tokens' too, as the oracle's append makes them of those keys
        assert (oracle.kv_append(o_m, kb, v_b, ctx) if ql is None else oracle.kv_append_chunk(o_m, kb, v_b, ql_, ctx)) >= 0
        for s, n in enumerate(ctx):
            if n:
                for a, b in zip(read[E4M3][s][1:], oracle.kv_read(o_m, s, 0, int(n))[1:]):
                    assert np.array_equal(a, b), s
    assert gpu.device_errors() == 0
    if rot:
        assert gpu.rotary_destroy(rid) == 0
    for x in c.values():
        x.close()
    for s in range(len(lens)):
        oracle.seq_release(o_m, s)
    assert oracle.balloon_resize(o_m, 0) == 0 and oracle.model_unregister(o_m) == 0 and oracle.pool_destroy(o_pool) == 0


def test_in_place_and_one_weight(gpu):
    """Packed queries may be written over; a weight of the queries alone norms the queries alone; no `before`: rows begin at zero."""
    hq, hkv, d, n = 16, 4, 128, 37
    c = P.Cache(gpu, hq, hkv, d, BF16, [n], frames=4)
    (q, k, v), (q_b, k_b, _) = inputs((81,), n, hq, hkv, d)
    q = q.contiguous()
    (wq, _), (wq64, _) = weights((82,), d)
    f = P.frequencies(d)
    rid = gpu.rotary_create(d, 0, f)
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, [n], P.i32([n]), q, wq, None, 1e-5, rid) == n
    torch.cuda.synchronize()
    assert close(P.f64(P.host(q)), *P.turned(P.f64(q_b), np.arange(n), wq64, 1e-5, d, False, f))
    assert close(c.read(0, 0, n)[0], *P.turned(P.f64(k_b), np.arange(n), None, 0, d, False, f))
    gpu.rotary_destroy(rid)
    c.close()


def test_zero_and_huge_rows(gpu):
    """A head of zeros stays zeros (eps alone under the root), and with eps zero its norm is 0 / 0: NaN, in that head alone; heads whose
    squares pass fp32 give zeros, as the formula does in fp32; the head beside them is right."""
    hq, hkv, d = 4, 1, 64
    c = P.Cache(gpu, hq, hkv, d, BF16, [16], frames=2)
    q = torch.randn((1, hq, d), generator=gen.generator(5)).to(torch.bfloat16)
    q[0, 1] = 0.0
    q[0, 2] = 1e30
    kv = torch.randn((1, hkv, d), generator=gen.generator(6)).to(torch.bfloat16)
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    out = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda")
    for eps in (1e-6, 0.0):
        assert gpu.qkv_append_dev(c.m, q.cuda(), kv.cuda(), kv.cuda(), P.i32([1]), out, w, w, eps) == 1
        got = out.cpu().double().numpy()
        assert (got[0, 1] == 0).all() if eps else np.isnan(got[0, 1]).all()
        assert (got[0, 2] == 0).all()
        for h in (0, 3):
            assert close(got[:, h:h + 1], *P.turned(q[:, h:h + 1].double().numpy(), [0], np.ones(d), eps))
    assert gpu.device_errors() == 0
    c.close()


def test_many_sequences(gpu):
    """More sequences than one launch holds, of 0 to 3 tokens, 64-wide heads."""
    hq, hkv, d, n = 4, 1, 64, 900
    rng = np.random.default_rng(4)
    ql = rng.integers(0, 4, n).astype(np.int32)
    ql[:3] = ql[-3:] = 0
    c = P.Cache(gpu, hq, hkv, d, BF16, [16] * n, frames=8)
    rows = int(ql.sum())
    (q, k, v), (q_b, k_b, v_b) = inputs((91,), rows, hq, hkv, d)
    out = torch.empty((rows, hq, d), dtype=torch.int16, device="cuda")
    before = rng.integers(0, 1 << 30, n).astype(np.int32)
    f = P.frequencies(d)
    rid = gpu.rotary_create(d, 1, f)
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, ql, P.i32(ql), out, None, None, 0.0, rid, P.i32(before)) == rows
    seq = np.repeat(np.arange(n), ql)
    pos = before.astype(np.int64)[seq] + np.concatenate([np.arange(x) for x in ql])
    torch.cuda.synchronize()
    assert close(P.f64(P.host(out)), *P.turned(P.f64(q_b), pos, None, 0, d, True, f))
    for s in (3, 100, 446, 447, 448, 449, 450, 451, 700, n - 4):
        at = int(ql[:s].sum())
        if ql[s]:
            k64, v64 = c.read(s, 0, int(ql[s]))
            sel = slice(at, at + int(ql[s]))
            assert close(k64, *P.turned(P.f64(k_b[sel]), pos[sel], None, 0, d, True, f)) and np.array_equal(v64, P.f64(v_b[sel]))
    assert gpu.device_errors() == 0
    gpu.rotary_destroy(rid)
    c.close()


def test_refused_context_and_other_rows(gpu):
    """A context length outside the row's blocks raises bit 1 and writes nothing of that row; queries come all the same."""
    hq, hkv, d = 8, 2, 64
    c = P.Cache(gpu, hq, hkv, d, BF16, [20, 20, 20], frames=2, poison=0x11)
    before = [gpu.kv_read(c.m, s, 0, 20) for s in range(3)]
    (q, k, v), (q_b, _, v_b) = inputs((95,), 3, hq, hkv, d)
    out = torch.zeros((3, hq, d), dtype=torch.int16, device="cuda")
    assert gpu.qkv_append_dev(c.m, q, k, v, P.i32([0, 7, 33]), out) == 3
    assert gpu.device_errors() == 2 and np.array_equal(P.host(out), q_b)
    for s in (0, 2):
        after = gpu.kv_read(c.m, s, 0, 20)
        assert np.array_equal(after[1], before[s][1]) and np.array_equal(after[2], before[s][2])
    got = gpu.kv_read(c.m, 1, 0, 20)[2]
    assert np.array_equal(got[6], v_b[1]) and np.array_equal(np.delete(got, 6, 0), np.delete(before[1][2], 6, 0))
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, [3, 0, 0], P.i32([2, 9, 9]), out) == 3 and gpu.device_errors() == 2
    c.close()


def test_refusals(gpu):
    hq, hkv, d = 8, 2, 64
    c = P.Cache(gpu, hq, hkv, d, BF16, [16, 16], frames=2)
    (q, k, v), _ = inputs((96,), 2, hq, hkv, d)
    out = torch.zeros((2, hq, d), dtype=torch.int16, device="cuda")
    one = P.i32([1, 1])
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    ok = dict(q_weight=w, k_weight=w)
    assert gpu.qkv_append_dev(c.m, q, k, v, P.i32([1, 1, 1]), out) == -6                       # more rows than the model has
    assert gpu.qkv_append_dev(c.m, q, k, v, one, None) == -1
    assert gpu.qkv_append_dev(c.m, q, k, v, one, out.view(-1)[1:], **ok) == -1    # q_out not on 16 bytes
    odd = torch.ones(d + 8, dtype=torch.bfloat16, device="cuda")[1:1 + d]
    assert gpu.qkv_append_dev(c.m, q, k, v, one, out, q_weight=odd) == -1 and gpu.qkv_append_dev(c.m, q, k, v, one, out, k_weight=odd) == -1
    assert gpu.qkv_append_dev(c.m, q, k, v, one, out, eps=-1.0, **ok) == -1
    assert gpu.qkv_append_dev(c.m, q, k, v, one, out, eps=float("nan"), **ok) == -1
    assert gpu.qkv_append_dev(c.m, q, k, v, one, out, rotary=5) == -2 and gpu.qkv_append_dev(c.m, q, k, v, one, out, rotary=-2) == -2
    wide = gpu.rotary_create(128, 0, P.frequencies(128))
    assert wide >= 0 and gpu.qkv_append_dev(c.m, q, k, v, one, out, rotary=wide) == -5
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, [2, -1], one, out) == -1
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, [1 << 24, 1], one, out) == -6
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, [0, 0], one, out) == 0
    assert gpu.qkv_append_dev(c.m, q[:0], k[:0], v[:0], one[:0], out) == 0
    assert gpu.rotary_destroy(wide) == 0 and gpu.rotary_destroy(wide) == -2
    ids = [gpu.rotary_create(2, 0, [1.0]) for _ in range(65)]
    assert ids == list(range(64)) + [-3]
    assert all(gpu.rotary_destroy(i) == 0 for i in ids[:64])
    assert gpu.device_errors() == 0
    c.close()


def test_captured_and_replayed(gpu):
    """A step captured into a graph follows the context lengths on the device, replay after replay, beside eager work."""
    hq, hkv, d = 16, 4, 64
    c = P.Cache(gpu, hq, hkv, d, E4M3, [64, 64], frames=4)
    e = P.Cache(gpu, hq, hkv, d, E4M3, [64, 64], frames=4)
    rid = gpu.rotary_create(64, 0, P.frequencies(64))
    (q, k, v), _ = inputs((97,), 2, hq, hkv, d)
    ctx, out, out2 = P.i32([0, 5]), torch.zeros((2, hq, d), dtype=torch.int16, device="cuda"), torch.zeros((2, hq, d), dtype=torch.int16, device="cuda")
    for x in (c, e):
        x.fill(1, gen.seq_kv((98, 1), 5, hkv, d, E4M3, 16))
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        gpu.use_current_stream()
        assert gpu.qkv_append_dev(c.m, q, k, v, ctx, out, rotary=rid) == 2
    gpu.use_current_stream()
    for step in range(5):
        ctx += 1
        q.mul_(1).add_(step)                              # other bits every time
        k.add_(3 * step)
        graph.replay()
        torch.cuda.synchronize()
        assert gpu.qkv_append_dev(e.m, q, k, v, ctx, out2, rotary=rid) == 2
        torch.cuda.synchronize()
        assert torch.equal(out, out2)
        for s in range(2):
            for a, b in zip(gpu.kv_read(c.m, s, 0, int(ctx[s])), gpu.kv_read(e.m, s, 0, int(ctx[s]))):
                assert np.array_equal(a, b)
    assert gpu.device_errors() == 0
    del graph
    gpu.rotary_destroy(rid)
    c.close()
    e.close()
