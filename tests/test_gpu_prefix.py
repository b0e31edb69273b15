"""Attention behind shared prefixes, decode steps and prefill chunks, against 64 bits (tolerances: plain_ops.attention), and the way such
sequences go through the library: filled, forked, appended to and attended to together."""
import numpy as np
import pytest
import torch

import plain_ops as P
from workloads import gen

pytestmark = pytest.mark.gpu

BF16, E4M3 = 0, 1
SHAPES = [(32, 8, 128, BF16), (8, 2, 64, BF16), (16, 1, 128, BF16), (3, 3, 64, BF16), (10, 2, 128, BF16), (32, 8, 128, E4M3), (12, 4, 64, E4M3), (5, 1, 64, E4M3)]


@pytest.fixture(scope="module")
def gpu():
    from paper_2505_04021_amd import PrismKV
    return PrismKV()


@pytest.fixture(params=[0, 1], ids=["once for all", "whole contexts"])
def form(gpu, request):
    """Both ways of walking the prefixes of a decode step."""
    assert gpu.set_prefix_form(request.param) == 0
    yield request.param
    gpu.set_prefix_form(-1)


def values(kv, dtype):
    """K and V of gen.seq_kv as float64."""
    if dtype == BF16:
        return P.f64(kv["k"]), P.f64(kv["v"])
    of = lambda c, s: torch.from_numpy(c).view(torch.float8_e4m3fn).double().numpy() * np.repeat(s.astype(np.float64), 16, axis=0)[:len(c), :, None]
    return of(kv["k"], kv["k_scale"]), of(kv["v"], kv["v_scale"])


class Rows:
    """A Cache whose rows are filled, with their values at hand."""

    def __init__(self, gpu, hq, hkv, d, dtype, lens, key=7, **kw):
        self.c = P.Cache(gpu, hq, hkv, d, dtype, lens, **kw)
        self.kv = []
        for s, n in enumerate(lens):
            kv = gen.seq_kv((key, s), max(n, 1), hkv, d, dtype, 16, peak_frac=0.02)
            self.c.fill(s, kv, n)
            self.kv.append([x[:n] for x in values(kv, dtype)])

    def context(self, prefix, blocks, row, n):
        parts = ([[x[:16 * blocks] for x in self.kv[prefix]]] if prefix >= 0 and blocks else []) + [[x[:n] for x in self.kv[row]]]
        return [np.concatenate(x) for x in zip(*parts)]


def check_decode(gpu, rows, q, prefix, blocks, ctx):
    c = rows.c
    out = torch.full((len(ctx), c.hq, c.d), float("nan"), device="cuda")
    assert gpu.decode_attention_prefix_dev(c.m, P.dev(q), prefix, blocks, P.i32(ctx), out) == 0
    got = out.cpu().double().numpy()
    for s, n in enumerate(ctx):
        k, v = rows.context(prefix[s], blocks[s], s, n)
        want, tol = P.attention(P.f64(q[s:s + 1]), k, v, [len(k)])
        err = np.abs(got[s:s + 1] - want)
        assert np.all(err <= tol + 1e-30), (s, n, prefix[s], blocks[s], float((err / np.maximum(tol, 1e-30)).max()))


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_decode(gpu, form, hq, hkv, d, dtype):
    """Groups of 1 to many members in no order, prefixes of one block to many and odd numbers, rows with and without a prefix, without tokens
    of their own, without either; the same row shared to different depths; a row of the batch that is itself a prefix."""
    n = 45
    own = [0, 1, 17, 33, 100, 16, 250, 5] + [int(x) for x in gen.ctx_lognormal(n - 8, 40, 1.0, 400, gen.generator(2, hq))]
    own[20] = 64                                                          # row 20 is shared by others
    prefix_tokens = [16, 48, 16 * 17, 16 * 70 + 9]
    rows = Rows(gpu, hq, hkv, d, dtype, own + prefix_tokens, frames=100)
    rng = np.random.default_rng(hq)
    choice = [(-1, 0), (n, 1), (n + 1, 3), (n + 1, 2), (n + 2, 17), (n + 3, 70), (n + 3, 70), (n + 3, 70), (20, 4), (n + 2, 0)]
    picks = [choice[i] for i in rng.integers(0, len(choice), n)]
    picks[0], picks[1], picks[20] = (-1, 0), (n + 3, 70), (-1, 0)
    q = gen.queries((3, d, hq), n, hq, d)
    check_decode(gpu, rows, q, [p for p, _ in picks], [b for _, b in picks], own)
    # a shared row without tokens of its own in most of the batch, one group, and shorter contexts than the rows hold
    check_decode(gpu, rows, q, [n + 3] * n, [70] * n, [0 if i % 3 else x // 2 for i, x in enumerate(own)])
    # few sequences
    check_decode(gpu, rows, q[:1], [n + 2], [16], own[:1])
    check_decode(gpu, rows, q[:3], [-1, n + 2, -1], [5, 17, 0], own[:3])
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, BF16), (6, 2, 64, E4M3), (5, 5, 64, BF16), (16, 1, 128, E4M3)])
def test_decode_narrow_groups(gpu, form, hq, hkv, d, dtype):
    """Groups of few columns (members x heads of a kv head: up to 16, one more, many), whose prefixes are walked by four waves on different
    pages, between groups whose prefixes are not and sequences without one; prefixes of one block, of odd numbers and of many parts."""
    g = hq // hkv
    sizes = [1, 16 // g, 16 // g + 1, 2, 40, 1]
    shared = [16, 16 * 7, 16 * 90, 16 * 300, 16 * 33, 16 * 131]
    group = [j for j, n in enumerate(sizes) for _ in range(n)] + [-1] * 3
    group = [group[i] for i in np.random.default_rng(g).permutation(len(group))]
    n = len(group)
    own = [int(x) for x in gen.ctx_lognormal(n, 30, 1.2, 300, gen.generator(23, hq))]
    own[0] = 0
    rows = Rows(gpu, hq, hkv, d, dtype, own + shared, frames=100)
    check_decode(gpu, rows, gen.queries((24, d), n, hq, d), [n + x if x >= 0 else -1 for x in group], [shared[x] // 16 if x >= 0 else 0 for x in group], own)
    assert gpu.last_prefix_form() == form and gpu.device_errors() == 0
    rows.c.close()


def test_decode_many_groups_and_members(gpu):
    """More groups, and more members of one, than a launch's plan holds."""
    hq, hkv, d, n = 4, 1, 64, 1300
    rng = np.random.default_rng(8)
    own = [int(x) for x in rng.integers(0, 20, n)]
    shared = [16 * int(x) for x in rng.integers(1, 5, 150)]
    rows = Rows(gpu, hq, hkv, d, BF16, own + shared, frames=40)
    prefix = [n + int(x) if x < 150 else n + 7 for x in rng.integers(0, 300, n)]
    blocks = [shared[p - n] // 16 for p in prefix]
    assert len(set(prefix)) > 64 and prefix.count(n + 7) > 512
    check_decode(gpu, rows, gen.queries((5,), n, hq, d), prefix, blocks, own)
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(16, 2, 128, BF16), (8, 8, 64, E4M3)])
def test_decode_long_rows(gpu, form, hq, hkv, d, dtype):
    """Long prefixes and long rows, both in many parts; one long row among short ones."""
    own = [5000, 3, 700, 2900]
    rows = Rows(gpu, hq, hkv, d, dtype, own + [16 * 401], frames=100)
    q = gen.queries((6, d), 4, hq, d)
    check_decode(gpu, rows, q, [4, 4, -1, 4], [401, 401, 0, 400], own)
    check_decode(gpu, rows, q, [4, 4, 4, 4], [401] * 4, [1, 0, 0, 2])
    assert gpu.device_errors() == 0
    rows.c.close()


def test_infinite_logits(gpu, form):
    """Keys of -inf against positive queries weigh nothing, wherever they stand: all of a prefix, all of a row, or both (then the row is zero)."""
    hq, hkv, d = 4, 2, 64
    c = P.Cache(gpu, hq, hkv, d, BF16, [40, 40, 40, 64, 64], frames=4)
    kv = [gen.seq_kv((9, s), 64, hkv, d, BF16, 16) for s in range(5)]
    for s in (1, 2, 4):                                                   # rows 1 and 2 and the prefix in row 4
        kv[s]["k"] = np.full_like(kv[s]["k"], 0xFF80)
    for s, n in enumerate(c.lens):
        c.fill(s, kv[s], n)
    q = np.full((3, hq, d), 0x3F80, dtype=np.uint16)
    out = torch.full((3, hq, d), float("nan"), device="cuda")
    assert gpu.decode_attention_prefix_dev(c.m, P.dev(q), [4, 3, 4], [4, 4, 4], P.i32([40, 40, 40]), out) == 0
    got = out.cpu().double().numpy()
    for s, (row, n) in enumerate(((0, 40), (3, 64))):
        want, tol = P.attention(P.f64(q[s:s + 1]), P.f64(kv[row]["k"][:n]), P.f64(kv[row]["v"][:n]), [n])
        assert np.all(np.abs(got[s:s + 1] - want) <= tol)
    assert (got[2] == 0).all()
    c.close()


@pytest.mark.parametrize("hkv,blocks", [(1, 100), (8, 200)])
def test_infinite_logits_over_many_parts(gpu, form, hkv, blocks):
    """The same where contexts come in several parts: nothing but -inf gives zero rows, one row with finite keys behind them is right."""
    d, n = 64, 12
    own = [700] * n
    c = P.Cache(gpu, 2 * hkv, hkv, d, BF16, own + [16 * blocks], frames=100)
    kv = gen.seq_kv((10,), 16 * blocks, hkv, d, BF16, 16)
    far = dict(kv, k=np.full_like(kv["k"], 0xFF80))
    for s, x in enumerate(own + [16 * blocks]):
        c.fill(s, kv if s == 3 else far, x)
    q = np.full((n, 2 * hkv, d), 0x3F80, dtype=np.uint16)
    out = torch.full((n, 2 * hkv, d), float("nan"), device="cuda")
    assert gpu.decode_attention_prefix_dev(c.m, P.dev(q), [n] * n, [blocks] * n, P.i32(own), out) == 0
    got = out.cpu().double().numpy()
    want, tol = P.attention(P.f64(q[3:4]), P.f64(kv["k"][:700]), P.f64(kv["v"][:700]), [700])
    assert np.all(np.abs(got[3:4] - want) <= tol) and (np.delete(got, 3, 0) == 0).all()
    c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_prefill(gpu, hq, hkv, d, dtype):
    """Chunks of 0, 1 and many tokens, behind tokens of their own or none, behind prefixes or none."""
    new = [5, 0, 1, 64, 130, 33, 16, 200, 7]
    old = [0, 30, 15, 0, 40, 16, 1, 100, 0]
    have = [a + b for a, b in zip(new, old)]
    n = len(new)
    rows = Rows(gpu, hq, hkv, d, dtype, have + [16, 16 * 33 + 3, 16 * 64], frames=100)
    prefix, blocks = [n, n, n + 1, n + 1, n + 1, -1, n + 2, n + 2, 4], [1, 1, 33, 2, 33, 0, 64, 63, 10]
    q = gen.queries((11, d, hq), sum(new), hq, d)
    out = torch.full((sum(new), hq, d), float("nan"), device="cuda")
    assert gpu.prefill_attention_prefix_dev(rows.c.m, P.dev(q), new, prefix, blocks, P.i32(have), out) == 0
    got = out.cpu().double().numpy()
    at = 0
    for s in range(n):
        k, v = rows.context(prefix[s], blocks[s], s, have[s])
        want, tol = P.attention(P.f64(q[at:at + new[s]]), k, v, [len(k) - new[s] + 1 + i for i in range(new[s])])
        err = np.abs(got[at:at + new[s]] - want)
        assert np.all(err <= tol), (s, float((err / tol).max()))
        at += new[s]
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(32, 8, 128, BF16), (16, 2, 64, E4M3)])
def test_prefill_few_queries_behind_a_long_prefix(gpu, hq, hkv, d, dtype):
    """Contexts are cut into parts: some lie in the prefix, some in the row, some in both."""
    new, old = [3, 20, 1], [0, 500, 15]
    have = [a + b for a, b in zip(new, old)]
    rows = Rows(gpu, hq, hkv, d, dtype, have + [16 * 151], frames=60)
    q = gen.queries((12, d), sum(new), hq, d)
    out = torch.full((sum(new), hq, d), float("nan"), device="cuda")
    assert gpu.prefill_attention_prefix_dev(rows.c.m, P.dev(q), new, [3, 3, 3], [151, 150, 151], P.i32(have), out) == 0
    assert gpu.last_prefill_parts() > 1
    got, at = out.cpu().double().numpy(), 0
    for s, b in enumerate((151, 150, 151)):
        k, v = rows.context(3, b, s, have[s])
        want, tol = P.attention(P.f64(q[at:at + new[s]]), k, v, [len(k) - new[s] + 1 + i for i in range(new[s])])
        assert np.all(np.abs(got[at:at + new[s]] - want) <= tol), s
        at += new[s]
    assert gpu.device_errors() == 0
    rows.c.close()


@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, E4M3)])
def test_prefill_of_queries_before_their_row(gpu, d, dtype):
    """Context lengths below the chunk's: queries that would stand before their row's first token see the prefix alone."""
    hq, hkv = 8, 2
    have, new, ctx = [100, 60, 40, 10], [90, 60, 40, 10], [70, 13, 0, -5]
    rows = Rows(gpu, hq, hkv, d, dtype, have + [16 * 20], frames=20)
    q = gen.queries((25, d), sum(new), hq, d)
    for blocks in (20, 1, 0):
        out = torch.full((sum(new), hq, d), float("nan"), device="cuda")
        assert gpu.prefill_attention_prefix_dev(rows.c.m, P.dev(q), new, [4] * 4, [blocks] * 4, P.i32(ctx), out) == 0
        got, at = out.cpu().double().numpy(), 0
        for s in range(4):
            k, v = rows.context(4, blocks, s, max(ctx[s], 0))
            own = [ctx[s] - new[s] + 1 + i for i in range(new[s])]
            want, tol = P.attention(P.f64(q[at:at + new[s]]), k, v, [16 * blocks + max(x, 0) for x in own])
            assert np.all(np.abs(got[at:at + new[s]] - want) <= tol), (blocks, s)
            at += new[s]
    assert gpu.device_errors() == 0
    rows.c.close()


def test_prefill_of_many_sequences(gpu):
    """More sequences than a launch of this kind holds."""
    hq, hkv, d, n = 4, 1, 64, 300
    rng = np.random.default_rng(13)
    new = [int(x) for x in rng.integers(0, 6, n)]
    old = [int(x) for x in rng.integers(0, 20, n)]
    have = [a + b for a, b in zip(new, old)]
    rows = Rows(gpu, hq, hkv, d, BF16, have + [48, 160], frames=20)
    pick = rng.integers(0, 3, n)
    prefix, blocks = [[-1, n, n + 1][i] for i in pick], [[0, 3, 9][i] for i in pick]
    q = gen.queries((14,), sum(new), hq, d)
    out = torch.full((sum(new), hq, d), float("nan"), device="cuda")
    assert gpu.prefill_attention_prefix_dev(rows.c.m, P.dev(q), new, prefix, blocks, P.i32(have), out) == 0
    got, at = out.cpu().double().numpy(), 0
    for s in range(n):
        k, v = rows.context(prefix[s], blocks[s], s, have[s])
        want, tol = P.attention(P.f64(q[at:at + new[s]]), k, v, [len(k) - new[s] + 1 + i for i in range(new[s])])
        assert np.all(np.abs(got[at:at + new[s]] - want) <= tol), s
        at += new[s]
    rows.c.close()


def test_refusals(gpu):
    rows = Rows(gpu, 8, 2, 64, BF16, [20, 20, 40], frames=4)
    c = rows.c
    q, out = P.dev(gen.queries((15,), 2, 8, 64)), torch.zeros((2, 8, 64), device="cuda")
    ctx = P.i32([20, 20])
    dec = lambda p, b, m=c.m, q=q, o=out, x=ctx: gpu.decode_attention_prefix_dev(m, q, p, b, x, o)
    pre = lambda p, b, m=c.m, q=q, o=out, x=ctx, ql=(1, 1): gpu.prefill_attention_prefix_dev(m, q, ql, p, b, x, o)
    for f in (dec, pre):
        assert f([2, 2], [2, 2], m=55) == -2
        assert f([3, 2], [1, 1]) == -1 and f([-2, 2], [1, 1]) == -1 and f([2, 2], [-1, 1]) == -1
        assert f([2, 2], [4, 1]) == -6 and f([2, 2], [2 ** 30, 1]) == -6 and f([0, 2], [3, 1]) == -6
        assert f([2, 2], [2, 2], q=q.view(-1)[1:]) == -1 and f([2, 2], [2, 2], o=out.view(-1)[1:]) == -1
        assert f([2, 2], [2, 2], o=None) == -1
        assert f([-1, -1], [99, 0]) == 0                                  # no prefix: its blocks are not looked at
    assert gpu.set_prefix_form(2) == -1 and gpu.set_prefix_form(-2) == -1
    four = P.i32([1, 1, 1, 1])
    assert gpu.decode_attention_prefix_dev(c.m, q, [2] * 4, [1] * 4, four, out) == -6
    assert pre([2, 2], [2, 2], ql=(1, -1)) == -1 and pre([2, 2], [2, 2], ql=(1 << 24, 1)) == -6 and pre([2, 2], [2, 2], ql=(0, 0)) == 0
    assert gpu.decode_attention_prefix_dev(c.m, q, [], [], ctx[:0], out) == 0
    lib = gpu.lib
    assert lib.decode_attention_prefix(c.m, 2, q.data_ptr(), None, None, ctx.data_ptr(), out.data_ptr()) == -1
    assert gpu.device_errors() == 0
    c.close()


def test_prefix_that_is_not_there(gpu):
    """A reservation that was enqueued and refused: the host believes the prefix's row to be long, the device knows it is empty.  The
    sequences that would share it get zero rows and bit 0 is raised; the others are right."""
    pool = gpu.pool_create(1 << 20, 16, 1 << 20)
    m = gpu.model_register(pool, 8, 2, 64, BF16, 3, 1000)                 # one frame: 128 blocks of 8 KiB
    assert gpu.balloon_resize(m, 1) == 1 and gpu.seq_reserve_batch(m, [0, 1], [20, 20]) == 4
    kv = gen.seq_kv((16,), 20, 2, 64, BF16, 16)
    for s in range(2):
        assert gpu.kv_write(m, s, 0, kv["k"], kv["v"]) == 20
    ticket = gpu.seq_reserve_batch_enqueue(m, [2], [16 * 500])
    assert ticket >= 0
    q = gen.queries((17,), 2, 8, 64)
    for prefill, how in ((False, 0), (False, 1), (True, -1)):
        out = torch.full((2, 8, 64), float("nan"), device="cuda")
        assert gpu.set_prefix_form(how) == 0
        if prefill:
            rc = gpu.prefill_attention_prefix_dev(m, P.dev(q), [1, 1], [2, -1], [400, 0], P.i32([20, 20]), out)
        else:
            rc = gpu.decode_attention_prefix_dev(m, P.dev(q), [2, -1], [400, 0], P.i32([20, 20]), out)
        assert rc == 0
        got = out.cpu().double().numpy()
        want, tol = P.attention(P.f64(q[1:]), P.f64(kv["k"]), P.f64(kv["v"]), [20])
        assert (got[0] == 0).all() and np.all(np.abs(got[1:] - want) <= tol)
    gpu.set_prefix_form(-1)
    assert gpu.device_errors() == 5 and gpu.ticket_result(ticket) == -4
    assert gpu.decode_attention_prefix_dev(m, P.dev(q), [2, -1], [400, 0], P.i32([20, 20]), out) == -6      # now the host knows
    for s in range(3):
        gpu.seq_release(m, s)
    assert gpu.balloon_resize(m, 0) == 0 and gpu.model_unregister(m) == 0 and gpu.pool_destroy(pool) == 0


def test_captured_and_replayed(gpu):
    """Both calls in a graph: refused while there is no workspace, then captured; replays follow contexts and queries on the device, also
    after a larger eager call has made a larger workspace."""
    hq, hkv, d = 16, 2, 64
    rows = Rows(gpu, hq, hkv, d, BF16, [300, 400, 300, 16 * 40, 16 * 200], frames=40)
    c = rows.c
    q = P.dev(gen.queries((18,), 3, hq, d))
    ctx = P.i32([250, 40, 1])
    a = dict(prefix=[3, 3, -1], blocks=[40, 40, 0])
    out, out2, eager = (torch.zeros((3, hq, d), device="cuda") for _ in range(3))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()

    def calls(o, o2):
        r = gpu.decode_attention_prefix_dev(c.m, q, a["prefix"], a["blocks"], ctx, o)
        return r, gpu.prefill_attention_prefix_dev(c.m, q, [1, 1, 1], a["prefix"], a["blocks"], ctx, o2)

    torch.cuda.synchronize()
    refused = torch.cuda.CUDAGraph()
    with torch.cuda.graph(refused, stream=stream):
        gpu.use_current_stream()
        assert calls(out, out2)[1] == -3 and "capture" in gpu.last_error()         # (a small decode step needs none)
    gpu.use_current_stream()
    assert calls(out, out2) == (0, 0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        gpu.use_current_stream()
        assert calls(out, out2) == (0, 0)
    gpu.use_current_stream()
    for step in range(5):
        ctx += torch.tensor([-50, 60, 37], dtype=torch.int32, device="cuda")
        q.copy_(P.dev(gen.queries((19, step), 3, hq, d)))
        graph.replay()
        torch.cuda.synchronize()
        for got in (out, out2):
            for s in range(3):
                n = int(ctx[s])
                k, v = rows.context(a["prefix"][s], a["blocks"][s], s, n)
                want, tol = P.attention(P.f64(P.host(q)[s:s + 1]), k, v, [len(k)])
                assert np.all(np.abs(got[s:s + 1].cpu().double().numpy() - want) <= tol), (step, s)
        out.zero_()
        out2.zero_()
        if step == 2:
            big = P.dev(gen.queries((20,), 3, hq, d))
            assert gpu.decode_attention_prefix_dev(c.m, big, [4, 3, 4], [200, 40, 199], P.i32([300, 300, 300]), eager) == 0
    assert gpu.device_errors() == 0
    del graph, refused
    c.close()


def test_large_step_captured_and_replayed(gpu):
    """The same for a decode step whose prefix is walked for all at once: refused without a workspace, then captured; a larger eager call in
    between makes a larger workspace, and the graph goes on with its own."""
    hq, hkv, d, n = 16, 2, 64, 60
    rows = Rows(gpu, hq, hkv, d, BF16, [300] * n + [16 * 400, 16 * 420], frames=60)
    c = rows.c
    q, ctx = P.dev(gen.queries((21,), n, hq, d)), P.i32([200] * n)
    prefix, blocks = [n] * (n - 1) + [-1], [400] * n
    out, eager = (torch.zeros((n, hq, d), device="cuda") for _ in range(2))
    call = lambda o, p=prefix, b=blocks: gpu.decode_attention_prefix_dev(c.m, q, p, b, ctx, o)
    stream, graph, refused = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
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
    for step in range(4):
        ctx += torch.arange(n, dtype=torch.int32, device="cuda") % 7 * 3
        q.copy_(P.dev(gen.queries((22, step), n, hq, d)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().double().numpy()
        for s in (0, 5, n - 2, n - 1):
            k, v = rows.context(prefix[s], blocks[s], s, int(ctx[s]))
            want, tol = P.attention(P.f64(P.host(q)[s:s + 1]), k, v, [len(k)])
            assert np.all(np.abs(got[s:s + 1] - want) <= tol), (step, s)
        out.zero_()
        if step == 1:                                                     # two groups of many parts
            assert call(eager, [n, n + 1] * (n // 2), [400, 420] * (n // 2)) == 0
    assert gpu.device_errors() == 0
    del graph, refused
    c.close()


@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_from_system_prompt_to_answers(gpu, dtype):
    """A system prompt is prefilled once; prompts of ragged length are prefilled behind its whole blocks, the tokens behind those copied into
    every row; then decode steps.  Everything goes through the calls as an engine makes them (projections, qkv_append, attention) and is compared with
    every sequence computed alone in 64 bits on what the cache holds."""
    hq, hkv, d, eps = 8, 2, 128, 1e-6
    prompt, prompts, steps = 16 * 9 + 5, [3, 40, 17, 1], 3
    whole, rest, n = prompt // 16, prompt % 16, len(prompts)
    c = P.Cache(gpu, hq, hkv, d, dtype, [rest + x + steps for x in prompts] + [prompt], frames=8)
    f = P.frequencies(d)
    rid = gpu.rotary_create(d, 0, f)
    w = torch.from_numpy(gen.to_bf16_bits(1 + 0.2 * torch.randn(d, generator=gen.generator(40))).view(np.int16)).cuda()
    w64 = P.f64(P.host(w))

    def project(key, rows):
        x = P.dev(gen.randn_bf16((rows, (hq + 2 * hkv) * d), gen.generator(41, key))).view(rows, -1, d)
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], torch.empty((rows, hq, d), dtype=torch.int16, device="cuda")

    # the system prompt in row n, as a chunk of its own
    q, k, v, qo = project(0, prompt)
    lens = [0] * n + [prompt]
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, lens, P.i32(lens), qo, w, w, eps, rid) == prompt
    out = torch.empty((prompt, hq, d), device="cuda")
    assert gpu.prefill_attention_dev(c.m, qo, np.array(lens, dtype=np.int32), P.i32(lens), out) == 0
    # its tokens behind the last whole block go into every row.  (Keys are rotated already.)
    kt, vt = (torch.empty((n * rest, hkv, d), dtype=torch.int16, device="cuda") for _ in range(2))
    assert gpu.kv_gather_dev(c.m, [n] * n, [16 * whole] * n, [rest] * n, kt, vt) == n * rest
    ctx = np.full(n, rest, dtype=np.int32)
    assert gpu.kv_append_chunk_dev(c.m, kt, vt, ctx, P.i32(ctx)) == n * rest
    before, prefix, blocks = P.i32([16 * whole] * n), [n] * n, [whole] * n

    def compare(qo, out, new):
        got, qs, at = out.cpu().double().numpy(), P.f64(P.host(qo)), 0
        shared = c.read(n, 0, 16 * whole)
        for s in range(n):
            mine = c.read(s, 0, int(ctx[s]))
            kk, vv = (np.concatenate(x) for x in zip(shared, mine))
            want, tol = P.attention(qs[at:at + new[s]], kk, vv, [len(kk) - new[s] + 1 + i for i in range(new[s])])
            assert np.all(np.abs(got[at:at + new[s]] - want) <= tol), s
            at += new[s]

    ctx = ctx + np.array(prompts, dtype=np.int32)
    q, k, v, qo = project(1, sum(prompts))
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, prompts, P.i32(ctx), qo, w, w, eps, rid, before) == sum(prompts)
    out = torch.empty((sum(prompts), hq, d), device="cuda")
    assert gpu.prefill_attention_prefix_dev(c.m, qo, prompts, prefix, blocks, P.i32(ctx), out) == 0
    compare(qo, out, prompts)
    # the last prompt's first query stands behind the system prompt
    pos = np.concatenate([prompt + np.arange(x) for x in prompts])
    want, size = P.turned(P.f64(P.host(q.contiguous())), pos, w64, eps, d, False, f)
    assert np.all(np.abs(P.f64(P.host(qo)) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * size)
    for step in range(steps):
        ctx = ctx + 1
        q, k, v, qo = project(2 + step, n)
        cd = P.i32(ctx)
        assert gpu.qkv_append_dev(c.m, q, k, v, cd, qo, w, w, eps, rid, before) == n
        out = torch.empty((n, hq, d), device="cuda")
        assert gpu.decode_attention_prefix_dev(c.m, qo, prefix, blocks, cd, out) == 0
        compare(qo, out, [1] * n)
    assert gpu.device_errors() == 0
    gpu.rotary_destroy(rid)
    c.close()


def test_layers_of_two_models_on_two_streams(gpu):
    """Models of several layers in elastic pools, each on a stream of its own, their calls in turn: a prefix and prompts behind it appended and
    attended to, then a decode step, layer by layer; all of it looked at when everything has been enqueued.  (Prompts end with a block: appended behind
    them, a decode step's token rescales no codes that the prompts' queries saw.)"""
    models = [(8, 2, 128, BF16, 3), (12, 4, 64, E4M3, 2)]
    new, prefix, blocks = [32, 64, 16, 16 * 12], [3, 3, -1, -1], [12, 7, 0, 0]
    n, todo = sum(new[:3]), []
    caches = [P.Cache(gpu, hq, hkv, d, t, [x + 1 for x in new], frames=4, n_layers=layers, elastic=True) for hq, hkv, d, t, layers in models]
    streams = [torch.cuda.Stream() for _ in models]
    rids = [gpu.rotary_create(m[2], i, P.frequencies(m[2])) for i, m in enumerate(models)]
    before, lens, now, dec = P.i32([16 * b for b in blocks]), P.i32(new), P.i32(new[:3]), P.i32([x + 1 for x in new[:3]])
    data = {}
    for i, (hq, hkv, d, _, layers) in enumerate(models):
        for layer in range(layers):
            for key, rows in ((0, sum(new)), (1, 3)):
                x = P.dev(gen.randn_bf16((rows, (hq + 2 * hkv) * d), gen.generator(50, i, layer, key))).view(rows, -1, d)
                data[i, layer, key] = (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], torch.empty((rows, hq, d), dtype=torch.int16, device="cuda"))
            data[i, layer, 2] = [torch.full((rows, hq, d), float("nan"), device="cuda") for rows in (n, 3)]
    torch.cuda.synchronize()
    for layer in range(3):
        for i, (c, m) in enumerate(zip(caches, models)):
            if layer >= m[4]:
                continue
            with torch.cuda.stream(streams[i]):
                gpu.use_current_stream()
                assert gpu.set_layer(c.m, layer) == 0
                (q, k, v, qo), (q1, k1, v1, qo1), out = (data[i, layer, key] for key in range(3))
                assert gpu.qkv_append_chunk_dev(c.m, q, k, v, new, lens, qo, None, None, 0.0, rids[i], before) == sum(new)
                assert gpu.prefill_attention_prefix_dev(c.m, qo, new[:3], prefix[:3], blocks[:3], now, out[0]) == 0
                assert gpu.qkv_append_dev(c.m, q1, k1, v1, dec, qo1, None, None, 0.0, rids[i], before) == 3
                assert gpu.decode_attention_prefix_dev(c.m, qo1, prefix[:3], blocks[:3], dec, out[1]) == 0
                todo.append((i, layer))
    torch.cuda.synchronize()
    gpu.use_current_stream()
    for i, layer in todo:
        c = caches[i]
        gpu.set_layer(c.m, layer)
        front, at = c.read(3, 0, 16 * 12), 0
        for s in range(3):
            k, v = (np.concatenate([a[:16 * blocks[s]], b]) for a, b in zip(front, c.read(s, 0, new[s] + 1)))
            for q, out, rows, seen in ((data[i, layer, 0][3], data[i, layer, 2][0], slice(at, at + new[s]), [16 * blocks[s] + 1 + j for j in range(new[s])]),
                                       (data[i, layer, 1][3], data[i, layer, 2][1], slice(s, s + 1), [len(k)])):
                want, tol = P.attention(P.f64(P.host(q)[rows]), k, v, seen)
                assert np.all(np.abs(out[rows].cpu().double().numpy() - want) <= tol), (i, layer, s, len(seen))
            at += new[s]
    assert gpu.device_errors() == 0
    for rid in rids:
        gpu.rotary_destroy(rid)
    for c in caches:
        c.close()
