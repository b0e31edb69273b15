"""Infinities and NaN in the keys and values of tokens that some queries see and others of the same work-group do not: what a query does not see does not
show in its row, and what it sees does, element by element.  Tolerances: masked_ops.attention."""
import numpy as np
import pytest
import torch

import masked_ops as M
import plain_ops as P
from test_gpu_prefix import BF16, E4M3, gpu, values  # noqa: F401  (gpu: fixture)
from test_gpu_windows import form  # noqa: F401  (fixture)
from workloads import gen

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), float("-inf")]


def spoiled_rows(gpu, rng, hq, hkv, d, dtype, ctx, spots):  # noqa: F811
    """A cache whose rows hold, at the given tokens, V with some elements that are not finite, or a K with one, or (e4m3) a block whose scale is none;
    and its values float64."""
    cache, kv = P.Cache(gpu, hq, hkv, d, dtype, ctx, frames=100), []
    for s, x in enumerate(ctx):
        raw = {name: None if a is None else a.copy() for name, a in gen.seq_kv((91, s), x, hkv, d, dtype, 16).items()}
        for i, t in enumerate(spots[s]):
            h, e = int(rng.integers(hkv)), rng.choice(d, 3, replace=False)
            bits = int(P.bits(np.array([BAD[i % 3]]))[0]) if dtype == BF16 else (0x7f, 0xff)[i % 2]
            if i % 4 == 3:
                raw["k"][t, h, e[0]] = bits
            elif dtype == E4M3 and i % 4 == 2:
                raw["v_scale"][t // 16, h] = BAD[s % 2]
            else:
                raw["v"][t, h, e] = bits
        cache.fill(s, raw)
        with np.errstate(invalid="ignore"):
            kv.append(values(raw, dtype))
    return cache, kv


def check(got, q, kv, n, seen_of):
    at = 0
    for s, m in enumerate(n):
        (k, v), seen = kv[s], seen_of(s)
        g = got.shape[1] // k.shape[1]
        want, tol = M.attention(P.f64(q[at:at + m]), np.nan_to_num(k, nan=0.0, posinf=0.0, neginf=0.0), np.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0), seen)
        lost = ~np.isfinite(v) | ~np.isfinite(k).all(axis=2, keepdims=True)              # [tokens][Hkv][D]
        lost = np.repeat(np.einsum("nt,thd->nhd", seen.astype(np.float64), lost.astype(np.float64)) > 0, g, axis=1)
        mine = got[at:at + m]
        assert np.array_equal(np.isfinite(mine), ~lost), (s, np.argwhere(np.isfinite(mine) == lost)[:5].tolist())
        assert np.all(np.abs(np.where(lost, 0.0, mine - want)) <= tol + 1e-30), s
        assert lost.any() and not lost.all(), s
        at += m


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 64, BF16), (32, 8, 128, BF16), (16, 1, 128, BF16), (32, 8, 128, E4M3), (8, 4, 64, E4M3)])
def test_trees(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Branches that hold such tokens beside branches that do not."""
    n, base = [7, 26, 40, 60], [50, 300, 3000, 0]
    rng = np.random.default_rng(d + hq)
    masks = [M.random_tree(rng, x, 0.7) for x in n]
    ctx = [a + b for a, b in zip(base, n)]
    spots = [[b + int(j) for j in rng.choice(np.arange(1, x), min(x // 3, 6), replace=False)] for x, b in zip(n, base)]
    if dtype == E4M3:
        spots = [x[:2] for x in spots]                                   # (a block's scale would be lost to nearly all)
    cache, kv = spoiled_rows(gpu, rng, hq, hkv, d, dtype, ctx, spots)
    q = gen.queries((92, d), sum(n), hq, d)
    out = torch.empty((sum(n), hq, d), device="cuda")
    for window in (0, 64):
        assert gpu.tree_attention_dev(cache.m, P.dev(q), n, P.i32(ctx), M.words_of(sum(masks, []), 1), out, window, 3) == 0
        check(out.cpu().double().numpy(), q, kv, n, lambda s: M.tree_seen(ctx[s], masks[s], window, 3))
    assert gpu.device_errors() == 0
    cache.close()


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 64, BF16), (32, 8, 128, BF16), (16, 1, 128, BF16), (32, 8, 128, E4M3), (8, 4, 64, E4M3)])
def test_windows(gpu, form, hq, hkv, d, dtype):  # noqa: F811
    """Such tokens where the windows of the first queries end and the later ones' have not begun, and among the chunk's own."""
    n, ctx, window, sinks = [20, 33, 70, 100], [300, 33, 4000, 2000], 48, 4
    rng = np.random.default_rng(d + hq)
    # token t is seen by the queries from t to t + window - 1
    spots = [sorted({max(x - m - window + 10, sinks), max(x - m - window + 17, sinks + 1), x - m // 2, x - 3}) for x, m in zip(ctx, n)]
    cache, kv = spoiled_rows(gpu, rng, hq, hkv, d, dtype, ctx, spots)
    q = gen.queries((93, d), sum(n), hq, d)
    out = torch.empty((sum(n), hq, d), device="cuda")
    assert gpu.prefill_attention_window_dev(cache.m, P.dev(q), n, P.i32(ctx), window, sinks, out) == 0
    check(out.cpu().double().numpy(), q, kv, n, lambda s: M.window_seen(ctx[s], n[s], window, sinks))
    assert gpu.device_errors() == 0
    cache.close()
