"""NaN in queries, keys and values of sequences that share prefixes: it reaches the rows whose formula it enters, in whichever way the library walks
the contexts, and no others; these are right (tolerances: plain_ops.attention)."""
import numpy as np
import pytest
import torch

import plain_ops as P
from test_gpu_prefix import BF16, E4M3, Rows, form, gpu  # noqa: F401  (fixtures)
from workloads import gen

pytestmark = pytest.mark.gpu

N, WIDE, NARROW = 16, 9, 3                   # the batch: members behind a prefix in row 16, behind one in row 17, the others without
PREFIX = [N] * WIDE + [N + 1] * NARROW + [-1] * (N - WIDE - NARROW)


def nan_of(dtype):
    return 0x7FC0 if dtype == BF16 else 0x7F


def fill(rows, s, kv, n, dtype):
    """Puts row s in the cache and into rows.kv."""
    from test_gpu_prefix import values
    rows.c.fill(s, kv, n)
    rows.kv[s] = [x[:n] for x in values(kv, dtype)]


def check(gpu, rows, q, blocks, own, prefill):
    c = rows.c
    out = torch.full((N, c.hq, c.d), 7.0, device="cuda")
    if prefill:
        assert gpu.prefill_attention_prefix_dev(c.m, P.dev(q), [1] * N, PREFIX, blocks, P.i32(own), out) == 0
    else:
        assert gpu.decode_attention_prefix_dev(c.m, P.dev(q), PREFIX, blocks, P.i32(own), out) == 0
    got, q64, g, seen = out.cpu().double().numpy(), P.f64(q), c.hq // c.hkv, 0
    for s, n in enumerate(own):
        k, v = rows.context(PREFIX[s], blocks[s], s, n)
        lost = np.zeros((c.hq, c.d), dtype=bool)                          # where the formula gives NaN
        for h in range(c.hq):
            lost[h] = np.isnan(k[:, h // g] @ q64[s, h]).any() | np.isnan(v[:, h // g]).any(axis=0)
        want, tol = P.attention(np.nan_to_num(q64[s:s + 1]), np.nan_to_num(k), np.nan_to_num(v), [len(k)])
        assert np.array_equal(np.isnan(got[s]), lost), (s, np.isnan(got[s]).sum(), lost.sum())
        assert np.all((np.abs(got[s] - want[0]) <= tol[0]) | lost), s
        seen += lost.any()
    assert seen and not gpu.device_errors()


@pytest.mark.parametrize("where", ["queries", "keys of rows", "values of rows far below", "keys of prefixes", "values of prefixes"])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, BF16), (8, 2, 64, E4M3)])
def test_nan(gpu, request, form, hq, hkv, d, dtype, where):  # noqa: F811
    """Wide and narrow groups and sequences without a prefix; prefixes in several parts, of which one holds nothing but NaN."""
    own = [int(x) for x in gen.ctx_lognormal(N, 60, 0.8, 300, gen.generator(31))]
    own[2] = 700                                                          # in several parts
    shared = [16 * 160, 16 * 100]
    rows = Rows(gpu, hq, hkv, d, dtype, own + shared, frames=40)
    request.addfinalizer(rows.c.close)
    blocks = [shared[p - N] // 16 if p >= 0 else 0 for p in PREFIX]
    q = gen.queries((32, d), N, hq, d)
    some = (1, 2, WIDE + 1, N - 2)                                        # two of the wide group, one of the narrow one, one without a prefix
    if where == "queries":
        for s, h in zip(some, (0, 3, 5, 7)):
            q[s, h, s] = nan_of(BF16)
    for s in some:
        kv = gen.seq_kv((7, s), own[s], hkv, d, dtype, 16, peak_frac=0.02)
        if where == "keys of rows":
            kv["k"][:, 1] = nan_of(dtype)
        if where == "values of rows far below":
            # logits of -16 sqrt(d) behind a prefix's of some 10: they weigh 2^-170 and less, and a NaN that they weigh is one
            q[s] = 0x3F80
            kv["k"][:] = 0xC180 if dtype == BF16 else 0xD8
            kv["v"][own[s] // 2, 0, 3] = nan_of(dtype)
            if dtype == E4M3:
                kv["k_scale"][:] = 1.0
        if where.endswith("rows") or where.endswith("far below"):
            fill(rows, s, kv, own[s], dtype)
    for i, n in enumerate(shared):
        kv = gen.seq_kv((7, N + i), n, hkv, d, dtype, 16, peak_frac=0.02)
        if where == "keys of prefixes":
            kv["k"][n // 2:, 0] = nan_of(dtype)                           # whole parts
        if where == "values of prefixes":
            kv["v"][n // 3, 1, 5] = nan_of(dtype)
        if where.endswith("prefixes"):
            fill(rows, N + i, kv, n, dtype)
    check(gpu, rows, q, blocks, own, False)
    assert gpu.last_prefix_form() == form
    check(gpu, rows, q, blocks, own, True)
