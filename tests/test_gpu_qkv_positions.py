"""Rotations at the ends of the range of positions, by frequencies of either sign and of many circles a token, against 64 bits (tolerance:
test_gpu_qkv_append)."""
import numpy as np
import pytest
import torch

import plain_ops as P
from test_gpu_qkv_append import BF16, close, gpu, inputs  # noqa: F401  (gpu: fixture)

pytestmark = pytest.mark.gpu


def turned(x, pos, freq, pairs):
    """x [rows][heads][D] float64; angles modulo a circle in 80 bits: 2^31 positions of 2^7 radians are off by 2^-26 of one."""
    circle = np.longdouble(2) * (np.longdouble(np.pi) + np.longdouble(1.2246467991473531772e-16))
    ang = np.fmod(np.asarray(pos, dtype=np.longdouble)[:, None] * freq.astype(np.longdouble)[None], circle).astype(np.float64)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    n = x.shape[-1]
    ia, ib = (np.arange(0, n, 2), np.arange(1, n, 2)) if pairs else (np.arange(n // 2), np.arange(n // 2, n))
    a, b = x[..., ia], x[..., ib]
    y, size = np.empty_like(x), np.empty_like(x)
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    size[..., ia] = size[..., ib] = np.abs(a) + np.abs(b)
    return y, size


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_far_positions(gpu, request, d, pairs):  # noqa: F811
    hq, hkv = 4, 2
    rng = np.random.default_rng(d)
    freq = rng.uniform(-1.0, 1.0, d // 2)
    freq[:8] = [1.0, -1.0, 6.5, -40.0, 100.25, -127.9, np.pi, -2.0 ** -40]
    before = np.array([-5, -2000000000, -2 ** 31, 2 ** 31 - 60, 0, 1 << 24, -(1 << 20)], dtype=np.int32)
    ql = np.array([12, 40, 33, 50, 1, 17, 30], dtype=np.int32)
    c = P.Cache(gpu, hq, hkv, d, BF16, [int(x) + 1 for x in ql], frames=8)
    request.addfinalizer(c.close)
    rid = gpu.rotary_create(d, int(pairs), freq)
    request.addfinalizer(lambda: gpu.rotary_destroy(rid))
    for n, ctx in ((ql, ql), (np.ones_like(ql), ql + 1)):
        rows = int(n.sum())
        (q, k, v), (q_b, k_b, _) = inputs((65, rows), rows, hq, hkv, d)
        out = torch.empty((rows, hq, d), dtype=torch.int16, device="cuda")
        if n is ql:
            assert gpu.qkv_append_chunk_dev(c.m, q, k, v, ql, P.i32(ctx), out, None, None, 0.0, rid, P.i32(before)) == rows
        else:
            assert gpu.qkv_append_dev(c.m, q, k, v, P.i32(ctx), out, None, None, 0.0, rid, P.i32(before)) == rows
        seq = np.repeat(np.arange(len(ql)), n)
        idx = np.concatenate([np.arange(a - b, a) for a, b in zip(ctx, n)])
        pos = before.astype(np.int64)[seq] + idx
        torch.cuda.synchronize()
        assert close(P.f64(P.host(out)), *turned(P.f64(q_b), pos, freq, pairs))
        got = np.concatenate([c.read(s, int(a - b), int(b))[0] for s, (a, b) in enumerate(zip(ctx, n))])
        assert close(got, *turned(P.f64(k_b), pos, freq, pairs))
    assert gpu.device_errors() == 0
