"""A token's key is the same to the bit whichever call appended it: a decode step, a chunk of one token or a longer chunk; and so are an e4m3
cache's codes and scales, and the queries."""
import numpy as np
import pytest
import torch

import plain_ops as P
from test_gpu_qkv_append import BF16, E4M3, gpu, inputs, weights  # noqa: F401  (gpu: fixture)

pytestmark = pytest.mark.gpu

N = 150


@pytest.mark.parametrize("dtype", [BF16, E4M3])
@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 128), (16, 8, 64)])
# rot, pairs, norm, pad, shift
@pytest.mark.parametrize("form", [("all", False, True, 0, 0), ("all", False, False, 0, 0), ("all", True, True, 0, 0), ("all", True, False, 8, 0), (64, False, True, 0, 0),
                                  (64, False, False, 3, 1), (32, False, True, 0, 0), (20, False, True, 5, 1), (34, True, True, 0, 0), (0, False, True, 0, 0)], ids=str)
def test_step_and_chunk_leave_the_same(gpu, request, dtype, hq, hkv, d, form):  # noqa: F811
    rot, pairs, norm, pad, shift = form
    rot = d if rot == "all" else rot
    rid = gpu.rotary_create(rot, int(pairs), P.frequencies(rot), 1.25) if rot else -1
    request.addfinalizer(lambda: gpu.rotary_destroy(rid))
    c = P.Cache(gpu, hq, hkv, d, dtype, [N, N, N], frames=16)
    request.addfinalizer(c.close)
    (wq, wk), _ = weights((61, d), d) if norm else ((None, None), None)
    (q, k, v), _ = inputs((62, d, rot), N, hq, hkv, d, pad, shift)
    outs = [torch.full((N, hq, d), -1, dtype=torch.int16, device="cuda") for _ in range(3)]
    before = P.i32([777, 777, 777])
    chunk = lambda rows, ql, ctx, out: gpu.qkv_append_chunk_dev(c.m, q[rows], k[rows], v[rows], ql, P.i32(ctx), out[rows], wq, wk, 1e-6, rid, before)
    for t in range(N):
        at = slice(t, t + 1)
        assert gpu.qkv_append_dev(c.m, q[at], k[at], v[at], P.i32([t + 1]), outs[0][at], wq, wk, 1e-6, rid, before) == 1
        assert chunk(at, [0, 1, 0], [0, t + 1, 0], outs[1]) == 1
    for lo, hi in ((0, 5), (5, 70), (70, N)):
        assert chunk(slice(lo, hi), [0, 0, hi - lo], [0, 0, hi], outs[2]) == hi - lo
    torch.cuda.synchronize()
    read = [gpu.kv_read(c.m, s, 0, N)[1:] for s in range(3)]
    for s in (1, 2):
        for x, y in zip(read[0], read[s]):
            assert x is None and y is None or np.array_equal(x, y), (s, int((x != y).sum()), x.size)
        assert torch.equal(outs[0], outs[s])
    assert gpu.device_errors() == 0
