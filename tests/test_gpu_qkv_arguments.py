"""qkv_append's refusals of tensors that hold less than a call reads or writes: nothing is enqueued, nothing written."""
import pytest
import torch

import plain_ops as P
from test_gpu_qkv_append import BF16, gpu, inputs  # noqa: F401  (gpu: fixture)

pytestmark = pytest.mark.gpu


def test_too_little(gpu, request):  # noqa: F811
    hq, hkv, d, n = 8, 2, 64, 4
    c = P.Cache(gpu, hq, hkv, d, BF16, [16] * n, frames=2)
    request.addfinalizer(c.close)
    (q, k, v), _ = inputs((63,), n, hq, hkv, d)
    out, ctx = torch.full((n, hq, d), 7, dtype=torch.int16, device="cuda"), P.i32([1] * n)
    wide = lambda x: x[:1].expand(n, -1, -1)
    bad = [dict(q=wide(q)), dict(k=wide(k)), dict(v=wide(v)), dict(q=q[:3]), dict(k=k[:3]), dict(v=v[:3]), dict(q_out=out[:3]), dict(before=P.i32([0] * 3))]
    for b in bad:
        a = dict(dict(q=q, k=k, v=v, q_out=out), **b)
        assert gpu.qkv_append_dev(c.m, ctx_lens=ctx, **a) == -1, b.keys()
        assert gpu.qkv_append_chunk_dev(c.m, ctx_lens=ctx, q_lens=[1] * n, **a) == -1, b.keys()
    torch.cuda.synchronize()
    assert (out == 7).all() and gpu.device_errors() == 0
    assert gpu.qkv_append_dev(55, q, k, v, ctx, out) == -2
    # more rows than the call takes are no fault
    assert gpu.qkv_append_chunk_dev(c.m, q, k, v, [1, 1, 0, 0], ctx, out) == 2
    torch.cuda.synchronize()
    assert torch.equal(out[:2], q[:2]) and (out[2:] == 7).all() and gpu.device_errors() == 0
