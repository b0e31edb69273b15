"""Decode steps behind shared prefixes, captured while the rows are short and replayed when they have grown far beyond the parts that the capture
cut them into (tolerances: plain_ops.attention)."""
import numpy as np
import pytest
import torch

import plain_ops as P
from test_gpu_prefix import BF16, E4M3, Rows, form, gpu  # noqa: F401  (fixtures)
from workloads import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, BF16), (16, 8, 64, E4M3)])
@pytest.mark.parametrize("short", ["one part", "several parts"])
def test_rows_grown_since_the_capture(gpu, request, form, hq, hkv, d, dtype, short):  # noqa: F811
    n = 12
    start = [100] * n if short == "one part" else [600, 40, 16, 700] * 3
    grown = [[1500, 2900, 200, 0, 3000, 17] * 2, [2999, 384, 385, 768, 769, 1600] * 2, start]
    rows = Rows(gpu, hq, hkv, d, dtype, [3000] * n + [16 * 40, 16 * 9], frames=100)
    c = rows.c
    request.addfinalizer(c.close)
    prefix, blocks = [n] * 8 + [n + 1, n + 1, -1, -1], [40] * 8 + [9, 7, 0, 0]
    for s in range(n):
        gpu.seq_release(c.m, s)
    assert gpu.seq_reserve_batch(c.m, list(range(n)), start) >= 0
    fill = lambda lens: [c.fill(s, gen.seq_kv((7, s), 3000, hkv, d, dtype, 16, peak_frac=0.02), x) for s, x in enumerate(lens)]
    fill(start)
    q, ctx = P.dev(gen.queries((51, d), n, hq, d)), P.i32(start)
    out = torch.zeros((n, hq, d), device="cuda")
    call = lambda: gpu.decode_attention_prefix_dev(c.m, q, prefix, blocks, ctx, out)
    assert call() == 0 and gpu.last_prefix_form() == form
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        gpu.use_current_stream()
        assert call() == 0
    gpu.use_current_stream()
    for upto in range(48, 3048, 48):
        assert gpu.seq_reserve_batch(c.m, list(range(n)), [min(upto, 3000)] * n) >= 0
    fill([3000] * n)
    for lens in [start] + grown:
        ctx.copy_(P.i32(lens))
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().double().numpy()
        for s, x in enumerate(lens):
            k, v = rows.context(prefix[s], blocks[s], s, x)
            want, tol = P.attention(P.f64(P.host(q)[s:s + 1]), k, v, [len(k)])
            assert np.all(np.abs(got[s:s + 1] - want) <= tol + 1e-30), (lens[:6], s)
    assert gpu.device_errors() == 0
