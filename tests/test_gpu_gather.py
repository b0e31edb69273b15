"""Cached tokens of several sequences as bf16 rows, against kv_read: bf16 caches bit for bit; e4m3 ones decode(code) * scale, rounded once
(a product of two fp32 numbers and one rounding are the same bits in any order of work)."""
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


def expected(c, entries):
    out = [[], []]
    for s, b, n in entries:
        if n == 0:
            continue
        rc, k, v, ks, vs = c.be.kv_read(c.m, s, b, n)
        assert rc == n
        for i, (x, sc) in enumerate(((k, ks), (v, vs))):
            if c.dtype == E4M3:
                y = torch.from_numpy(x).view(torch.float8_e4m3fn).float().numpy() * sc[:, :, None]
                x = gen.to_bf16_bits(torch.from_numpy(y))
            out[i].append(x)
    return [np.concatenate(x) for x in out]


@pytest.mark.parametrize("hkv,d,dtype", [(8, 128, BF16), (2, 64, BF16), (5, 128, BF16), (8, 128, E4M3), (3, 64, E4M3), (1, 128, E4M3)])
def test_ranges(gpu, hkv, d, dtype):
    lens = [37, 16, 1, 100, 400, 0]
    c = P.Cache(gpu, hkv, hkv, d, dtype, lens)
    for s, n in enumerate(lens):
        if n:
            c.fill(s, gen.seq_kv((31, s), n, hkv, d, dtype, 16))
    entries = [(0, 0, 37), (3, 5, 1), (3, 15, 2), (4, 3, 397), (5, 0, 0), (1, 16, 0), (1, 0, 16), (2, 0, 1), (3, 16, 16), (3, 31, 50), (0, 36, 1), (4, 0, 400)]
    n = sum(e[2] for e in entries)
    guard = 64
    k, v = (torch.full((n * hkv * d + 2 * guard,), 0x5555, dtype=torch.int16, device="cuda") for _ in range(2))
    kv = [x[guard:guard + n * hkv * d].view(n, hkv, d) for x in (k, v)]
    assert gpu.kv_gather_dev(c.m, *zip(*entries), *kv) == n
    torch.cuda.synchronize()
    for got, want in zip(kv, expected(c, entries)):
        assert np.array_equal(P.host(got), want)
    for x in (k, v):
        assert (x[:guard] == 0x5555).all() and (x[-guard:] == 0x5555).all()
    assert gpu.device_errors() == 0
    c.close()


def test_many_entries_and_layers(gpu):
    """More entries than a launch holds, the same sequence many times, the second of two layers."""
    c = P.Cache(gpu, 4, 2, 64, E4M3, [200, 90], n_layers=2)
    for layer in range(2):
        gpu.set_layer(c.m, layer)
        for s, n in enumerate(c.lens):
            c.fill(s, gen.seq_kv((33, layer, s), n, 2, 64, E4M3, 16))
    rng = np.random.default_rng(2)
    entries = []
    for _ in range(700):
        s = int(rng.integers(0, 2))
        b = int(rng.integers(0, c.lens[s]))
        entries.append((s, b, int(rng.integers(0, min(6, c.lens[s] - b + 1)))))
    n = sum(e[2] for e in entries)
    k, v = (torch.zeros((n, 2, 64), dtype=torch.int16, device="cuda") for _ in range(2))
    for layer in (1, 0):
        gpu.set_layer(c.m, layer)
        assert gpu.kv_gather_dev(c.m, *zip(*entries), k, v) == n
        torch.cuda.synchronize()
        for got, want in zip((k, v), expected(c, entries)):
            assert np.array_equal(P.host(got), want)
    c.close()


def test_fork_behind_the_last_whole_block(gpu):
    """The tokens of a prefix behind its last whole block, copied to another row."""
    c = P.Cache(gpu, 4, 2, 128, BF16, [40, 30])
    c.fill(0, gen.seq_kv((35,), 40, 2, 128, BF16, 16))
    k, v = (torch.zeros((8, 2, 128), dtype=torch.int16, device="cuda") for _ in range(2))
    assert gpu.kv_gather_dev(c.m, [0], [32], [8], k, v) == 8
    assert gpu.kv_append_chunk_dev(c.m, k, v, [0, 8], P.i32([40, 8])) == 8 and gpu.device_errors() == 0
    for x, y in zip(c.read(0, 32, 8), c.read(1, 0, 8)):
        assert np.array_equal(x, y)
    c.close()


def test_refusals(gpu):
    c = P.Cache(gpu, 4, 2, 64, BF16, [40, 10], frames=2)
    k, v = (torch.zeros((64, 2, 64), dtype=torch.int16, device="cuda") for _ in range(2))
    g = lambda *e, ko=k, vo=v: gpu.kv_gather_dev(c.m, *zip(*e), ko, vo)
    assert gpu.kv_gather_dev(77, [0], [0], [1], k, v) == -2
    assert g((2, 0, 1)) == -1 and g((-1, 0, 1)) == -1 and g((0, -1, 1)) == -1 and g((0, 0, -1)) == -1
    assert g((0, 0, 49)) == -6 and g((0, 48, 1)) == -6 and g((1, 0, 16), (1, 16, 1)) == -6 and g((0, 2 ** 31 - 1, 2 ** 31 - 1)) == -6
    assert g((0, 0, 1), ko=k.view(-1)[1:]) == -1 and g((0, 0, 1), vo=None) == -1
    assert gpu.kv_gather_dev(c.m, [], [], [], k, v) == 0 and g((0, 0, 0)) == 0 and g((1, 2 ** 31 - 1, 0)) == 0
    assert gpu.kv_gather_dev(c.m, [0] * 4097, [0] * 4097, [0] * 4097, k, v) == -6
    assert gpu.device_errors() == 0 and not k.any() and not v.any()
    c.close()
