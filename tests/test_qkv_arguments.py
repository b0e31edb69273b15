"""What the binding makes of the tensors of qkv_append before the library sees them (CPU): every row that a call reads or writes is there, or the library
is told to refuse it."""
import numpy as np
import pytest
import torch

from paper_2505_04021_amd import PrismKV, binding

HQ, HKV, D = 8, 2, 64


class Library:
    """Takes down what it is called with."""

    def qkv_append(self, model, batch, x, ctx_lens, q_out):
        self.x = x
        return batch

    def qkv_append_chunk(self, model, batch, x, q_lens, ctx_lens, q_out):
        self.x = x
        return int(np.frombuffer(q_lens, dtype=np.int32).sum())


@pytest.fixture
def kv():
    kv = PrismKV.__new__(PrismKV)
    kv.torch, kv.lib, kv._shape, kv._bf16 = torch, Library(), {0: (HQ, HKV, D, 0)}, {torch.bfloat16, torch.int16, torch.uint16}
    return kv


def tensors(n, dtype=torch.bfloat16):
    x = torch.zeros((n, HQ + 2 * HKV, D), dtype=dtype)
    return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], torch.zeros((n, HQ, D), dtype=dtype)


def both(kv, n, q, k, v, out, lens=None, **kw):
    """The calls' arguments as the library gets them, as (strides, whole tuple), or None."""
    seen = []
    for chunk in (False, True):
        ctx = torch.ones(n, dtype=torch.int32)
        if chunk:
            kv.qkv_append_chunk_dev(0, q, k, v, lens or [1] * n, ctx, out, **kw)
        else:
            kv.qkv_append_dev(0, q, k, v, ctx, out, **kw)
        seen.append(kv.lib.x and binding._QKV.unpack(kv.lib.x))
    assert seen[0] == seen[1]
    return seen[0]


def test_layouts_that_go_as_they_are(kv):
    row = (HQ + 2 * HKV) * D
    for dtype in (torch.bfloat16, torch.int16, torch.uint16):
        q, k, v, out = tensors(3, dtype)
        assert both(kv, 3, q, k, v, out)[:6] == (q.data_ptr(), k.data_ptr(), v.data_ptr(), row, row, row)
        assert both(kv, 2, q, k, v, out)[3] == row                        # more rows than the call takes
    q, k, v, out = tensors(1)
    assert both(kv, 1, q, k, v, out)[3:6] == (0, 0, 0)
    assert both(kv, 1, q.expand(1, HQ, D), k, v, out)[3] == 0


def test_tokens_in_one_place(kv):
    """A broadcast axis of tokens has a distance of 0, which says "packed" to the library: it gets one that it refuses, less than a row."""
    q, k, v, out = tensors(4)
    for i in range(3):
        x = [q, k, v]
        x[i] = x[i][:1].expand(4, -1, -1)
        assert 0 < both(kv, 4, *x, out)[3 + i] < HKV * D
        x[i] = x[i][0].contiguous().expand(4, -1, -1)
        assert 0 < both(kv, 4, *x, out)[3 + i] < HKV * D


def test_tensors_that_hold_too_little(kv):
    q, k, v, out = tensors(4)
    one = torch.ones(D, dtype=torch.bfloat16)
    for i in range(4):
        x = [q, k, v, out]
        x[i] = x[i][:3]
        assert both(kv, 4, *x) is None
    for bad in (None, out[:, :, :32], torch.zeros((HQ, 4, D), dtype=out.dtype).transpose(0, 1), out[:1].expand(4, -1, -1)):
        assert both(kv, 4, q, k, v, bad) is None
    assert both(kv, 4, q, k, v, out, before=torch.zeros(4, dtype=torch.int32), q_weight=one, k_weight=one) is not None
    for bad in (torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32).expand(4)):
        assert both(kv, 4, q, k, v, out, before=bad) is None
    for bad in (one[:32], one.float(), torch.ones(2 * D, dtype=torch.bfloat16)[::2], one[:1].expand(D)):
        assert both(kv, 4, q, k, v, out, q_weight=bad) is None and both(kv, 4, q, k, v, out, k_weight=bad) is None
    # chunks: by the sum of their lengths, few sequences and many
    ctx = torch.ones(100, dtype=torch.int32)
    for lens, fits in (([1, 3], True), ([2, 3], False), ([0, 0], True), ([0] * 99 + [4], True), ([0] * 99 + [5], False)):
        kv.qkv_append_chunk_dev(0, q, k, v, lens, ctx[:len(lens)], out)
        assert (kv.lib.x is not None) == fits, lens
    kv.qkv_append_chunk_dev(0, q, k, v, [1, 1], ctx[:1], out)
    assert kv.lib.x is None
    kv.qkv_append_dev(7, q, k, v, ctx[:4], out)                           # no such model: the library says so
    assert kv.lib.x is None


def test_layouts_that_cannot_be_said(kv):
    q, k, v, out = tensors(2)
    for bad in (q.half(), q.float(), q.transpose(0, 1), q[:, :4], q[:, :, :32], q[:, ::2], torch.zeros((2, D, HQ), dtype=q.dtype).transpose(1, 2), q[0]):
        with pytest.raises(ValueError):
            both(kv, 2, bad, k, v, out)
