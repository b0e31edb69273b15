"""What the binding makes of the tensors of the drafted trees' calls before the library sees them (CPU): where one holds less than the call reads or writes,
the library is told to refuse it."""
import numpy as np
import pytest
import torch

from paper_2505_04021_amd import PrismKV
from test_qkv_arguments import D, HKV, HQ, tensors


class Library:
    """Takes down what it is called with."""

    def __getattr__(self, name):
        def call(*args):
            self.__dict__["args"] = args
            return 0
        return call


@pytest.fixture
def kv():
    kv = PrismKV.__new__(PrismKV)
    kv.torch, kv.lib, kv._shape, kv._bf16 = torch, Library(), {0: (HQ, HKV, D, 0)}, {torch.bfloat16, torch.int16, torch.uint16}
    return kv


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


def test_masks(kv):
    q, k, v, out = tensors(5)
    good = torch.zeros((5, 2), dtype=torch.int64)
    words = lambda sees, n=(3, 2), ctx=i32(2): (kv.tree_attention_dev(0, q, list(n), ctx, sees, out), kv.lib.args[6])[1]
    assert words(good) == 2 and words(good.view(torch.uint64)) == 2 and words(good[:, :1].contiguous()) == 1 and words(good, (2, 2)) == 2
    for bad in (good[:4], good.int(), good[:, :1], good.flatten(), good.t().contiguous().t(), good[:1].expand(5, 2)):
        assert words(bad) == 0, bad.shape
    assert words(good, ctx=i32(1)) == 0
    kv.qkv_append_tree_dev(0, q, k, v, [3, 2], i32(2), good, out)
    assert kv.lib.args[2] is not None and kv.lib.args[6] == 2 and np.array_equal(np.frombuffer(kv.lib.args[3], dtype=np.int32), [3, 2])
    kv.qkv_append_tree_dev(0, q, k, v, [3, 3], i32(2), good, out)
    assert kv.lib.args[2] is None and kv.lib.args[6] == 0 and kv.lib.args[7] is None
    kv.qkv_append_tree_dev(0, q, k[:4], v, [3, 2], i32(2), good, out)
    assert kv.lib.args[2] is None


def test_kept(kv):
    call = lambda n=(3, 2), ctx=i32(2), kept=i32(5), count=i32(2), lens=i32(2): (kv.kv_keep_dev(0, list(n), ctx, kept, count, lens), kv.lib.args[4])[1]
    assert call() is not None and call(lens=None) is not None and call(n=(1, 1)) is not None and call(n=()) is not None
    assert call(n=[1] * 300, ctx=i32(300), kept=i32(300), count=i32(300), lens=None) is not None
    for bad in (dict(kept=i32(4)), dict(count=i32(1)), dict(lens=i32(1)), dict(ctx=i32(1)), dict(kept=i32(10)[::2]), dict(count=i32(4)[::2]), dict(n=(3, 2, 1)),
                dict(n=[1] * 300, ctx=i32(300), kept=i32(299), count=i32(300), lens=None)):
        assert call(**bad) is None, bad


def test_windows(kv):
    q = torch.zeros((5, HQ, D), dtype=torch.bfloat16)
    kv.decode_attention_window_dev(0, q, i32(5), 7, 3, q)
    assert kv.lib.args[:2] == (0, 5) and kv.lib.args[4:6] == (7, 3)
    kv.prefill_attention_window_dev(0, q, np.array([3, 2]), i32(2), 7, 3, q)
    assert kv.lib.args[1] == 2 and kv.lib.args[5:7] == (7, 3)
    with pytest.raises(AssertionError):
        kv.prefill_attention_window_dev(0, q, [3, 2], i32(3), 7, 3, q)
