"""Differential attention over the 8-bit cache, without a GPU: what the library and the binding refuse, and a pin of the plain statement."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2605_06113_amd import binding, kv
from tests import kv_oracle as ko
from tests.kv_diff_oracle import attend_diff

GOOD = dict(rows=96, n_blocks=512, max_blocks=64, n_kv_heads=8, n_q_heads=32, head_dim=128)


def test_library_refuses_what_is_missing():
    assert kv.load().br_kv_attend_diff(None, None, None, None) == binding.BR_EINVAL


def test_binding_refuses_what_does_not_fit():
    import torch
    c = object.__new__(kv.KvCache)
    c._sizes(torch, None, kv.KvConfig(**GOOD), torch.device("cpu"))
    c.ctx = None
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    layer = c.layer(u8(512, 8, 16, 128), u8(512, 8, 128, 16), torch.zeros(512, 8), torch.zeros(512, 8))
    q, lam = torch.zeros((5, 32, 128), dtype=torch.float16), torch.zeros(32)
    for bad in (dict(lam=torch.zeros(31)), dict(lam=torch.zeros(5, 31)), dict(lam=torch.zeros(4, 32)), dict(lam=torch.zeros(32).half()), dict(lam=torch.zeros(64)[::2]),
                dict(lam=torch.zeros(32, 5).t()), dict(lam=torch.zeros(())), dict(lse=torch.zeros(5, 32)), dict(lse=torch.zeros(5, 32, 3)), dict(lse=torch.zeros(5, 2, 32)),
                dict(q=q.float(), out=q.float()), dict(out=q.bfloat16()), dict(out=q[:4]), dict(start=torch.zeros((1, 96), dtype=torch.int32)), dict(window=2 ** 31)):
        a = {**dict(q=q, out=q, lam=lam), **bad}
        with pytest.raises(kv.BrError):
            c.attend_diff_device(layer, a.pop("q"), a.pop("out"), a.pop("lam"), **a)


def test_plain_statement_by_hand():
    """One key head of two halves of 32 channels, two tokens: maps (e, e^2) and (1, 1)."""
    k = np.zeros((1, 1, 16, 64), np.uint8)
    k[0, 0, 0, 0], k[0, 0, 1, 0], k[0, 0, :2, 32] = 1, 2, 5
    v = np.zeros((1, 1, 64, 16), np.uint8)
    v[0, 0, 0, :2] = [10, 20]
    one, q = np.ones((1, 1), np.float32), np.zeros((2, 1, 64))
    q[:, 0, 0] = 1.0
    r = attend_diff(q, k, v, one, one, np.array([[0]]), [2], [0], [2], np.array([[0.5], [0.25]]), 1, 16, "int8", scale=1.0)
    first = (10 * math.e + 20 * math.e ** 2) / (math.e + math.e ** 2)
    assert r["out"][0, 0, 0] == 5.0 and r["out"][1, 0, 0] == pytest.approx(first - 0.25 * 15)
    assert r["lse"][1, 0].tolist() == pytest.approx([math.log(math.e + math.e ** 2), math.log(2)])
    r = attend_diff(q, k, v, one, one, np.array([[0]]), [1], [0], [2], np.full((2, 1), math.inf), 1, 16, "int8", scale=1.0)
    assert not r["out"][0].any() and (r["lse"][0] == -math.inf).all() and not np.isfinite(r["out"][1, 0, 0])
