"""The worker's part of the library without a GPU: exported symbols, structs, refused configurations and arguments; and pins of the
plain implementations that the GPU tests compare with."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest

from paper_2605_06113_amd import binding, kv
from tests import kv_oracle as ko

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GOOD = dict(rows=96, n_blocks=512, max_blocks=64, n_kv_heads=8, n_q_heads=32, head_dim=128)


def test_library_exports_every_declared_symbol():
    hdr = open(os.path.join(ROOT, "include", "br_kv.h")).read()
    declared = set(re.findall(r"^\s*(?:uint64_t|int32_t|void)\s+(br_kv_[a-z_]+)\s*\(", hdr, re.M))
    assert declared == set(kv.EXPORTS)
    lib = kv.load()
    for name in declared:
        assert hasattr(lib, name)


def test_struct_sizes_match_header():
    assert C.sizeof(kv._Config) == 10 * 4 + 3 * 8
    assert C.sizeof(kv._StepOut) == 6 * 8 + 8
    assert C.sizeof(kv._Tokens) == 3 * 8 + 4 * 8 + 8
    assert C.sizeof(kv._Attention) == 7 * 8 + 4 * 8 + 6 * 4
    for packed, struct in ((kv._PACK_LENGTHS, kv._Lengths), (kv._PACK_STEP, kv._StepOut), (kv._PACK_TOKENS, kv._Tokens), (kv._PACK_ATTENTION, kv._Attention)):
        assert packed.size == C.sizeof(struct)
    # the packed form of the longest one, field by field
    a = kv._Attention.from_buffer_copy(kv._PACK_ATTENTION.pack(*range(1, 16), 0.5, 0))
    assert [getattr(a, f) for f, _ in kv._Attention._fields_] == list(range(1, 16)) + [0.5, 0]


@pytest.mark.parametrize("bad", [dict(rows=0), dict(rows=1025), dict(n_workers=0), dict(n_workers=1 << 20, rows=64), dict(block_tokens=8), dict(block_tokens=48),
                                 dict(block_tokens=256), dict(n_blocks=0), dict(n_blocks=262145), dict(max_blocks=0), dict(max_blocks=65537),
                                 dict(block_tokens=128, max_blocks=8193), dict(n_kv_heads=0), dict(n_q_heads=4), dict(n_q_heads=33), dict(n_q_heads=1032),
                                 dict(head_dim=80), dict(head_dim=32), dict(fmt="int4")])
def test_invalid_config_refused(bad):
    cfg = kv.KvConfig(**{**GOOD, **bad})
    assert kv.workspace_bytes(cfg) == 0
    c, ctx = kv._config(cfg, workspace=256, workspace_bytes=1 << 40), C.c_void_p()
    assert kv.load().br_kv_init(C.byref(c), None, C.byref(ctx)) == binding.BR_EINVAL and not ctx.value


def test_init_argument_errors():
    lib, cfg, ctx = kv.load(), kv.KvConfig(**GOOD), C.c_void_p()
    need = kv.workspace_bytes(cfg)
    assert need % 256 == 0 and need > 96 * 64 * 4
    for at, size, rc in ((0, need, binding.BR_EINVAL), (256 + 4, need, binding.BR_EINVAL), (256, need - 1, binding.BR_ENOMEM)):
        c = kv._config(cfg, workspace=at, workspace_bytes=size)
        assert lib.br_kv_init(C.byref(c), None, C.byref(ctx)) == rc
    c = kv._config(cfg, workspace=256, workspace_bytes=need)
    assert lib.br_kv_init(C.byref(c), None, None) == binding.BR_EINVAL
    half = kv._State(lens=256, table=0)
    assert lib.br_kv_init(C.byref(c), C.byref(half), C.byref(ctx)) == binding.BR_EINVAL
    for call in (lib.br_kv_step, lib.br_kv_append, lib.br_kv_read, lib.br_kv_attend):
        assert call(None, None, None) == binding.BR_EINVAL
    assert lib.br_kv_get_layout(None, None) == binding.BR_EINVAL
    assert lib.br_kv_last_hip_error(None) == 0
    lib.br_kv_free(None)


def _cache(**kw):
    """A cache object without a context: what the checks look at."""
    import torch
    c = object.__new__(kv.KvCache)
    c._sizes(torch, None, kv.KvConfig(**{**GOOD, **kw}), torch.device("cpu"))
    c.ctx = None
    return c


def test_binding_refuses_what_does_not_fit():
    """Shapes, types, strides and devices, before anything reaches the library (there is none here: lib is None)."""
    import torch
    c = _cache()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    f16 = lambda *s: torch.zeros(s, dtype=torch.float16)
    out = c.alloc_step(7)
    with pytest.raises(kv.BrError):
        c.step_device(i32(1, 95), i32(1, 96), out)
    with pytest.raises(kv.BrError):
        c.step_device(i32(1, 96), i32(1, 96).long(), out)
    with pytest.raises(kv.BrError):
        c.step_device(i32(1, 96), i32(1, 96), dict(out, pos=i32(1, 6)))
    with pytest.raises(kv.BrError):
        c.step_device(i32(1, 96), i32(1, 96), dict(out, stats=i32(1, 8)))
    k = f16(7, 8, 128)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    layer = c.layer(u8(512, 8, 16, 128), u8(512, 8, 128, 16), torch.zeros(512, 8), torch.zeros(512, 8))
    for bad in (dict(k=f16(6, 8, 128)), dict(k=f16(7, 8, 64)), dict(k=f16(7, 128, 8).transpose(1, 2)), dict(v=k.float()), dict(k=k.double(), v=k.double()),
                dict(slot=i32(7).long()), dict(slot=i32(14)[::2])):
        a = {**dict(k=k, v=k, slot=i32(7)), **bad}
        with pytest.raises(kv.BrError):
            c.append_device(layer, a["k"], a["v"], a["slot"])
        with pytest.raises(kv.BrError):
            c.read_device(layer, a["slot"], a["k"], a["v"])
    q = f16(5, 32, 128)
    for bad in (dict(q=f16(5, 31, 128)), dict(q=q.float(), out=q.float()), dict(out=q.bfloat16()), dict(out=f16(4, 32, 128)), dict(lse=f16(5, 32)),
                dict(lse=torch.zeros(5, 31)), dict(start=i32(1, 96)), dict(start=i32(1, 95), count=i32(1, 96)), dict(lens=i32(1, 97)), dict(table=i32(1, 96, 63))):
        a = {**dict(q=q, out=q), **bad}
        with pytest.raises(kv.BrError):
            c.attend_device(layer, a.pop("q"), a.pop("out"), **a)
    with pytest.raises(kv.BrError):
        c.layer(*[torch.zeros(512, 8, 16, 128, dtype=torch.uint8)] * 2, torch.zeros(512, 8), torch.zeros(512, 8))
    two = _cache(n_workers=2)
    wide = two.layer(u8(1024, 8, 16, 128), u8(1024, 8, 128, 16), torch.zeros(1024, 8), torch.zeros(1024, 8))
    with pytest.raises(kv.BrError):
        two.append_device(wide, k, k, i32(7))
    for call in (lambda: c.append_device(wide, k, k, i32(7)), lambda: c.read_device(wide, i32(7), k, k), lambda: c.attend_device(wide, q, q)):  # another cache's layer
        with pytest.raises(kv.BrError):
            call()
    for bad in (dict(window=2 ** 31), dict(max_count=1.5), dict(scale="1")):
        with pytest.raises(kv.BrError):
            c.attend_device(layer, q, q, **bad)


def test_e4m3_of_the_oracle():
    import torch
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, ko.E4M3, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).normal(size=4000) * 60, (ko.E4M3[:126] + ko.E4M3[1:127]) / 2, [0.0, -0.0, 448.0, -448.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = x[np.abs(x) <= 448].astype(np.float32)
    assert np.array_equal(ko.encode(x, "fp8"), torch.tensor(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_scales_of_the_oracle(fmt):
    top = ko.TOP[fmt]
    for e in (-100, -99, -7, 0, 5, 90):
        s = 2.0 ** e
        assert ko.scale_for(top * s, fmt) == s
        assert ko.scale_for(np.nextafter(np.float32(top * s), np.float32(np.inf)), fmt) == 2 * s
        assert ko.scale_for(top * s * 0.50001, fmt) == s
    assert ko.scale_for(0.0, fmt) == ko.scale_for(1e-38, fmt) == 2.0 ** -100


def test_tables_of_the_oracle():
    """A worked step: blocks go back before any is taken, lowest first; refusals by table, room and blocks."""
    t = ko.Tables(4, 16, 6, 3)
    o = t.step([0] * 4, [20, 16, 1, 0], 64)
    assert t.rows == [[0, 1], [2], [3], []] and o["stats"] == [37, 4, 2, 3, 37, 0, 0, 4]
    o = t.step([-1, 0, 1, 0], [1, 0, 16, 49], 64)
    assert t.rows == [[0, 1], [], [3, 2], []]
    assert o["slot"][:17] == [1 * 16 + 4] + [3 * 16 + x for x in range(1, 16)] + [2 * 16] and o["slot"][17:] == [-1] * 47
    assert o["status"] == [0, 0, 0, 2] and o["start"] == [0, 1, 1, 17] and o["count"] == [1, 0, 16, 0]
    o = t.step([-1] * 4, [5, 48, 1, 0], 8)
    assert o["status"] == [0, 3, 3, 0]
    o = t.step([-1] * 4, [0, 16, 20, 1], 64)
    assert o["status"] == [0, 0, 0, 1] and t.lens == [26, 16, 37, 0]


def test_attention_of_the_oracle():
    """One key head, one block, by hand; a query that sees nothing; the window."""
    k = ko.encode(np.array([[[[1.0] + [0] * 63, [2.0] + [0] * 63] + [[0.0] * 64] * 14]]), "int8")
    v = np.zeros((1, 1, 64, 16), np.uint8)
    v[0, 0, 0, :2] = [10, 20]
    one = np.ones((1, 1), np.float32)
    q = np.zeros((3, 1, 64))
    q[:, 0, 0] = 1.0
    a = dict(start=[0], count=[3], group=1, block=16, fmt="int8", scale=1.0)
    out, lse, *_ = ko.attend(q, k, v, one, one, np.array([[0]]), [2], **a)
    assert not out[0].any() and lse[0, 0] == -math.inf
    assert out[1, 0, 0] == 10.0 and lse[1, 0] == 1.0
    assert out[2, 0, 0] == pytest.approx((10 * math.e + 20 * math.e ** 2) / (math.e + math.e ** 2)) and lse[2, 0] == pytest.approx(math.log(math.e + math.e ** 2))
    out, lse, *_ = ko.attend(q, k, v, one, one, np.array([[0]]), [2], window=1, **a)
    assert out[2, 0, 0] == 20.0 and lse[2, 0] == 2.0
