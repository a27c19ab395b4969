"""Blocks that several rows hold, without a GPU: what the library and the binding refuse, and pins of the plain statement that the GPU tests
compare with."""
import ctypes as C

import pytest

from paper_2605_06113_amd import binding, kv
from tests.kv_pages_oracle import SharedTables

GOOD = dict(rows=96, n_blocks=512, max_blocks=64, n_kv_heads=8, n_q_heads=32, head_dim=128)


def test_structs():
    assert C.sizeof(kv._Families) == kv._PACK_FAMILIES.size == 32 and C.sizeof(kv._Diff) == kv._PACK_DIFF.size == 16
    assert C.sizeof(kv._Forks) == kv._PACK_FORKS.size == 16 and C.sizeof(kv._Moves) == kv._PACK_MOVES.size == 32 and C.sizeof(kv._SharedLayout) == 16
    m = kv._Moves.from_buffer_copy(kv._PACK_MOVES.pack(1, 2, 3, 4, 5))
    assert [getattr(m, f) for f, _ in kv._Moves._fields_] == [1, 2, 3, 4, 5]


def test_workspaces():
    one, more = kv.workspace_bytes(kv.KvConfig(**GOOD)), kv.workspace_bytes(kv.KvConfig(**GOOD, shared=True))
    # a second table, lengths twice, two numbers for each block, one for each worker, thirteen for each row's part in a plan
    need = 4 * (96 * 64 + 2 * 96 + 2 * 512 + 1 + 13 * 96)
    assert one + need <= more <= one + need + 8 * 256
    for bad in (dict(rows=0), dict(head_dim=32), dict(n_blocks=262145), dict(block_tokens=8)):
        assert kv.workspace_bytes(kv.KvConfig(**{**GOOD, **bad}, shared=True)) == 0


def test_init_refusals():
    lib, cfg, ctx = kv.load(), kv.KvConfig(**GOOD, shared=True), C.c_void_p()
    need = kv.workspace_bytes(cfg)
    for at, size, rc in ((0, need, binding.BR_EINVAL), (256 + 4, need, binding.BR_EINVAL), (256, need - 1, binding.BR_ENOMEM)):
        c = kv._config(cfg, workspace=at, workspace_bytes=size)
        assert lib.br_kv_init_shared(C.byref(c), None, C.byref(ctx)) == rc and not ctx.value
    c = kv._config(cfg, workspace=256, workspace_bytes=need)
    assert lib.br_kv_init_shared(C.byref(c), None, None) == binding.BR_EINVAL
    half = kv._State(lens=256, table=0)
    assert lib.br_kv_init_shared(C.byref(c), C.byref(half), C.byref(ctx)) == binding.BR_EINVAL
    for call in (lib.br_kv_fork, lib.br_kv_compact, lib.br_kv_plan):
        assert call(None, None) == binding.BR_EINVAL
    assert lib.br_kv_attend_shared(None, None, None) == binding.BR_EINVAL
    assert lib.br_kv_copy(None, None, None) == binding.BR_EINVAL and lib.br_kv_step_shared(None, None, None, None) == binding.BR_EINVAL
    assert lib.br_kv_get_shared_layout(None, None) == binding.BR_EINVAL


def _cache(**kw):
    """A cache object without a context: what the checks look at."""
    import torch
    c = object.__new__(kv.KvCache)
    c._sizes(torch, None, kv.KvConfig(**{**GOOD, **kw}), torch.device("cpu"))
    c.ctx, c.stream = None, None
    return c


def test_binding_refuses_what_does_not_fit():
    import torch
    c, plain, two = _cache(shared=True), _cache(), _cache(shared=True, n_workers=2)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    out = c.alloc_step(7)
    assert set(out) - set(plain.alloc_step(7)) == {"copy_src", "copy_dst"} and out["copy_src"].shape == (1, 96)
    layer = c.layer(u8(512, 8, 16, 128), u8(512, 8, 128, 16), torch.zeros(512, 8), torch.zeros(512, 8))
    moves, q = c.alloc_moves(5), torch.zeros((5, 32, 128), dtype=torch.float16)
    refused = [
        lambda: plain.fork_device(i32(1, 96)), lambda: plain.compact_device(moves),  # one holder each
        lambda: c.fork_device(i32(96)), lambda: c.fork_device(i32(1, 95)), lambda: c.fork_device(i32(1, 96).long()), lambda: c.fork_device(i32(1, 96), i32(1, 97)),
        lambda: c.fork_device(i32(96, 1).t().expand(1, 96)[:, ::2]), lambda: c.fork_device(i32(1, 192)[:, ::2]),
        lambda: c.step_device(i32(1, 96), i32(1, 96), dict(out, copy_src=i32(1, 95))), lambda: c.step_device(i32(1, 96), i32(1, 96), dict(out, copy_dst=i32(1, 96).float())),
        lambda: c.compact_device(dict(src=i32(5), dst=i32(5))), lambda: c.compact_device(dict(src=i32(1, 5), dst=i32(1, 4))), lambda: c.compact_device(dict(src=i32(2, 5), dst=i32(2, 5))),
        lambda: c.copy_device(layer, i32(5), i32(5)), lambda: c.copy_device(layer, i32(1, 5), i32(1, 6)), lambda: c.copy_device(layer, i32(1, 5).long(), i32(1, 5)),
        lambda: c.copy_device(layer, i32(1, 5), i32(1, 5), src_worker=i32(1, 4)), lambda: c.copy_device(layer, i32(2, 5), i32(2, 5)),
        lambda: two.copy_device(layer, i32(2, 5), i32(2, 5)),  # another cache's layer
        lambda: plain.plan_device(i32(1, 96), 4), lambda: plain.attend_shared_device(layer, q, q),
        lambda: c.plan_device(i32(1, 95), 4), lambda: c.plan_device(i32(1, 96).long(), 4), lambda: c.plan_device(i32(1, 96), 4, start=i32(1, 96)),
        lambda: c.plan_device(i32(1, 96), 4, count=i32(1, 96)), lambda: c.plan_device(i32(1, 96), 4, start=i32(1, 96), count=i32(95)), lambda: c.plan_device(i32(1, 96), 1.5),
        lambda: c.plan_device(i32(1, 96), 2 ** 31),
        lambda: c.attend_shared_device(layer, q[:, :31], q), lambda: c.attend_shared_device(layer, q, q.bfloat16()), lambda: c.attend_shared_device(layer, q, q, lse=torch.zeros(5, 31)),
        lambda: c.attend_shared_device(layer, q, q, window=2 ** 31), lambda: c.attend_shared_device(layer, q.float(), q.float()),
    ]
    for call in refused:
        with pytest.raises(kv.BrError):
            call()
    with pytest.raises(KeyError):
        c.step_device(i32(1, 96), i32(1, 96), plain.alloc_step(7))


def test_forks_of_the_plain_statement():
    t = SharedTables(5, 16, 12, 4)
    t.step([0] * 5, [20, 32, 0, 0, 1], 64)
    assert t.rows == [[0, 1], [2, 3], [], [], [4]]
    t.fork([1, 0, 0, -1, 9], [-1, 100, 16, 3, 0])  # trade places, cut; out of range: as it is
    assert t.rows == [[2, 3], [0, 1], [0], [], [4]] and t.lens == [32, 20, 16, 0, 1]
    assert t.holders()[:5] == [2, 1, 1, 1, 1]
    t.fork([0, 1, 1, 1, 4], [-1, -1, -1, -1, 0])
    assert t.rows == [[2, 3], [0, 1], [0, 1], [0, 1], []] and t.holders()[:5] == [3, 3, 1, 1, 0]
    # all three write into block 1: each gets another, and nobody holds it any more
    o = t.step([-1] * 5, [1, 1, 13, 1, 0], 64)
    assert t.rows == [[2, 3, 4], [0, 5], [0, 6, 7], [0, 8], []]
    assert o["copy_src"] == [-1, 1, 1, 1, -1] and o["copy_dst"] == [-1, 5, 6, 8, -1] and o["slot"][1] == 5 * 16 + 4
    assert o["stats"] == [33 + 21 + 33 + 21, 8, 4, 4, 16, 0, 0, 5]
    # cut back to a point inside block 0, which three hold: one of them writes there
    o = t.step([-1, 5, -1, -1, -1], [0, 2, 0, 0, 0], 64)
    assert t.rows[1] == [1] and o["copy_src"] == [-1, 0, -1, -1, -1] and o["slot"][:2] == [16 + 5, 16 + 6] and t.holders()[0] == 2


def test_refusals_of_the_plain_statement():
    t = SharedTables(3, 16, 3, 4)
    t.step([0] * 3, [20, 0, 0], 64)
    t.fork([0, 0, 0])
    o = t.step([-1] * 3, [1, 1, 1], 64)  # one block is free
    assert o["status"] == [0, 1, 1] and t.rows == [[0, 2], [0, 1], [0, 1]] and t.lens == [21, 20, 20]
    o = t.step([-1, 0, -1], [0, 0, 1], 64)  # block 1 has one holder left
    assert o["status"] == [0, 0, 0] and o["copy_src"] == [-1] * 3 and t.rows[2] == [0, 1]


def test_compaction_of_the_plain_statement():
    t = SharedTables(4, 16, 10, 4)
    t.step([0] * 4, [48, 16, 48, 32], 200)
    t.fork([0, 1, 2, 2], None)
    t.step([0, -1, -1, -1], [0] * 4, 0)
    assert t.rows == [[], [3], [4, 5, 6], [4, 5, 6]]
    one = SharedTables(4, 16, 10, 4, t.lens, [r + [-1] * (4 - len(r)) for r in t.rows])
    assert t.compact(5) == dict(src=[6, 5, 4, -1, -1], dst=[0, 1, 2, -1, -1]) and t.rows == [[], [3], [2, 1, 0], [2, 1, 0]]
    assert one.compact(2) == dict(src=[6, 5], dst=[0, 1]) and one.rows[2] == [4, 1, 0]
    assert t.compact(5)["src"] == [-1] * 5
