"""Shared blocks and differential attention in a cache whose codes lie beyond 4 GiB: the same tokens in a small cache give the same bits."""
import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests.test_kv_gpu import _cache_of, _dev, _say, _torch

pytestmark = pytest.mark.gpu

H, D, B, FAR = 8, 128, 128, 33000  # 128 KB a block: FAR of them pass 2^32 bytes


def _i32(x):
    return _dev(np.asarray(x), _torch().int32)


def test_blocks_beyond_32_bits():
    torch = _torch()
    _say("far", H, D, B, FAR)
    rng = np.random.default_rng(1)
    R, group = 8, 4
    lens = rng.integers(100, 900, (1, R))
    lens[0, 3], lens[0, 5] = 0, 1
    small, near, h = _cache_of(rng, "int8", 1, R, B, D, H, group, lens)
    N = h["N"]
    table = h["table"].copy()
    lead = np.array([[0, 0, 0, 3, 4, 5, 4, 4]])
    for r in (1, 2, 6, 7):  # blocks held together, as many as both have full
        n = min(lens[0, r], lens[0, lead[0, r]]) // B
        table[0, r, :n] = table[0, lead[0, r], :n]
    small.close()
    caches = []
    for off in (0, FAR):
        cfg = kv.KvConfig(rows=R, block_tokens=B, n_blocks=off + 2 * N, max_blocks=h["M"], n_kv_heads=H, n_q_heads=H * group, head_dim=D, fmt="int8", shared=True)
        cache = kv.KvCache(cfg, lens=_i32(lens), table=_dev(np.where(table >= 0, table + off, table).astype(np.int32)))
        layer = cache.new_layer()
        for name in ("k", "v", "k_scale", "v_scale"):
            getattr(layer, name)[off:off + N] = getattr(near, name)
        caches.append((cache, layer, off))
    assert caches[1][1].k.numel() > 2 ** 32
    q = torch.tensor(rng.normal(size=(64, H * group, D)), dtype=torch.bfloat16, device="cuda:0")
    lam = torch.tensor(rng.normal(size=H * group), dtype=torch.float32, device="cuda:0")
    single, many = torch.arange(R, dtype=torch.int32, device="cuda:0")[None], _i32(np.minimum(lens, 8))
    results = []
    for cache, layer, off in caches:
        outs = []
        src, dst = off + np.arange(N)[None], off + N + np.arange(N)[None]
        cache.copy_device(layer, _i32(src), _i32(dst))
        outs += [getattr(layer, name)[off + N:off + 2 * N].view(torch.uint8 if "scale" not in name else torch.int32).clone() for name in ("k", "v", "k_scale", "v_scale")]
        for x in range(2):  # from the first half, then from the copy of it
            for members in (1, 4, 8, 16):
                out, lse = torch.zeros((R, H * group, D), dtype=q.dtype, device="cuda:0"), torch.zeros((R, H * group), device="cuda:0")
                cache.plan_device(_i32(lead), members)
                cache.attend_shared_device(layer, q[:R], out, lse=lse)
                outs += [out, lse.view(torch.int32)]
            for count, longest in ((torch.ones_like(many), 1), (many, 8), (many, 40)):
                out, lse = torch.zeros_like(q), torch.zeros((64, H * group, 2), device="cuda:0")
                cache.attend_diff_device(layer, q, out, lam, lse=lse, start=single * 8, count=count, max_count=longest)
                outs += [out, lse.view(torch.int32)]
            cache.table.copy_(torch.where(cache.table >= 0, cache.table + N, cache.table))
        results.append(outs)
    half = (len(results[0]) - 4) // 2
    for a, b in zip(*results):
        assert torch.equal(a, b)
    for outs in results:
        assert all(bool(torch.isfinite(x.float()).all()) for x in outs[4:] if x.is_floating_point())
        assert any(bool(x.any()) for x in outs[4:])
        for a, b in zip(outs[4:4 + half], outs[4 + half:]):
            assert torch.equal(a, b), "the copy's bits"
    for cache, _, _ in caches:
        cache.close()


def test_compaction_from_beyond_32_bits():
    """One row's blocks lie behind FAR others; as they move to the front their tokens go with them."""
    torch = _torch()
    rng = np.random.default_rng(2)
    n = 5
    lens, table = np.array([[n * B - 3, 0]]), np.full((1, 2, n), -1)
    table[0, 0] = FAR + rng.permutation(2 * n)[:n]
    cfg = kv.KvConfig(rows=2, block_tokens=B, n_blocks=FAR + 2 * n, max_blocks=n, n_kv_heads=H, n_q_heads=H, head_dim=D, fmt="int8", shared=True)
    cache = kv.KvCache(cfg, lens=_i32(lens), table=_i32(table))
    layer = cache.new_layer()
    want = {}
    for name in ("k", "v", "k_scale", "v_scale"):
        x = getattr(layer, name)
        part = x[FAR:]
        part.copy_(torch.randint(0, 256, part.shape, dtype=torch.uint8, device="cuda:0") if "scale" not in name else torch.rand(part.shape, device="cuda:0"))
        want[name] = x[torch.tensor(table[0, 0], device="cuda:0")].clone()
    moves = cache.alloc_moves(n)
    cache.compact_device(moves)
    cache.copy_device(layer, moves["src"], moves["dst"])
    torch.cuda.synchronize()
    ids = cache.table.view(2, n)[0].long()
    assert sorted(ids.tolist()) == list(range(n)) and cache.holders.view(-1)[:n].tolist() == [1] * n and int(cache.holders.sum()) == n
    for name, x in want.items():
        assert torch.equal(getattr(layer, name)[ids], x), name
    cache.close()
