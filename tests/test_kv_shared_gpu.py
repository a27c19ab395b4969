"""Attention that reads what rows hold together once, on the GPU: each row's result is that of its own tokens (the plain statement in 64 bits, with the
tolerances of attention), whatever is said of who leads whom."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests import kv_oracle as ko
from tests.test_kv_gpu import _cache_of, _check_attention, _dev, _say, _token_type, _torch

pytestmark = pytest.mark.gpu


def _i32(x):
    return _dev(np.asarray(x), _torch().int32)


def _shared_cache(rng, fmt, W, R, b, D, H, group, lens, lead, together, spread=1.0):
    """A cache in which row r holds its leader's first together[r] blocks (as far as both have them, and the leader's are full or as long as the row's)."""
    one, layer, h = _cache_of(rng, fmt, W, R, b, D, H, group, lens, spread)
    table = h["table"].copy()
    for w in range(W):
        for r in range(R):
            f = int(lead[w, r])
            if not 0 <= f < R or f == r:
                continue
            n = min(int(together[w, r]), -(-int(lens[w, r]) // b), -(-int(lens[w, f]) // b))
            while n and lens[w, f] < min(n * b, lens[w, r]):
                n -= 1
            table[w, r, :n] = h["table"][w, f, :n]
    cfg = kv.KvConfig(**{**one.cfg.__dict__, "shared": True})
    cache = kv.KvCache(cfg, lens=_i32(lens), table=_dev(table))
    one.close()
    return cache, cache.layer(layer.k, layer.v, layer.k_scale, layer.v_scale), dict(h, table=table)


def _reference(q, h, lens, start, count, W, group, b, fmt, window, scale):
    ref = None
    R = lens.shape[1]
    for w in range(W):
        blocks, rows = slice(w * h["N"], (w + 1) * h["N"]), slice(w * R, (w + 1) * R)
        one = ko.attend(q, h["k"][blocks], h["v"][blocks], h["ks"][blocks], h["vs"][blocks], h["table"][w], lens[w], start[rows], count[rows], group, b, fmt, window=window, scale=scale)
        if ref is None:
            ref = list(one)
            continue
        m = ~np.isnan(one[1])
        ref[0], ref[1] = np.where(m[..., None], one[0], ref[0]), np.where(m, one[1], ref[1])
        for k in (2, 3, 4):
            ref[k] = ref[k] + one[k]
    return ref


def _case(tag, fmt, dt, D, H, group, b, lens, lead, together, members, counts=None, window=0, wide=True, scale=None, spread=1.0, seed=0, said=None):
    """lens, lead, together [W][R]; counts: rows of one token have a part in it; said: leads that the call is given in place of those that the tables were made with."""
    torch = _torch()
    lens, lead = np.asarray(lens), np.asarray(lead)
    W, R = lens.shape
    together = np.broadcast_to(np.asarray(together), (W, R))
    _say("shared", tag, fmt, dt, "D", D, "H", H, "group", group, "block", b, "rows", (W, R), "longest", lens.max(), "members", members, "window", window)
    rng = np.random.default_rng(seed + D + b)
    cache, layer, h = _shared_cache(rng, fmt, W, R, b, D, H, group, lens, lead, together, spread)
    flat = np.ones(W * R, np.int64) if counts is None else np.asarray(counts).reshape(-1)
    start, at = np.zeros(W * R, np.int64), 1
    for r in rng.permutation(W * R):
        start[r] = at
        at += flat[r] + int(rng.integers(0, 2))
    T, pad, Hq = at + 1, 0 if wide else 1, H * group
    if counts is None:
        start, T = np.arange(W * R), W * R
    q = torch.tensor(rng.normal(size=(T, Hq, D + pad)), dtype=_token_type(dt), device="cuda:0")[:, :, pad:]
    out, lse = torch.full((T, Hq, D + pad), 3.0, dtype=q.dtype, device="cuda:0")[:, :, pad:], torch.full((T, Hq), 3.0, device="cuda:0")
    lists = {} if counts is None else dict(start=_i32(start.reshape(W, R)), count=_i32(flat.reshape(W, R)))
    cache.plan_device(_i32(lead if said is None else said), members, **lists)
    cache.attend_shared_device(layer, q, out, lse=lse, window=window, scale=scale)
    one = np.where(flat == 1, 1, 0)
    ref = _reference(q.double().cpu().numpy(), h, lens, start, one, W, group, b, fmt, window, scale)
    _check_attention(tag, cache, q, out, lse, ref, dt)
    untouched = np.isnan(ref[1])
    assert (out.float().cpu().numpy()[untouched] == 3.0).all() and (lse.cpu().numpy()[untouched] == 3.0).all(), tag
    again = torch.full_like(out, 5.0)
    cache.attend_shared_device(layer, q, again, window=window, scale=scale)
    assert np.array_equal(again.float().cpu().numpy()[~untouched], out.float().cpu().numpy()[~untouched], equal_nan=True), (tag, "equal inputs, equal outputs")
    cache.close()


def _families(R, f):
    return (np.arange(R) // f * f)[None]


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("b", [16, 32, 64, 128])
def test_families(fmt, D, b):
    lens = np.array([[300, 310, 290, 300, 65, 64, 130, 0, 1, 40, 1000, 1025, 1040, 900, 20, 600]])
    dt = "bfloat16" if b in (16, 64) else "float16"
    _case("families", fmt, dt, D, 2, 4, b, lens, _families(16, 4), 256 // b, 4)


@pytest.mark.parametrize("case", [
    # rows, family, group, members, window, shared tokens
    (1, 1, 1, 1, 0, 0), (5, 5, 1, 100, 0, 192), (20, 20, 1, 20, 0, 320), (70, 70, 1, 70, 0, 128), (40, 13, 3, 13, 0, 256), (12, 6, 7, 6, 0, 448), (9, 9, 16, 9, 0, 256),
    (6, 3, 33, 3, 0, 256), (4, 4, 70, 4, 0, 128), (24, 8, 8, 8, 0, 512), (24, 8, 8, 3, 0, 512), (24, 8, 8, 1, 0, 512), (16, 4, 4, 4, 100, 512), (16, 8, 2, 8, 700, 512), (10, 5, 5, 5, 1, 512),
    (10, 10, 2, 10, 64, 192)], ids=str)
@pytest.mark.parametrize("fmt,dt,D", [("int8", "bfloat16", 64), ("fp8", "float16", 128)])
def test_company_sizes(case, fmt, dt, D):
    rows, family, group, members, window, shared = case
    rng = np.random.default_rng(rows)
    lens = shared + rng.integers(0, 150, (1, rows))
    _case("sizes", fmt, dt, D, 1 if group > 16 else 2, group, 16, lens, _families(rows, family), shared // 16, members, window=window)


def test_whatever_is_said_of_leaders():
    """Leads out of range, chains, rings, rows without a common block, rows that share other entries than the first, shorter leaders, members that go apart early."""
    rng = np.random.default_rng(8)
    R = 30
    lens = rng.integers(0, 500, (2, R))
    lens[:, 5], lens[:, 9], lens[0, 0] = 0, 64, 512
    lead = np.concatenate([_families(R, 6), _families(R, 10)])
    together = rng.integers(0, 30, (2, R))
    for k in range(6):
        said = [lead, rng.integers(0, R, (2, R)), np.roll(np.arange(R), 1)[None].repeat(2, 0), rng.choice([-1, R, 2 ** 31 - 1, -2 ** 31, 3], (2, R)), np.zeros((2, R), int),
                np.where(rng.random((2, R)) < 0.5, lead, R - 1 - lead)][k]
        _case(("said", k), "int8", "float16", 64, 2, 3, 16, lens, lead, together, [6, 30, 4, 8, 30, 5][k], said=said, seed=k)


def test_rows_without_a_token_and_with_several():
    """Only rows whose count is 1 are served, leaders without a token lead all the same."""
    rng = np.random.default_rng(9)
    lens = 200 + rng.integers(0, 100, (2, 18))
    counts = rng.choice([0, 1, 1, 1, 2], (2, 18))
    counts[0, 0], counts[1, 6] = 0, 3
    _case("counts", "fp8", "bfloat16", 64, 2, 4, 16, lens, _families(18, 6).repeat(2, 0), 12, 6, counts=counts)


def test_many_rows_and_workers():
    rng = np.random.default_rng(10)
    lens = 70 + rng.integers(0, 60, (3, 300))  # rows beyond the threads of a block
    _case("rows", "int8", "bfloat16", 64, 1, 2, 16, lens, _families(300, 7).repeat(3, 0), 4, 7)
    lens = 130 + rng.integers(0, 9, (1, 1024))
    _case("rows", "int8", "float16", 64, 1, 1, 64, lens, _families(1024, 1024), 2, 1024)


@pytest.mark.parametrize("D", [64, 128, 192, 256])
def test_divisions_of_the_work(D):
    """A company to a block, to several blocks, several to a block, and cut wherever a block's share ends."""
    rng = np.random.default_rng(D)
    for tag, rows, family, members, group, shared, own, H in (("split", 8, 8, 8, 4, 1920, 100, 1), ("split", 5, 5, 5, 12, 2304, 30, 2), ("split", 4, 4, 4, 4, 1500, 60, 3), ("one each", 24, 8, 8, 4, 128, 60, 2),
                                                          ("rounds", 264, 2, 2, 12, 64, 40, 2), ("rounds", 180, 4, 4, 16, 64, 70, 7), ("cut", 264, 2, 2, 9, 64, 40, 2), ("cut", 12, 4, 4, 5, 640, 100, 2)):
        lens = shared + rng.integers(0, own, (1, rows))
        lens[:, :2] += 4000 * (tag == "cut")
        _case((tag, rows), "fp8" if group % 8 else "int8", "bfloat16", D, H, group, 64, lens, _families(rows, family), -(-shared // 64), members, seed=rows)


def test_long_prefixes_that_many_blocks_share():
    _case("long", "fp8", "bfloat16", 128, 2, 4, 64, [[20000, 20100, 19900, 20001]], [[0] * 4], 300, 4)
    _case("long", "int8", "float16", 64, 1, 8, 16, [[9000, 9500, 30, 9100, 9000]], [[0, 0, 2, 0, 0]], 560, 5, wide=False)
    _case("window", "int8", "bfloat16", 128, 1, 4, 32, [[9000, 9500, 8200, 9100]], [[0] * 4], 250, 4, window=3000)
    _case("scale", "fp8", "float16", 96, 2, 4, 32, [[3000, 3100, 2900, 3001]], [[0] * 4], 90, 4, scale=-0.2, spread=3.0)


def test_after_forks_and_steps_captured_with_them():
    """Fork, step, copies, append, plan and attention in one graph, replayed with eager calls between; each time attention's result."""
    torch = _torch()
    W, B, b, H, group, D, F = 1, 12, 16, 2, 4, 64, 4
    side = torch.cuda.Stream()
    cache = kv.KvCache(kv.KvConfig(rows=B, block_tokens=b, n_blocks=400, max_blocks=40, n_kv_heads=H, n_q_heads=H * group, head_dim=D, fmt="fp8", shared=True), stream=side)
    layer, step, prompts = cache.new_layer(), cache.alloc_step(B), cache.alloc_step(2000)
    lead = _i32(_families(B, F))
    cut, one, every = _i32(np.where(np.arange(B) % F, 500, -1)[None]), _i32(np.ones((1, B))), _i32(np.full((1, B), -1))
    first = _i32(np.where(np.arange(B) % F, 0, 200 + 30 * np.arange(B))[None])
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn((2, 2000, H, D), generator=g, device="cuda:0").bfloat16()
    q, k = torch.randn((B, H * group, D), generator=g, device="cuda:0").bfloat16(), torch.randn((2, B, H, D), generator=g, device="cuda:0").bfloat16()
    out, want, lse, lse_want = torch.empty_like(q), torch.empty_like(q), torch.empty((B, H * group), device="cuda:0"), torch.empty((B, H * group), device="cuda:0")
    torch.cuda.synchronize()
    cache.step_device(_i32(np.zeros((1, B))), first, prompts)
    cache.copy_device(layer, prompts["copy_src"], prompts["copy_dst"])
    cache.append_device(layer, x[0], x[1], prompts["slot"])

    def run():
        cache.fork_device(lead, cut)
        cache.step_device(every, one, step)
        cache.copy_device(layer, step["copy_src"], step["copy_dst"])
        cache.append_device(layer, k[0], k[1], step["slot"])
        cache.plan_device(lead, F, start=step["start"], count=step["count"])
        cache.attend_shared_device(layer, q, out, lse=lse)

    def check(tag):
        cache.attend_device(layer, q, want, lse=lse_want, start=step["start"], count=step["count"])
        torch.cuda.synchronize()
        # both are off by the weights' rounding at most, 2^-11 of values up to 448 scales, and by the result's
        assert torch.allclose(lse, lse_want, atol=2.0 ** -18, rtol=0), tag
        assert (out.float() - want.float()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -11) * x.float().abs().max(), tag
        assert bool(torch.isfinite(out.float()).all()) and out.float().abs().max() > 0.01

    run()
    check("eager")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for n in range(4):
        k.copy_(torch.randn(k.shape, generator=g, device="cuda:0")), q.copy_(torch.randn(q.shape, generator=g, device="cuda:0"))
        out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        check(("replay", n))
        if n == 1:  # a plan with other sizes in between
            cache.plan_device(lead, 1)
            cache.attend_shared_device(layer, q, out, lse=lse)
            check("alone")
    cache.close()


def test_a_captured_attention_follows_the_last_plan():
    """Plans with fewer or more members between its replays: the kernel is another plan's, the results are not."""
    torch = _torch()
    for D, group, members in ((64, 4, 8), (128, 2, 4), (192, 4, 16), (128, 4, 2)):
        rng = np.random.default_rng(D + group)
        lens = 200 + rng.integers(0, 200, (1, 16))
        cache, layer, h = _shared_cache(rng, "int8", 1, 16, 16, D, 2, group, lens, _families(16, 16), np.full((1, 16), 12))
        lead = _i32(_families(16, 16))
        q = torch.tensor(rng.normal(size=(16, 2 * group, D)), dtype=torch.float16, device="cuda:0")
        out, lse = torch.empty_like(q), torch.empty((16, 2 * group), device="cuda:0")
        side = torch.cuda.Stream()
        own = kv.KvCache(cache.cfg, lens=cache.lens.clone(), table=cache.table.clone(), stream=side)
        torch.cuda.synchronize()
        own.plan_device(lead, members)
        torch.cuda.synchronize()
        for window in (0, 150):
            ref = _reference(q.double().cpu().numpy(), h, lens, np.arange(16), np.ones(16, np.int64), 1, group, 16, "int8", window, None)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                own.attend_shared_device(layer, q, out, lse=lse, window=window)
            for other in (members, 1, 16, 3, 64):
                with torch.cuda.stream(side):
                    own.plan_device(lead, other)
                    out.fill_(7.0), lse.fill_(7.0)
                    graph.replay()
                torch.cuda.synchronize()
                _check_attention((D, group, members, other, window), own, q, out, lse, ref, "float16")
            own.plan_device(lead, members)
            torch.cuda.synchronize()
        cache.close(), own.close()


def test_a_plan_that_was_captured_and_has_not_run():
    """It has planned nothing: the attention behind it writes no row; once it has run it does."""
    torch = _torch()
    for members in (2, 6, 16):
        rng = np.random.default_rng(members)
        lens = 100 + rng.integers(0, 200, (1, 16))
        cache, layer, h = _shared_cache(rng, "fp8", 1, 16, 16, 128, 2, 4, lens, _families(16, 16), np.full((1, 16), 6))
        side = torch.cuda.Stream()
        own = kv.KvCache(cache.cfg, lens=cache.lens.clone(), table=cache.table.clone(), stream=side)
        lead = _i32(_families(16, 16))
        q = torch.tensor(rng.normal(size=(16, 8, 128)), dtype=torch.float16, device="cuda:0")
        out, lse = torch.full_like(q, 7.0), torch.full((16, 8), 7.0, device="cuda:0")
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            own.plan_device(lead, members)
        own.attend_shared_device(layer, q, out, lse=lse)
        torch.cuda.synchronize()
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
        with torch.cuda.stream(side):
            graph.replay()
            own.attend_shared_device(layer, q, out, lse=lse)
        torch.cuda.synchronize()
        ref = _reference(q.double().cpu().numpy(), h, lens, np.arange(16), np.ones(16, np.int64), 1, 4, 16, "fp8", 0, None)
        _check_attention(("captured", members), own, q, out, lse, ref, "float16")
        cache.close(), own.close()


def test_refusals():
    torch = _torch()
    sizes = dict(rows=2, n_blocks=4, max_blocks=2, head_dim=64)
    one, more = kv.KvCache(kv.KvConfig(**sizes)), kv.KvCache(kv.KvConfig(**sizes, shared=True))
    q = torch.zeros((2, 1, 64), dtype=torch.float16, device="cuda:0")
    p, lib, layer = q.data_ptr(), one.lib, more.new_layer()
    good = dict(q=p, out=p, q_token=64, q_head=64, out_token=64, out_head=64, n_tokens=2, max_count=1, window=0, dtype=0, scale=1.0)
    a = lambda **kw: C.byref(kv._Attention(**{**good, **kw}))
    fam = lambda **kw: C.byref(kv._Families(**{**dict(lead=None, members=2), **kw}))
    assert lib.br_kv_attend_shared(more.ctx, layer.ref, a()) == -1  # no plan
    assert lib.br_kv_plan(one.ctx, fam()) == -1
    for bad in (fam(members=0), fam(members=-3), fam(start=p), fam(count=p)):
        assert lib.br_kv_plan(more.ctx, bad) == -1
    assert lib.br_kv_attend_shared(more.ctx, layer.ref, a()) == -1
    assert lib.br_kv_plan(more.ctx, fam()) == 0 and lib.br_kv_plan(more.ctx, fam(members=2 ** 31 - 1)) == 0
    for bad in (dict(q=None), dict(out=None), dict(n_tokens=-1), dict(max_count=0), dict(window=-1), dict(dtype=2), dict(scale=math.inf), dict(start=p, count=p), dict(lens=p), dict(table=p)):
        assert lib.br_kv_attend_shared(more.ctx, layer.ref, a(**bad)) == -1
    assert lib.br_kv_attend_shared(one.ctx, layer.ref, a()) == -1 and lib.br_kv_attend_shared(more.ctx, None, a()) == -1
    out = torch.full_like(q, 3.0)
    assert lib.br_kv_attend_shared(more.ctx, layer.ref, a(out=out.data_ptr())) == 0
    torch.cuda.synchronize()
    assert not bool(out.any())  # rows of no tokens
    one.close(), more.close()
