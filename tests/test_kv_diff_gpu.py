"""Differential attention over the 8-bit cache on the GPU, against the plain statement in 64 bits.

What it may be off: each map as attention may be (weights times their scales in f16, 2^-11 of each and 2^-32 of the largest for the smallest; scores and sums in
32 bits, 2^-20 of the magnitudes that enter them), the second one lambda times that; the products with lambda and the difference in 32 bits (2^-22 of the two);
and the result is rounded once to its type (2^-12 or 2^-9 of itself, doubled for a value at the type's step)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests.kv_diff_oracle import attend_diff
from tests.test_kv_gpu import _cache_of, _dev, _say, _token_type, _torch

pytestmark = pytest.mark.gpu


def _check(tag, out, lse, r, lam, dt):
    named = ~np.isnan(r["lse"][..., 0])
    got, glse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    wide = 2.0 ** -20 * (8 + r["S"])
    part = r["A"] * (2.0 ** -11 + wide[..., None]) + r["Z"] * 2.0 ** -32
    l = np.abs(lam)[..., None]
    u = 2.0 ** -8 if dt == "bfloat16" else 2.0 ** -11
    tol = part[0] + l * part[1] + 2.0 ** -22 * (r["A"][0] + l * r["A"][1]) + np.abs(np.nan_to_num(r["out"])) * u + 2.0 ** -24 * (dt == "float16")
    bad = named[..., None] & ~(np.abs(got - r["out"]) <= tol)
    assert not bad.any(), (tag, "out", np.argwhere(bad)[:3], got[bad][:3], r["out"][bad][:3], tol[bad][:3])
    seen = named[..., None] & np.isfinite(r["lse"])
    assert np.array_equal(glse[named[..., None] & ~seen], r["lse"][named[..., None] & ~seen]), tag
    bad = seen & ~(np.abs(glse - np.where(seen, r["lse"], 0.0)) <= np.moveaxis(wide, 0, -1))
    assert not bad.any(), (tag, "lse", glse[bad][:3], r["lse"][bad][:3])


def _case(tag, fmt, dt, D, H, group, b, lens, counts, window=0, spread=1.0, max_count=None, wide=True, scale=None, own=True, seed=0, per_token=False, lam_of=None):
    """lens, counts [W][R]; query tokens in an order of their own with gaps between the rows."""
    torch = _torch()
    _say("diff", tag, fmt, dt, "D", D, "H", H, "group", group, "block", b, "rows", np.shape(lens), "longest", np.max(lens), "queries", np.max(counts), "window", window)
    rng = np.random.default_rng(seed + D + b)
    lens, counts = np.asarray(lens), np.asarray(counts)
    W, R = lens.shape
    cache, layer, h = _cache_of(rng, fmt, W, R, b, D, H, group, lens, spread)
    flat = counts.reshape(-1)
    order, start, at = rng.permutation(W * R), np.zeros(W * R, np.int64), 1
    for r in order:
        start[r] = at
        at += flat[r] + int(rng.integers(0, 2))
    T, pad, Hq = at + 1, 0 if wide else 1, H * group
    q = torch.tensor(rng.normal(size=(T, Hq, D + pad)), dtype=_token_type(dt), device="cuda:0")[:, :, pad:]
    out = torch.full((T, Hq, D + pad), 3.0, dtype=q.dtype, device="cuda:0")[:, :, pad:]
    lse = torch.full((T, Hq, 2), 3.0, device="cuda:0")
    lam = rng.normal(size=(T, Hq + 3) if per_token else Hq).astype(np.float32)
    if lam_of is not None:
        lam[...] = lam_of
    dl = torch.tensor(lam, device="cuda:0")
    dl, lam = (dl[:, 2:2 + Hq], lam[:, 2:2 + Hq]) if per_token else (dl, np.broadcast_to(lam, (T, Hq)))
    own_args = {}
    if not own:  # somebody else's tables
        own_args = dict(lens=_dev(lens, torch.int32), table=_dev(h["table"]))
        cache.lens.fill_(1), cache.table.fill_(-1)
    args = dict(lse=lse, start=_dev(start.reshape(W, R), torch.int32), count=_dev(counts, torch.int32), max_count=max_count or max(1, int(counts.max())), window=window, scale=scale, **own_args)
    cache.attend_diff_device(layer, q, out, dl, **args)
    hq, r = q.double().cpu().numpy(), None
    for w in range(W):
        blocks, rows = slice(w * h["N"], (w + 1) * h["N"]), slice(w * R, (w + 1) * R)
        one = attend_diff(hq, h["k"][blocks], h["v"][blocks], h["ks"][blocks], h["vs"][blocks], h["table"][w], lens[w], start[rows], flat[rows], lam, group, b, fmt, window=window, scale=scale)
        if r is None:
            r = one
        else:
            m = ~np.isnan(one["lse"][..., 0])
            for k in ("out", "lse"):
                r[k][m] = one[k][m]
            for k in ("A", "S", "Z"):
                r[k] = r[k] + one[k]
    _check(tag, out, lse, r, lam, dt)
    untouched = np.isnan(r["lse"][..., 0])
    assert (out.float().cpu().numpy()[untouched] == 3.0).all() and (lse.cpu().numpy()[untouched] == 3.0).all(), tag
    again = torch.full_like(out, 5.0)
    cache.attend_diff_device(layer, q, again, dl, **args)
    assert np.array_equal(again.float().cpu().numpy()[~untouched], out.float().cpu().numpy()[~untouched], equal_nan=True), (tag, "equal inputs, equal outputs")
    cache.close()
    return r


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("b", [16, 32, 64, 128])
def test_single_tokens(fmt, D, b):
    lens = [[0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 511, 1000, 1025]]
    _case("single", fmt, "bfloat16" if b in (16, 64) else "float16", D, 2, 4, b, lens, [[1] * 16], per_token=b < 64)


@pytest.mark.parametrize("case", [
    # H, group, lens, counts, window
    (1, 1, [[700, 3, 64]], [[1, 1, 1]], 0), (3, 7, [[33, 900, 260, 5]], [[4, 4, 4, 4]], 0), (2, 16, [[257, 70]], [[1, 1]], 0), (1, 17, [[257, 70]], [[1, 1]], 0),
    (2, 5, [[400, 90, 12]], [[13, 2, 0]], 0), (2, 4, [[333, 64, 500]], [[40, 64, 1]], 0), (1, 8, [[300, 1, 150]], [[300, 1, 150]], 0), (2, 3, [[131, 700]], [[70, 90]], 50),
    (1, 1, [[5, 3, 0, 40]], [[9, 3, 4, 41]], 0), (2, 2, [[1000, 64, 65, 100]], [[1, 1, 1, 2]], 1), (2, 2, [[1000, 640, 65]], [[3, 5, 2]], 64), (1, 6, [[2000]], [[30]], 200),
    (2, 4, [[100, 0, 77], [0, 0, 0], [640, 65, 1]], [[1, 0, 2], [0, 1, 3], [5, 1, 1]], 0), (1, 40, [[500]], [[3]], 0), (40, 1, [[70, 200]], [[1, 2]], 0)], ids=str)
@pytest.mark.parametrize("fmt,dt", [("int8", "float16"), ("fp8", "bfloat16")])
def test_queries(case, fmt, dt):
    H, group, lens, counts, window = case
    _case("queries", fmt, dt, 64, H, group, 16, lens, counts, window=window, per_token=True)
    if H < 5:
        _case("queries", fmt, dt, 128, H, group, 32, lens, counts, window=window, own=False)


@pytest.mark.parametrize("D", [96, 192, 256])
@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_prompts_of_other_widths(D, fmt):
    _case("prompt", fmt, "bfloat16", D, 2, 3, 64, [[200, 90]], [[120, 33]], per_token=True)
    _case("drafts", fmt, "float16", D, 1, 5, 16, [[200, 90, 40]], [[3, 3, 2]], wide=False)


def test_long_rows_that_many_blocks_share():
    _case("long", "fp8", "bfloat16", 128, 2, 4, 64, [[30000]], [[1]])
    _case("long", "int8", "float16", 64, 1, 3, 16, [[20000, 37]], [[5, 1]], per_token=True)
    _case("long", "int8", "bfloat16", 128, 1, 4, 128, [[9000]], [[40]])
    _case("long", "fp8", "float16", 96, 1, 9, 32, [[7000, 5000]], [[2, 1]])


@pytest.mark.parametrize("D", [64, 128, 192, 256])
def test_divisions_of_the_work(D):
    """A query tile to a block, to several blocks, several to a block; few and many query rows; calls of both in one launch and in two."""
    rng = np.random.default_rng(D)
    for tag, H, group, lens, counts in (("split", 1, 16, [[2000]], [[1]]), ("split", 2, 32, [[1500, 1600]], [[1, 1]]), ("split", 2, 4, [[1800]], [[12]]), ("split", 1, 8, [[1500, 300]], [[40, 5]]),
                                        ("many", 2, 4, [[700]], [[300]]), ("rounds", 3, 4, [rng.integers(1, 90, 200)], [[17] + [1] * 199]), ("rounds", 2, 12, [rng.integers(5, 60, 300)], [[1] * 299 + [5]]),
                                        ("one", 2, 4, [rng.integers(20, 90, 30)], [[20] + [1] * 29])):
        _case((tag, H, group), "int8" if group % 8 else "fp8", "bfloat16", D, H, group, 32, np.asarray(lens), np.asarray(counts))


def test_rows_that_are_not_aligned_and_scales_of_any_sign():
    _case("narrow", "int8", "float16", 64, 2, 3, 16, [[100, 400]], [[1, 2]], wide=False, per_token=True)
    _case("narrow", "fp8", "bfloat16", 128, 1, 2, 32, [[100, 300]], [[40, 70]], wide=False)
    for scale in (0.0, -0.3, 1.0):
        _case("scale", "int8", "bfloat16", 64, 1, 4, 16, [[300, 50]], [[1, 40]], scale=scale)


def test_more_query_tiles_than_a_thread_counts():
    """One row of some 5000 query tiles behind a short window: what pieces of it give, every token of it."""
    torch = _torch()
    n, step, window, b, D = 330000, 33000, 150, 128, 64
    _say("diff", "query tiles", n // 64)
    M = -(-n // b)
    cache = kv.KvCache(kv.KvConfig(rows=1, block_tokens=b, n_blocks=M, max_blocks=M, n_kv_heads=1, n_q_heads=1, head_dim=D), lens=_dev(np.array([[n]]), torch.int32),
                       table=_dev(np.arange(M, dtype=np.int32).reshape(1, 1, M)))
    g = torch.Generator("cuda").manual_seed(5)
    layer = cache.new_layer()
    for x in (layer.k, layer.v):
        x.copy_(torch.randint(0, 256, x.shape, generator=g, device="cuda:0", dtype=torch.uint8))
    layer.k_scale.fill_(0.01), layer.v_scale.fill_(1 / 128)
    q = torch.randn((n, 1, D), generator=g, device="cuda:0").half()
    lam = torch.full((1,), 0.3, device="cuda:0")
    out, want, lse, lse_want = torch.full_like(q, 7.0), torch.full_like(q, 7.0), torch.zeros((n, 1, 2), device="cuda:0"), torch.ones((n, 1, 2), device="cuda:0")
    one = lambda x: _dev(np.array([[x]]), torch.int32)
    cache.attend_diff_device(layer, q, out, lam, lse=lse, start=one(0), count=one(n), max_count=n, window=window)
    for at in range(0, n, step):
        cache.attend_diff_device(layer, q, want, lam, lse=lse_want, start=one(at), count=one(step), max_count=step, window=window, lens=one(at + step))
    torch.cuda.synchronize()
    # values of 1 at most: in both results the maps' weights are off by 2^-11 + 2^-15 of them (scores and sums of magnitudes up to 24: 2^-20 of 32), the second map's times
    # 0.3, and each result is rounded by half a step of 1.3
    assert (out.float() - want.float()).abs().max() <= 2 * 1.3 * (2.0 ** -11 + 2.0 ** -15 + 2.0 ** -11)
    assert torch.allclose(lse, lse_want, atol=2 * 2.0 ** -15, rtol=0)
    cache.close()


def test_more_queries_than_said():
    _case("more", "int8", "bfloat16", 64, 2, 4, 16, [[300, 200, 100]], [[9, 1, 30]], max_count=1)


def test_first_map_alone_is_attention():
    """lambda 0 and queries without a second half: attention's result."""
    for counts in ([[1, 1, 1]], [[50, 3, 20]]):
        r = _case("zero", "int8", "float16", 64, 2, 2, 16, [[300, 90, 40]], counts, lam_of=0.0)
        m = ~np.isnan(r["lse"][..., 0])
        assert np.array_equal(r["out"][m], r["o"][0][m])


@pytest.mark.parametrize("lam", [math.inf, math.nan])
def test_lambda_that_is_no_number(lam):
    """A query that sees nothing gets zeros all the same; the others' results are none."""
    torch = _torch()
    rng = np.random.default_rng(2)
    for counts in ([[1, 1, 3]], [[1, 1, 90]]):
        lens = np.array([[0, 50, 2]])
        cache, layer, _ = _cache_of(rng, "int8", 1, 3, 16, 64, 2, 2, lens)
        T = sum(counts[0])
        q = torch.randn((T, 4, 64), device="cuda:0").half()
        out, lse = torch.full_like(q, 3.0), torch.empty((T, 4, 2), device="cuda:0")
        cache.attend_diff_device(layer, q, out, torch.full((4,), lam, device="cuda:0"), lse=lse, start=_dev([[0, 1, 2]], torch.int32), count=_dev(counts, torch.int32), max_count=counts[0][2])
        nothing = lse[..., 0] == -math.inf
        assert nothing.sum().item() == 4 * (1 + counts[0][2] - 2)
        assert not bool(out[nothing].any()) and not bool(torch.isfinite(out[~nothing]).any())
        cache.close()


def test_hidden_tokens_may_be_anything():
    """The largest codes, NaN and infinite scales where the window hides tokens (codes of NaN are no codes of a cache); a scale that is none where it does not."""
    torch = _torch()
    rng = np.random.default_rng(4)
    cache, layer, h = _cache_of(rng, "fp8", 1, 1, 16, 64, 1, 2, np.array([[200]]))
    q, lam = torch.randn((1, 2, 64), device="cuda:0").half(), torch.tensor([0.5, 0.25], device="cuda:0")
    one, two = torch.empty_like(q), torch.empty_like(q)
    cache.attend_diff_device(layer, q, one, lam, window=40)
    for j in range(9):  # tokens 0..143 are hidden
        i = int(h["table"][0, 0, j])
        layer.k[i], layer.v[i] = 0x7E, 0xFE
        layer.k_scale[i], layer.v_scale[i] = math.nan, math.inf
    cache.attend_diff_device(layer, q, two, lam, window=40)
    assert torch.equal(one, two) and bool(torch.isfinite(one).all())
    layer.v_scale[int(h["table"][0, 0, 11])] = math.nan
    cache.attend_diff_device(layer, q, two, lam, window=40)
    assert bool(torch.isnan(two).all())
    cache.close()


def test_captured_and_replayed():
    torch = _torch()
    rng = np.random.default_rng(6)
    for counts in ([[1] * 6], [[70, 1, 2, 1, 1, 33]]):
        lens = np.array([[900, 300, 77, 2000, 5, 640]])
        cache, layer, _ = _cache_of(rng, "int8", 1, 6, 16, 128, 2, 4, lens)
        stream, T = cache.stream, sum(counts[0])
        start, count = _dev(np.cumsum([[0] + counts[0][:-1]], 1), torch.int32), _dev(counts, torch.int32)
        q, lam = torch.randn((T, 8, 128), device="cuda:0").bfloat16(), torch.rand((T, 8), device="cuda:0")
        out, want = torch.empty_like(q), torch.empty_like(q)
        run = lambda o: cache.attend_diff_device(layer, q, o, lam, start=start, count=count, max_count=max(counts[0]))
        run(out)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        own = kv.KvCache(cache.cfg, lens=cache.lens.clone(), table=cache.table.clone(), stream=side)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            own.attend_diff_device(layer, q, out, lam, start=start, count=count, max_count=max(counts[0]))
        for k in range(4):
            q.copy_(torch.randn((T, 8, 128), device="cuda:0")), lam.copy_(torch.rand((T, 8), device="cuda:0"))
            out.zero_()
            run(want)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), k
        cache.close(), own.close()


def test_refusals():
    torch = _torch()
    D = 64
    cache = kv.KvCache(kv.KvConfig(rows=2, n_blocks=4, max_blocks=2, head_dim=D))
    layer, lib = cache.new_layer(), cache.lib
    q = torch.zeros((2, 1, D), dtype=torch.float16, device="cuda:0")
    p = q.data_ptr()
    good = dict(q=p, out=p, q_token=D, q_head=D, out_token=D, out_head=D, n_tokens=2, max_count=1, window=0, dtype=0, scale=1.0)
    lam = C.byref(kv._Diff(lam=p, lambda_token=0))
    for bad in (dict(q=None), dict(out=None), dict(n_tokens=-1), dict(max_count=0), dict(window=-1), dict(dtype=2), dict(scale=math.inf), dict(start=p), dict(count=p), dict(q=p + 1), dict(lse=p + 2),
                dict(n_tokens=2 ** 30)):
        assert lib.br_kv_attend_diff(cache.ctx, layer.ref, C.byref(kv._Attention(**{**good, **bad})), lam) == -1
    a = C.byref(kv._Attention(**good))
    for bad in (None, C.byref(kv._Diff(lam=None)), C.byref(kv._Diff(lam=p + 2))):
        assert lib.br_kv_attend_diff(cache.ctx, layer.ref, a, bad) == -1
    assert lib.br_kv_attend_diff(cache.ctx, None, a, lam) == -1
    assert lib.br_kv_attend_diff(cache.ctx, layer.ref, C.byref(kv._Attention(**{**good, "n_tokens": 0, "q": None})), lam) == 0
    cache.close()
