"""Block tables, the 8-bit cache and the attention over it on the GPU, against plain implementations in whole numbers and 64 bits.

Tables, codes and scales have to be equal.  What attention may be off: weights, times their tokens' scales, are rounded to f16 (2^-11 of
each, 2^-32 of the largest for the smallest), scores and sums are formed in 32 bits (2^-20 of the magnitudes that enter them, with room for 256 terms and
the exponential's last bits), and the result is rounded once to its type (2^-11 or 2^-8 of itself)."""
import math

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests import kv_oracle as ko

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _dev(x, dtype=None):
    torch = _torch()
    return torch.as_tensor(np.ascontiguousarray(x), device="cuda:0") if dtype is None else torch.as_tensor(np.ascontiguousarray(x), dtype=dtype, device="cuda:0")


def _say(*a):
    print(*a, flush=True)


# -- tables -----------------------------------------------------------------
TABLES = [  # workers, rows, block, n_blocks, max_blocks, cap, longest request
    (1, 1, 16, 1, 1, 1, 16), (1, 4, 16, 31, 8, 64, 100), (3, 7, 32, 33, 5, 100, 160), (2, 64, 16, 400, 40, 700, 500), (1, 96, 16, 3000, 300, 4096, 2000),
    (5, 255, 64, 900, 30, 2000, 1500), (2, 256, 16, 1025, 64, 0, 900), (1, 257, 128, 700, 20, 5000, 2000), (2, 1024, 16, 9000, 70, 3001, 1000),
    (1, 40, 16, 262144, 65536, 300000, 200000), (300, 13, 32, 64, 9, 77, 200),
]


@pytest.mark.parametrize("case", TABLES, ids=str)
def test_tables(case):
    W, B, b, N, M, cap, longest = case
    _say("tables", case)
    rng = np.random.default_rng(W * 1000 + B)
    cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M))
    oracles = [ko.Tables(B, b, N, M) for _ in range(W)]
    out = cache.alloc_step(cap)
    for k in range(12):
        lens = np.array([o.lens for o in oracles])
        keep = np.where(rng.random((W, B)) < 0.7, -1, rng.integers(-2, longest, (W, B)))
        keep = np.where(rng.random((W, B)) < 0.2, 0, keep)
        add = np.where(rng.random((W, B)) < 0.7, 1, np.exp(rng.uniform(0, math.log(longest), (W, B))).astype(int))
        add = np.where(rng.random((W, B)) < 0.1, rng.choice([0, -5, 2 ** 31 - 1, M * b, M * b + 1], (W, B)), add)
        if k == 6:
            keep, add = np.zeros((W, B), int), np.zeros((W, B), int)  # everything leaves
        for x in out.values():
            x.fill_(-77)
        cache.step_device(_dev(keep, _torch().int32), _dev(add, _torch().int32), out)
        ref = [o.step(keep[w], add[w], cap) for w, o in enumerate(oracles)]
        got = {n: x.cpu().numpy() for n, x in out.items()}
        for w in range(W):
            ref[w]["start"] = [w * cap + x for x in ref[w]["start"]]
            for name in ("count", "status", "start", "slot", "pos", "stats"):
                assert np.array_equal(got[name][w], ref[w][name]), (case, k, w, name)
        assert np.array_equal(cache.lens.cpu().numpy(), [o.lens for o in oracles]), (case, k)
        if W * B * M < 3e6:
            assert np.array_equal(cache.table.cpu().numpy(), [o.table() for o in oracles]), (case, k)
    cache.close()


def _scattered(rng, lens, b, N, M):
    """Block tables of rows of those lengths, in any order of blocks: [W, R, M]."""
    W, R = lens.shape
    table = np.full((W, R, M), -1, np.int32)
    for w in range(W):
        ids, at = rng.permutation(N), 0
        for r in range(R):
            n = -(-int(lens[w, r]) // b)
            table[w, r, :n] = ids[at:at + n]
            at += n
        assert at <= N
    return table


def test_tables_start_from_given_requests_and_skip_outputs():
    rng = np.random.default_rng(5)
    W, B, b, N, M = 2, 30, 16, 200, 20
    lens = rng.integers(0, 100, (W, B))
    table = _scattered(rng, lens, b, N, M)
    stale = np.where(table < 0, 7, table)  # entries behind a row's blocks are not looked at
    cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M), lens=_dev(lens, _torch().int32), table=_dev(stale))
    assert np.array_equal(cache.table.cpu().numpy(), table) and np.array_equal(cache.lens.cpu().numpy(), lens)
    oracles = [ko.Tables(B, b, N, M, lens[w], table[w]) for w in range(W)]
    keep, add = rng.integers(-1, 90, (W, B)), rng.integers(0, 60, (W, B))
    import ctypes as C
    dk, da = _dev(keep, _torch().int32), _dev(add, _torch().int32)
    a, o = kv._Lengths(keep=dk.data_ptr(), add=da.data_ptr()), kv._StepOut(token_cap=900)
    assert cache.lib.br_kv_step(cache.ctx, C.byref(a), C.byref(o)) == 0  # every output left out
    for w in range(W):
        oracles[w].step(keep[w], add[w], 900)
    assert np.array_equal(cache.table.cpu().numpy(), [x.table() for x in oracles])
    for bad in (kv._StepOut(token_cap=-1), kv._StepOut(token_cap=2 ** 30)):
        assert cache.lib.br_kv_step(cache.ctx, C.byref(a), C.byref(bad)) == -1
    # ids outside the worker's blocks count as none; lengths are clamped to the table
    table[0, 0, :3], lens[0, 0], lens[1, 1] = [5, N, -3], 40, 10 ** 6
    table[0, 1:], table[1] = -1, -1
    c2 = kv.KvCache(kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M), lens=_dev(lens, _torch().int32), table=_dev(table))
    assert c2.table[0, 0, :4].tolist() == [5, -1, -1, -1] and c2.lens[1, 1].item() == M * b
    cache.close(), c2.close()


# -- append and read ----------------------------------------------------------
def _token_type(name):
    return getattr(_torch(), name)


APPEND = [(fmt, dt, D, b, H, W) for fmt in ("int8", "fp8") for dt, D, b, H, W in (
    ("bfloat16", 128, 16, 8, 1), ("float16", 64, 32, 1, 1), ("float32", 96, 64, 5, 2), ("bfloat16", 256, 128, 2, 1), ("float16", 192, 16, 3, 3))]


@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append_and_read(case):
    """Steps of prompts, single tokens and rejected drafts; magnitudes over many orders; zeros, values that are not finite."""
    torch = _torch()
    fmt, dt, D, b, H, W = case
    _say("append", case)
    rng = np.random.default_rng(D + b)
    B, N, M, cap = 9, 60, 12, 150
    cfg = kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=H, n_q_heads=H, head_dim=D, fmt=fmt)
    cache = kv.KvCache(cfg)
    layer = cache.new_layer()
    layer.k.fill_(0xFF), layer.v.fill_(0xFF), layer.k_scale.fill_(float("nan")), layer.v_scale.fill_(float("nan"))
    k, v = layer.k.cpu().numpy(), layer.v.cpu().numpy()
    ks, vs = layer.k_scale.cpu().numpy(), layer.v_scale.cpu().numpy()
    out = cache.alloc_step(cap)
    for step in range(9):
        keep = np.where(rng.random((W, B)) < 0.75, -1, rng.integers(0, 60, (W, B)))
        add = np.where(rng.random((W, B)) < 0.6, 1, rng.integers(0, 40, (W, B)))
        cache.step_device(_dev(keep, torch.int32), _dev(add, torch.int32), out)
        x = rng.normal(size=(2, W * cap, H, D)) * np.exp(rng.normal(size=(2, W * cap, H, 1)) * 2) * rng.choice([1.0, 1e-3, 50.0])
        x[:, rng.random(W * cap) < 0.05] = 0.0
        x[0, 3, 0, 1], x[1, 5, H - 1, 0], x[0, 40, 0, D - 1] = math.nan, math.inf, -math.inf
        if step == 4:
            x *= 1e-30 if dt != "float16" else 1e-4
        # keys and values as slices of one wider array, as a projection leaves them
        both = _dev(np.concatenate([x[0].reshape(W * cap, H * D), x[1].reshape(W * cap, H * D)], 1), _token_type(dt))
        xk, xv = both[:, :H * D].view(W * cap, H, D), both[:, H * D:].view(W * cap, H, D)
        cache.append_device(layer, xk, xv, out["slot"])
        slot = out["slot"].cpu().numpy()
        hk, hv = xk.double().cpu().numpy(), xv.double().cpu().numpy()
        for w in range(W):
            own = slice(w * N, (w + 1) * N)
            ko.append(k[own], ks[own], hk[w * cap:(w + 1) * cap], slot[w], b, fmt)
            ko.append(v.transpose(0, 1, 3, 2)[own], vs[own], hv[w * cap:(w + 1) * cap], slot[w], b, fmt)
        for name, got, ref in (("k_scale", layer.k_scale, ks), ("v_scale", layer.v_scale, vs)):
            assert np.array_equal(got.cpu().numpy(), ref, equal_nan=True), (case, step, name)
        # whole cache but what a NaN scale covers, where codes mean nothing
        for name, got, ref, s in (("k", layer.k, k, ks), ("v", layer.v, v, vs)):
            ok = np.isfinite(s)
            assert np.array_equal(got.cpu().numpy()[ok], ref[ok]), (case, step, name)
        # read: the rows' tokens, some slots twice, some outside the cache
        slots = np.concatenate([slot, np.array([[-1, N * b, -2 ** 31, 2 ** 31 - 1]] * W), slot[:, :11][:, ::-1], rng.integers(0, b, (W, 5))], 1).astype(np.int32)
        n = slots.shape[1]
        for t in (torch.float32, _token_type(dt)):
            rk, rv = torch.full((W * n, H, D), 7.0, dtype=t, device="cuda:0"), torch.full((H, W * n, D), 7.0, dtype=t, device="cuda:0").transpose(0, 1)
            cache.read_device(layer, _dev(slots), rk, rv)
            for got, codes, s, tr in ((rk, k, ks, False), (rv, v, vs, True)):
                want = np.zeros((W, n, H, D))
                for w in range(W):
                    for i in range(n):
                        at = int(slots[w, i])
                        if 0 <= at < N * b:
                            c = codes[w * N + at // b]
                            want[w, i] = ko.decode(c[:, :, at % b] if tr else c[:, at % b], fmt) * s[w * N + at // b][:, None].astype(np.float64)
                want = torch.tensor(want.reshape(W * n, H, D)).to(t)
                assert torch.equal(got.cpu().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0)), (case, step, t)
    cache.close()


def test_append_scales_that_are_no_powers_of_two_and_refusals():
    """Earlier tokens of a cache that was written elsewhere; scales of zero, below zero and infinite; lists of no tokens."""
    torch = _torch()
    import ctypes as C
    D, b, N = 64, 16, 12
    cache = kv.KvCache(kv.KvConfig(rows=2, block_tokens=b, n_blocks=N, max_blocks=4, head_dim=D, fmt="int8"))
    layer = cache.new_layer()
    rng = np.random.default_rng(1)
    layer.k.copy_(_dev(rng.integers(0, 256, (N, 1, b, D)), torch.uint8))
    layer.v.copy_(layer.k.transpose(2, 3))
    s = np.array([0.3, 0.5, 3.0, 0.0, -1.0, math.inf, 2.0 ** -100, 1e-38, 0.01, 100.0, 0.7, 1.0], np.float32)[:, None]
    layer.k_scale.copy_(_dev(s)), layer.v_scale.copy_(_dev(s))
    k, ks = layer.k.cpu().numpy(), s.copy()
    ks[4] = ks[5] = np.nan  # (no scales: the block reads as NaN from here on)
    x = rng.normal(size=(N, 1, D)).astype(np.float32) * 20
    slot = np.arange(N) * b + 5
    cache.append_device(layer, _dev(x), _dev(x), _dev(slot, torch.int32))
    ko.append(k, ks, x, slot, b, "int8")
    assert np.array_equal(layer.k_scale.cpu().numpy(), ks, equal_nan=True) and np.array_equal(layer.v_scale.cpu().numpy(), ks, equal_nan=True)
    ok = np.isfinite(ks[:, 0])
    assert ok.sum() == 10 and np.array_equal(layer.k.cpu().numpy()[ok], k[ok]) and np.array_equal(layer.v.transpose(2, 3).cpu().numpy()[ok], k[ok])
    none = torch.empty((0, 1, D), device="cuda:0")
    cache.append_device(layer, none, none, torch.empty(0, dtype=torch.int32, device="cuda:0"))
    lib, t = cache.lib, _dev(x)
    good = dict(k=t.data_ptr(), v=t.data_ptr(), slot=t.data_ptr(), k_token=D, k_head=D, v_token=D, v_head=D, n_tokens=N, dtype=2)
    for bad in (dict(k=None), dict(v=None), dict(slot=None), dict(n_tokens=-1), dict(dtype=3), dict(dtype=-1), dict(k=t.data_ptr() + 2), dict(slot=t.data_ptr() + 1)):
        a = kv._Tokens(**{**good, **bad})
        assert lib.br_kv_append(cache.ctx, layer.ref, C.byref(a)) == -1 and lib.br_kv_read(cache.ctx, layer.ref, C.byref(a)) == -1
    a = kv._Tokens(**good)
    for bad in (dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=layer.k.data_ptr() + 8)):
        l = kv._Layer(**{**{n: getattr(layer.struct, n) for n in ("k", "v", "k_scale", "v_scale")}, **bad})
        assert lib.br_kv_append(cache.ctx, C.byref(l), C.byref(a)) == -1
    q = torch.zeros((2, 1, D), dtype=torch.float16, device="cuda:0")
    good = dict(q=q.data_ptr(), out=q.data_ptr(), q_token=D, q_head=D, out_token=D, out_head=D, n_tokens=2, max_count=1, window=0, dtype=0, scale=1.0)
    for bad in (dict(q=None), dict(out=None), dict(n_tokens=-1), dict(max_count=0), dict(window=-1), dict(dtype=2), dict(scale=math.inf), dict(scale=math.nan),
                dict(start=q.data_ptr()), dict(count=q.data_ptr()), dict(q=q.data_ptr() + 1), dict(lse=q.data_ptr() + 2)):
        a = kv._Attention(**{**good, **bad})
        assert lib.br_kv_attend(cache.ctx, layer.ref, C.byref(a)) == -1
    a = kv._Attention(**{**good, "n_tokens": 0, "q": None})
    assert lib.br_kv_attend(cache.ctx, layer.ref, C.byref(a)) == 0
    cache.close()


# -- attention ------------------------------------------------------------------
def _cache_of(rng, fmt, W, R, b, D, H, group, lens, spread=1.0, M=None):
    """A cache with scattered blocks; memory that no token lives in holds what 8 bits can hold, codes of NaN among it, and NaN scales."""
    torch = _torch()
    need = max(1, int(max((-(-lens // b)).sum(1))))
    N, M = need + 3, M or max(1, int(max(-(-lens.max() // b), 1)) + 1)
    table = _scattered(rng, lens, b, N, M)
    k, v = rng.integers(0, 256, (W * N, H, b, D)).astype(np.uint8), rng.integers(0, 256, (W * N, H, D, b)).astype(np.uint8)
    ks, vs = np.full((W * N, H), np.nan, np.float32), np.full((W * N, H), np.nan, np.float32)
    for w in range(W):
        for r in range(R):
            for j in range(-(-int(lens[w, r]) // b)):
                i, n = w * N + table[w, r, j], min(b, int(lens[w, r]) - j * b)
                k[i, :, :n] = ko.encode(np.clip(rng.normal(size=(H, n, D)) * 40, -127, 127), fmt)
                v[i, :, :, :n] = ko.encode(np.clip(rng.normal(size=(H, D, n)) * 40, -127, 127), fmt)
                ks[i], vs[i] = np.exp(rng.normal(size=H) * 0.3) / 40, np.exp(rng.normal(size=H) * spread) / 40
    cfg = kv.KvConfig(n_workers=W, rows=R, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=H, n_q_heads=H * group, head_dim=D, fmt=fmt)
    cache = kv.KvCache(cfg, lens=_dev(lens, torch.int32), table=_dev(table))
    layer = cache.layer(_dev(k), _dev(v), _dev(ks), _dev(vs))
    return cache, layer, dict(k=k, v=v, ks=ks, vs=vs, table=table, N=N, M=M)


def _check_attention(tag, c, q, out, lse, ref, dt):
    o, l, A, S, Z = ref
    named = ~np.isnan(l)
    got, glse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    u = 2.0 ** -8 if dt == "bfloat16" else 2.0 ** -11
    wide = 2.0 ** -20 * (8 + S)
    tol = A * (2.0 ** -11 + wide[..., None]) + Z * 2.0 ** -32 + np.abs(np.nan_to_num(o)) * u + 2.0 ** -24 * (dt == "float16")
    if dt == "float16":  # beyond its range the result rounds to infinity
        over = named[..., None] & (np.abs(np.nan_to_num(o)) >= 65520 + tol)
        assert np.array_equal(got[over], np.sign(o[over]) * np.inf), (tag, "beyond f16")
        got, o = np.where(over, 0.0, got), np.where(over, 0.0, o)
    err = np.abs(got - o)
    bad = named[..., None] & ~(err <= tol)
    assert not bad.any(), (tag, "out", np.argwhere(bad)[:3], got[bad][:3], o[bad][:3], tol[bad][:3])
    seen = named & np.isfinite(l)
    assert np.array_equal(glse[named & ~seen], l[named & ~seen]), tag
    bad = seen & ~(np.abs(glse - np.where(seen, l, 0.0)) <= wide)
    assert not bad.any(), (tag, "lse", glse[bad][:3], l[bad][:3])


def _attend_case(tag, fmt, dt, D, H, group, b, lens, counts, window=0, spread=1.0, max_count=None, wide=True, scale=None, own=True, seed=0, qmul=1.0):
    """lens, counts [W][R]; query tokens in an order of their own with gaps between the rows."""
    torch = _torch()
    _say("attend", tag, fmt, dt, "D", D, "H", H, "group", group, "block", b, "rows", np.shape(lens), "longest", np.max(lens), "queries", np.max(counts), "window", window)
    rng = np.random.default_rng(seed + D + b)
    lens, counts = np.asarray(lens), np.asarray(counts)
    W, R = lens.shape
    cache, layer, h = _cache_of(rng, fmt, W, R, b, D, H, group, lens, spread)
    flat = counts.reshape(-1)
    order, start, at = rng.permutation(W * R), np.zeros(W * R, np.int64), 1
    for r in order:
        start[r] = at
        at += flat[r] + int(rng.integers(0, 2))
    T, pad = at + 1, 0 if wide else 1
    qs = torch.tensor(rng.normal(size=(T, H * group, D + pad)) * qmul, dtype=_token_type(dt), device="cuda:0")
    q = qs[:, :, pad:]
    out = torch.full((T, H * group, D + pad), 3.0, dtype=q.dtype, device="cuda:0")[:, :, pad:]
    lse = torch.full((T, H * group), 3.0, device="cuda:0")
    own_args = {}
    if not own:  # somebody else's tables
        own_args = dict(lens=_dev(lens, torch.int32), table=_dev(h["table"]))
        cache.lens.fill_(1), cache.table.fill_(-1)
    cache.attend_device(layer, q, out, lse=lse, start=_dev(start.reshape(W, R), torch.int32), count=_dev(counts, torch.int32),
                        max_count=max_count or max(1, int(counts.max())), window=window, scale=scale, **own_args)
    hq = q.double().cpu().numpy()
    parts = []
    for w in range(W):
        own_blocks = slice(w * h["N"], (w + 1) * h["N"])
        sl = slice(w * R, (w + 1) * R)
        parts.append(ko.attend(hq, h["k"][own_blocks], h["v"][own_blocks], h["ks"][own_blocks], h["vs"][own_blocks], h["table"][w], lens[w], start[sl], flat[sl], group, b, fmt,
                               window=window, scale=scale))
    ref = list(parts[0])
    for o, l, A, S, Z in parts[1:]:
        m = ~np.isnan(l)
        ref[1] = np.where(m, l, ref[1])
        ref[0] = np.where(m[..., None], o, ref[0])
        ref[2], ref[3], ref[4] = ref[2] + A, ref[3] + S, ref[4] + Z
    _check_attention(tag, cache, q, out, lse, ref, dt)
    untouched = np.isnan(ref[1])
    assert (out.float().cpu().numpy()[untouched] == 3.0).all() and (lse.cpu().numpy()[untouched] == 3.0).all(), tag
    cache.close()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("b", [16, 32, 64, 128])
def test_attention_single_tokens(fmt, D, b):
    """Every head width and block size; lengths about the tiles' and blocks' ends, one, and none."""
    lens = [[0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 511, 1000, 1025]]
    _attend_case("single", fmt, "bfloat16" if b in (16, 64) else "float16", D, 2, 4, b, lens, [[1] * 16])


@pytest.mark.parametrize("case", [
    # H, group, lens, counts, window
    (1, 1, [[700, 3, 64]], [[1, 1, 1]], 0), (3, 7, [[33, 900, 260, 5]], [[4, 4, 4, 4]], 0), (2, 16, [[257, 70]], [[1, 1]], 0), (1, 17, [[257, 70]], [[1, 1]], 0),
    (2, 5, [[400, 90, 12]], [[13, 2, 0]], 0), (2, 4, [[333, 64, 500]], [[40, 64, 1]], 0), (1, 8, [[300, 1, 150]], [[300, 1, 150]], 0), (2, 3, [[131, 700]], [[70, 90]], 50),
    (1, 1, [[5, 3, 0, 40]], [[9, 3, 4, 41]], 0), (2, 2, [[1000, 64, 65, 100]], [[1, 1, 1, 2]], 1), (2, 2, [[1000, 640, 65]], [[3, 5, 2]], 64), (1, 6, [[2000]], [[30]], 200),
    (2, 4, [[100, 0, 77], [0, 0, 0], [640, 65, 1]], [[1, 0, 2], [0, 1, 3], [5, 1, 1]], 0), (1, 64, [[500]], [[3]], 0), (40, 1, [[70, 200]], [[1, 2]], 0)], ids=str)
@pytest.mark.parametrize("fmt,dt", [("int8", "float16"), ("fp8", "bfloat16")])
def test_attention_queries(case, fmt, dt):
    H, group, lens, counts, window = case
    _attend_case("queries", fmt, dt, 64, H, group, 16, lens, counts, window=window)
    if H < 5:
        _attend_case("queries", fmt, dt, 128, H, group, 32, lens, counts, window=window, own=False)


@pytest.mark.parametrize("D", [96, 192, 256])
@pytest.mark.parametrize("fmt,dt", [("fp8", "float16"), ("int8", "bfloat16")])
def test_attention_queries_of_wide_heads(D, fmt, dt):
    _attend_case("wide", fmt, dt, D, 2, 4, 16, [[200, 31, 650]], [[7, 3, 12]])
    _attend_case("wide", fmt, dt, D, 1, 4, 64, [[200, 31, 650]], [[150, 3, 60]], window=90)


def test_attention_many_rows_and_long_ones():
    """Rows beyond a thread's one each; one row whose tokens all blocks of the launch share; a few long beside many short."""
    rng = np.random.default_rng(8)
    _attend_case("many", "int8", "bfloat16", 64, 1, 2, 16, rng.integers(0, 90, (3, 500)), rng.integers(0, 3, (3, 500)))
    _attend_case("long", "fp8", "bfloat16", 128, 1, 4, 64, [[100001]], [[1]])
    _attend_case("long", "int8", "float16", 64, 2, 2, 128, [[60000, 1, 0, 17, 300]], [[3, 1, 1, 1, 1]])
    _attend_case("mixed", "fp8", "float16", 128, 2, 8, 16, [[9000] + [20] * 60], [[1] * 61])
    _attend_case("hint", "int8", "bfloat16", 64, 1, 4, 16, [[400, 90]], [[50, 60]], max_count=1)


def test_attention_of_unaligned_views_and_extremes():
    """Queries and outputs that cannot be read 16 bytes at a time; scales of the values over 60 binary orders; sharp and flat scores."""
    for fmt in ("int8", "fp8"):
        _attend_case("unaligned", fmt, "bfloat16", 96, 2, 3, 32, [[77, 300]], [[2, 1]], wide=False)
        _attend_case("spread", fmt, "float16", 64, 2, 2, 16, [[500, 40]], [[1, 2]], spread=6.0, seed=3)
        _attend_case("sharp", fmt, "bfloat16", 128, 1, 4, 16, [[500, 40]], [[1, 2]], qmul=30.0)
        _attend_case("flat", fmt, "float16", 128, 1, 4, 16, [[700, 40]], [[1, 2]], scale=0.0)
        _attend_case("negative", fmt, "bfloat16", 64, 1, 4, 16, [[700, 40]], [[1, 2]], scale=-0.5)
        _attend_case("tiny queries", fmt, "bfloat16", 64, 1, 4, 16, [[70, 40]], [[1, 2]], qmul=1e-30)


def test_attention_of_what_is_not_finite():
    """A NaN scale of keys or values, a NaN or infinite query: NaN in the rows and heads that see it, and nowhere else."""
    torch = _torch()
    rng = np.random.default_rng(2)
    W, R, b, D, H, group = 1, 5, 16, 64, 2, 2
    lens = np.array([[100, 50, 100, 100, 64]])
    cache, layer, h = _cache_of(rng, "fp8", W, R, b, D, H, group, lens)
    clean = torch.tensor(rng.normal(size=(R, H * group, D)), dtype=torch.bfloat16, device="cuda:0")
    out0, out = torch.empty_like(clean), torch.empty_like(clean)
    cache.attend_device(layer, clean, out0, window=40)
    q = clean.clone()
    q[3, 0, 5], q[3, 3, 0] = math.nan, math.inf
    layer.k_scale[h["table"][0, 0, 6], 1] = math.nan   # seen by row 0's head 1
    layer.v_scale[h["table"][0, 2, 5], 0] = math.nan   # seen by row 2's head 0
    layer.v_scale[h["table"][0, 4, 0], 0] = math.nan   # behind row 4's window
    layer.k_scale[h["table"][0, 4, 1], 1] = math.nan   # ... which ends at this block's middle: token 24 is the first seen
    cache.attend_device(layer, q, out, window=40)
    nan = torch.isnan(out.float())
    want = torch.zeros_like(nan)
    want[0, 2:], want[2, :2], want[3, 0], want[3, 3], want[4, 2:] = True, True, True, True, True
    assert torch.equal(nan, want)
    assert torch.equal(out[~want], out0[~want])
    cache.close()


def test_attention_bounds_of_what_it_reads_on_the_device():
    """Block ids, lengths, starts and counts out of range: tokens without a block are not seen, tokens outside the list not written."""
    torch = _torch()
    rng = np.random.default_rng(4)
    b, D, H, group = 16, 64, 1, 2
    lens = np.array([[100, 50, 30, 20]])
    cache, layer, h = _cache_of(rng, "int8", 1, 4, b, D, H, group, lens)
    table = h["table"].copy()
    table[0, 0, 1], table[0, 0, 4], table[0, 1, :4], table[0, 2, 0] = -1, 10 ** 9, h["N"], -2 ** 31
    said = np.array([[100, 50, 30, 10 ** 9]])  # the last row's table ends before: -1 from its third block on
    start, count = np.array([[0, 2, -1, 7]]), np.array([[2, 1, 3, 1]])
    q = torch.tensor(rng.normal(size=(8, H * group, D)), dtype=torch.float16, device="cuda:0")
    out, lse = torch.full_like(q, 3.0), torch.full((8, H * group), 3.0, device="cuda:0")
    cache.attend_device(layer, q, out, lse=lse, start=_dev(start, torch.int32), count=_dev(count, torch.int32), max_count=3, lens=_dev(said, torch.int32), table=_dev(table))
    # rows 0 and 2 name token 0 and 1 both: row 2 is checked alone
    ref = ko.attend(q.double().cpu().numpy(), h["k"], h["v"], h["ks"], h["vs"], table[0], said[0], start[0], [0, 1, 0, 1], group, b, "int8")
    assert ref[1][2, 0] == -math.inf and np.isfinite(ref[1][7]).all()
    named = [2, 7]
    _check_attention("bounds", cache, q, out[named], lse[named], [x[named] for x in ref], "float16")
    out.fill_(3.0), lse.fill_(3.0)
    count = np.array([[0, -5, 3, 2]])
    cache.attend_device(layer, q, out, lse=lse, start=_dev(start, torch.int32), count=_dev(count, torch.int32), max_count=1, lens=_dev(said, torch.int32), table=_dev(table))
    ref = ko.attend(q.double().cpu().numpy(), h["k"], h["v"], h["ks"], h["vs"], table[0], said[0], start[0], [0, 0, 3, 2], group, b, "int8")
    named = [0, 1, 7]
    _check_attention("bounds", cache, q, out[named], lse[named], [x[named] for x in ref], "float16")
    assert bool((out[2:7] == 3.0).all()) and bool((lse[2:7] == 3.0).all())
    cache.close()


# -- together ---------------------------------------------------------------------
def test_a_step_as_a_graph():
    """Tables, write and attention captured once and replayed with other inputs, eager work between the replays, against eager calls; two runs of
    the same inputs are equal bit for bit."""
    torch = _torch()
    B, b, N, M, H, group, D, cap = 20, 16, 400, 40, 2, 4, 128, 300
    cfg = kv.KvConfig(rows=B, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=H, n_q_heads=H * group, head_dim=D, fmt="fp8")
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(11)
    with torch.cuda.stream(stream):
        both = [kv.KvCache(cfg, stream=stream) for _ in range(2)]
        layers = [c.new_layer() for c in both]
        steps = [c.alloc_step(cap) for c in both]
        keep, add = torch.zeros((1, B), dtype=torch.int32, device="cuda:0"), torch.zeros((1, B), dtype=torch.int32, device="cuda:0")
        x = torch.zeros((2, cap, H, D), dtype=torch.bfloat16, device="cuda:0")
        q = torch.zeros((cap, H * group, D), dtype=torch.bfloat16, device="cuda:0")
        outs = [torch.zeros_like(q) for _ in range(2)]

        def call(i):
            both[i].step_device(keep, add, steps[i])
            both[i].append_device(layers[i], x[0], x[1], steps[i]["slot"])
            both[i].attend_device(layers[i], q, outs[i], start=steps[i]["start"], count=steps[i]["count"], max_count=30)

        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(0)
        for k in range(6):
            keep.copy_(torch.as_tensor(np.where(rng.random((1, B)) < 0.8, -1, 0), dtype=torch.int32))
            add.copy_(torch.as_tensor(np.where(rng.random((1, B)) < 0.6, 1, rng.integers(0, 30, (1, B))), dtype=torch.int32))
            x.copy_(torch.as_tensor(rng.normal(size=x.shape)))
            q.copy_(torch.as_tensor(rng.normal(size=q.shape)))
            graph.replay()
            call(1)
            stream.synchronize()
            assert all(torch.equal(steps[0][n], steps[1][n]) for n in steps[0]), k
            assert torch.equal(both[0].table, both[1].table)
            assert torch.equal(outs[0], outs[1]), k
            outs[0].mul_(0)
            outs[1].mul_(0)
    for c in both:
        c.close()


def test_offsets_beyond_32_bits():
    """A cache of 9 GB: the last blocks' codes lie beyond 4 GB in both arrays."""
    torch = _torch()
    D, H, b, N = 256, 8, 128, 17000
    cache = kv.KvCache(kv.KvConfig(rows=2, block_tokens=b, n_blocks=N, max_blocks=4, n_kv_heads=H, n_q_heads=H, head_dim=D, fmt="int8"),
                       lens=torch.zeros((1, 2), dtype=torch.int32, device="cuda:0"), table=torch.full((1, 2, 4), -1, dtype=torch.int32, device="cuda:0"))
    layer = cache.new_layer()
    rng = np.random.default_rng(6)
    table = np.full((1, 2, 4), -1, np.int32)
    table[0, 0, :2], table[0, 1, :1] = [N - 1, 3], [N - 2]
    lens = np.array([[200, 90]])
    slot = np.concatenate([(N - 1) * b + np.arange(128), 3 * b + np.arange(72), (N - 2) * b + np.arange(90)]).astype(np.int32)
    x = torch.tensor(rng.normal(size=(2, 290, H, D)), dtype=torch.float16, device="cuda:0")
    cache.append_device(layer, x[0], x[1], _dev(slot))
    back = torch.empty_like(x)
    cache.read_device(layer, _dev(slot), back[0], back[1])
    assert (back - x).abs().max().item() < 0.05
    q = torch.tensor(rng.normal(size=(2, H, D)), dtype=torch.float16, device="cuda:0")
    out = torch.empty_like(q)
    cache.attend_device(layer, q, out, lens=_dev(lens, torch.int32), table=_dev(table))
    for r, rows in enumerate((slice(0, 200), slice(200, 290))):
        k, v = back[0, rows].double().cpu(), back[1, rows].double().cpu()
        w = torch.softmax(torch.einsum("hd,thd->ht", q[r].double().cpu(), k) / 16.0, 1)
        ref = torch.einsum("ht,thd->hd", w, v)
        assert ((out[r].double().cpu() - ref).abs().max() < 2e-3).item()
    cache.close()


@pytest.mark.parametrize("fmt,policy", [("fp8", False), ("int8", True)])
def test_routed_requests_on_their_workers(fmt, policy):
    """The example: the router's loads are the workers' cached tokens in every step (it compares them itself)."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_workers.py")
    spec = importlib.util.spec_from_file_location("decode_workers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    log = example.run(steps=40, fmt=fmt, policy=policy, block=16 if policy else 32)
    assert len(log) == 40 and max(r["requests"] for r in log) > 20
