"""Calls on both sides of the rules by which the worker's kernels divide their work, and scales that are none, on the GPU.

Tables, codes and what is read back have to be equal; attention as `test_kv_gpu` states."""
import math

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests import kv_oracle as ko, test_kv_gpu
from tests.test_kv_gpu import _attend_case, _cache_of, _dev, _say, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [
    # rows of lens, their query tokens, group, window: query tiles of 128 rows
    ([3100], [3000], 4, 0),                              # more query tiles in a row than lanes
    ([3100, 40], [2500, 3], 7, 900),
    ([70] * 199 + [900], [1] * 199 + [700], 2, 0),       # a chunk behind as many rows as a block has threads, nearly
    ([40] * 128 + [600, 1], [2] * 128 + [500, 1], 3, 0),
    ([33] * 400 + [500], [1] * 400 + [300], 4, 0),       # more rows than threads
    ([9000, 8000], [20, 25], 8, 0)], ids=lambda c: "%d rows, %d queries" % (len(c[0]), sum(c[1])))
@pytest.mark.parametrize("fmt,dt,D", [("int8", "bfloat16", 64), ("fp8", "float16", 128)])
def test_attention_of_chunks(case, fmt, dt, D):
    lens, counts, group, window = case
    _attend_case("chunks", fmt, dt, D, 1, group, 32, [lens], [counts], window=window)


def test_attention_of_chunks_of_wide_heads():
    for D in (192, 256):
        _attend_case("chunks", "fp8", "float16", D, 1, 5, 128, [[5000, 300, 7]], [[90, 60, 1]])


READS = [  # rows, tokens a row, block, heads, D
    (5, 600, 128, 4, 256),   # short list, long rows: pieces by blocks
    (3, 333, 16, 2, 96),
    (100, 9, 16, 3, 64),     # short list, short rows: pieces by waves
    (40, 16, 128, 8, 128),
    (1, 1, 32, 1, 192),
    (60, 700, 64, 1, 64),    # long lists
    (300, 60, 32, 5, 96),
    (4000, 4, 16, 2, 64), (4000, 1, 16, 3, 128)]


@pytest.mark.parametrize("fmt,dt", [("int8", "bfloat16"), ("fp8", "float32")])
@pytest.mark.parametrize("case", READS, ids=str)
def test_tokens_in_and_out(case, fmt, dt):
    """Lists that begin and end inside blocks, with gaps; slots in order, and in an order that has no runs."""
    torch = _torch()
    R, n, b, H, D = case
    W = max(1, R // 1000)
    R //= W
    _say("tokens", case, fmt, dt)
    rng = np.random.default_rng(R + n)
    per = -(-(n + b) // b)
    N = R * per
    cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=R, block_tokens=b, n_blocks=N, max_blocks=per, n_kv_heads=H, n_q_heads=H, head_dim=D, fmt=fmt))
    layer = cache.new_layer()
    slot = []
    for w in range(W):
        ids, one = rng.permutation(N).reshape(R, per), []
        for r in range(R):
            p = int(rng.integers(0, b)) + np.arange(int(rng.integers(max(1, n // 2), n + 1)))
            one += list(ids[r, p // b] * b + p % b) + [-1] * int(rng.integers(0, 3))
        slot.append((one + [-1] * (R * (n + 3)))[:R * (n + 3)])
    slot = np.array(slot, np.int32)
    T = slot.shape[1]
    x = torch.tensor(rng.normal(size=(2, W * T, H, D)), dtype=getattr(torch, dt), device="cuda:0")
    k, v = (rng.integers(0, 256, t.shape).astype(np.uint8) for t in (layer.k, layer.v))  # earlier tokens' codes, of blocks that lists begin inside of
    ks, vs = np.full((W * N, H), 2.0 ** -9, np.float32), np.full((W * N, H), 2.0 ** -9, np.float32)
    for t, a in ((layer.k, k), (layer.v, v), (layer.k_scale, ks), (layer.v_scale, vs)):
        t.copy_(torch.tensor(a))
    # ... which may hold codes of NaN here: what those become is not said
    written = np.zeros((W * N, b), bool)
    for w in range(W):
        s = slot[w][slot[w] >= 0]
        written[w * N + s // b, s % b] = True
    said_k = written[:, None, :, None] | (fmt == "int8") | ((k & 127) != 127)
    said_v = written[:, None, None, :] | (fmt == "int8") | ((v & 127) != 127)
    cache.append_device(layer, x[0], x[1], _dev(slot))
    hx = x.double().cpu().numpy().reshape(2, W, T, H, D)
    for w in range(W):
        own = slice(w * N, (w + 1) * N)
        ko.append(k[own], ks[own], hx[0, w], slot[w], b, fmt)
        ko.append(v.transpose(0, 1, 3, 2)[own], vs[own], hx[1, w], slot[w], b, fmt)
    for got, want, said in ((layer.k, k, said_k), (layer.v, v, said_v), (layer.k_scale, ks, True), (layer.v_scale, vs, True)):
        assert ((got.cpu().numpy() == want) | ~np.asarray(said)).all(), case
    for order in (np.arange(T), rng.permutation(T)):
        at = slot[:, order]
        out = torch.full((2, W * T, H, D), 7.0, dtype=x.dtype, device="cuda:0")
        cache.read_device(layer, _dev(at), out[0], out[1])
        ids, off, ok = np.where(at < 0, 0, at) // b + np.arange(W)[:, None] * N, np.where(at < 0, 0, at) % b, at >= 0
        for got, codes, s in ((out[0], k, ks), (out[1], v.transpose(0, 1, 3, 2), vs)):
            want = np.where(ok[..., None, None], ko.decode(codes[ids, :, off], fmt) * s[ids][..., None].astype(np.float64), 0.0)
            assert torch.equal(got.cpu(), torch.tensor(want.reshape(W * T, H, D)).to(x.dtype)), case
    cache.close()


@pytest.mark.parametrize("none", [-1.0, -0.5, math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("chunk", [1, 70])
def test_scales_that_are_none(none, chunk):
    """Below zero or not finite: NaN to who sees the block, in reads and attention, and nothing to anybody else."""
    torch = _torch()
    rng = np.random.default_rng(6)
    R, b, D, H, group = 4, 16, 64, 2, 2
    lens = np.array([[200, 90, 128, 70]])
    cache, layer, h = _cache_of(rng, "int8", 1, R, b, D, H, group, lens)
    q = torch.tensor(rng.normal(size=(R * chunk, H * group, D)), dtype=torch.float16, device="cuda:0")
    start, count = _dev(np.arange(R)[None] * chunk, torch.int32), _dev(np.full((1, R), chunk), torch.int32)
    a = dict(start=start, count=count, max_count=chunk, window=40)
    out0, out = torch.empty_like(q), torch.empty_like(q)
    cache.attend_device(layer, q, out0, **a)
    layer.k_scale[h["table"][0, 0, 12], 1] = none  # tokens 192 ..: row 0's last 8 positions
    layer.v_scale[h["table"][0, 2, 7], 0] = none   # tokens 112 ..: row 2's last 16
    layer.v_scale[h["table"][0, 1, 0], 0] = none   # tokens 0 .. 15: behind the window of all queries of row 1 at positions from 55 on
    cache.attend_device(layer, q, out, **a)
    want = torch.zeros(R, chunk, H, dtype=torch.bool, device="cuda:0")
    pos = torch.arange(chunk, device="cuda:0")
    want[0, pos + 200 - chunk >= 192, 1] = True
    want[2, pos + 128 - chunk >= 112, 0] = True
    want[1, (pos + 90 - chunk) - 40 < 15, 0] = True
    want = want.reshape(R * chunk, H, 1, 1).expand(-1, H, group, D).reshape(R * chunk, H * group, D)
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(out[~want], out0[~want])
    slot = torch.tensor([int(h["table"][0, 0, 12]) * b, int(h["table"][0, 2, 7]) * b + 3, int(h["table"][0, 3, 0]) * b], dtype=torch.int32, device="cuda:0")
    k, v = torch.empty(2, 3, H, D, device="cuda:0")
    cache.read_device(layer, slot, k, v)
    for x, bad in ((k, {(0, 1)}), (v, {(1, 0)})):
        for t in range(3):
            for g in range(H):
                assert bool(torch.isnan(x[t, g]).all()) == ((t, g) in bad) and bool(torch.isnan(x[t, g]).any()) == ((t, g) in bad)
    cache.close()


def test_tokens_too_far_apart_are_refused():
    """Token strides of 2^23 elements and more: offsets inside a run have 32 bits."""
    torch = _torch()
    cache = kv.KvCache(kv.KvConfig(rows=2, n_blocks=4, max_blocks=2, n_kv_heads=2, n_q_heads=2, head_dim=64))
    layer = cache.new_layer()
    far, near = torch.zeros(2, 2 ** 23, dtype=torch.float16, device="cuda:0")[:, :128].view(2, 2, 64), torch.zeros(2, 2, 64, dtype=torch.float16, device="cuda:0")
    slot = torch.zeros(2, dtype=torch.int32, device="cuda:0")
    for k, v in ((far, near), (near, far)):
        with pytest.raises(kv.BrError):
            cache.append_device(layer, k, v, slot)
        with pytest.raises(kv.BrError):
            cache.read_device(layer, slot, k, v)
    cache.append_device(layer, near, near, slot)
    cache.close()


@pytest.mark.parametrize("case", [(5, 40, 16, 900, 60, 4099, 900), (3, 300, 32, 600, 40, 4097, 600), (4, 512, 16, 3000, 100, 8190, 700), (2, 513, 64, 1100, 30, 9001, 900),
                                  (7, 9, 16, 2100, 300, 4095, 4000), (3, 257, 128, 700, 9, 3, 500)], ids=str)
def test_token_lists_of_odd_lengths(case):
    """Several workers' lists side by side, none but the first at 16 bytes; both sides of the step's own lists and of rows to a thread."""
    test_kv_gpu.test_tables(case)
