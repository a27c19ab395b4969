"""What a query does not see has no part in its attention, and neither does how the scales of what it sees are spread, on the GPU.

Against 64 bits.  The bound is `test_kv_gpu`'s but for the weights e^(s - m) v_scale in f16: each is off by 2^-11 of itself at most, and by 2^-33 of the
largest that the query sees."""
import math

import numpy as np
import pytest

from tests import kv_oracle as ko
from tests.test_kv_gpu import _cache_of, _dev, _say, _token_type, _torch

pytestmark = pytest.mark.gpu


def _largest_weights(q, h, lens, start, count, group, block, fmt, window, scale):
    """[T, Hq, D]: the largest seen weight times v_scale over the sum of the weights, times the sums of the seen codes' magnitudes."""
    T, Hq, D = q.shape
    H = Hq // group
    P = np.zeros((T, Hq, D))
    for r in range(len(lens)):
        L = int(lens[r])
        ids = h["table"][0][r][:-(-L // block)].astype(np.int64)
        k = (ko.decode(h["k"][ids], fmt) * h["ks"][ids].astype(np.float64)[:, :, None, None]).transpose(1, 0, 2, 3).reshape(H, -1, D)[:, :L]
        code = np.abs(ko.decode(h["v"][ids], fmt)).transpose(1, 0, 3, 2).reshape(H, -1, D)[:, :L]
        vs = np.repeat(h["vs"][ids].astype(np.float64), block, 0)[:L]
        for i in range(int(count[r])):
            t, p = int(start[r]) + i, L - int(count[r]) + i
            see = slice(max(0, p - window + 1) if window else 0, max(p + 1, 0))
            for hq in range(Hq):
                if see.stop <= see.start:
                    continue
                s = scale * (k[hq // group][see] @ q[t, hq].astype(np.float64))
                w = np.exp(s - s.max())
                P[t, hq] = (w * vs[see, hq // group]).max() / w.sum() * code[hq // group][see].sum(0)
    return P


def _run(h, cache, layer, q, lens, start, count, window=0, scale=None):
    torch = _torch()
    layer.k.copy_(_dev(h["k"])), layer.v.copy_(_dev(h["v"])), layer.k_scale.copy_(_dev(h["ks"])), layer.v_scale.copy_(_dev(h["vs"]))
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda:0")
    cache.attend_device(layer, q, out, lse=lse, start=_dev(start[None], torch.int32), count=_dev(count[None], torch.int32), max_count=int(count.max()), window=window, scale=scale)
    return out, lse


def _check(tag, h, q, out, lse, lens, start, count, group, block, fmt, window=0, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    hq = q.double().cpu().numpy()
    o, l, A, S, _ = ko.attend(hq, h["k"], h["v"], h["ks"], h["vs"], h["table"][0], lens, start, count, group, block, fmt, window=window, scale=scale)
    P = _largest_weights(hq, h, lens, start, count, group, block, fmt, window, scale)
    wide = 2.0 ** -20 * (8 + S)
    tol = A * (2.0 ** -11 + wide[..., None]) + P * 2.0 ** -33 * (1 + wide[..., None]) + np.abs(o) * 2.0 ** -8
    err = np.abs(out.double().cpu().numpy() - o)
    bad = ~(err <= tol)
    assert not bad.any(), (tag, np.argwhere(bad)[:3], out.double().cpu().numpy()[bad][:3], o[bad][:3], tol[bad][:3])
    seen = np.isfinite(l)
    assert (np.abs(lse.double().cpu().numpy() - np.where(seen, l, 0.0)) <= wide)[seen].all(), tag


CHUNKS = [(2, 1), (9, 4), (70, 2), (40, 16)]  # query tokens of a row, group: tiles of 16, 64 and 128 rows of queries


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("chunk", CHUNKS, ids=str)
def test_scales_of_what_others_see(fmt, D, chunk):
    """Blocks that only some queries of a tile see have value scales 2^20 to 2^60 of the others': the last ones of a chunk, and the first ones
    of a window.  Right for everybody, and bit for bit the same for who does not see them."""
    torch = _torch()
    n, group = chunk
    b, H = 16, 2
    _say("others", fmt, D, n, group)
    rng = np.random.default_rng(D + n)
    lens = np.array([200, 5 * 16 + n // 2 + 1, 331])
    count, start = np.array([n, n, n]), np.array([0, n, 2 * n])
    cache, layer, h = _cache_of(rng, fmt, 1, 3, b, D, H, group, lens[None])
    q = torch.tensor(rng.normal(size=(3 * n, H * group, D)), dtype=torch.bfloat16, device="cuda:0")
    own = h["vs"].copy()
    for window in (0, 70):
        h["vs"] = own.copy()
        clean, clean_lse = _run(h, cache, layer, q, lens, start, count, window)
        for ratio in (20, 26, 30, 34, 60):
            # the block of each row's last token; with a window, the block of the first token of the first query's
            at = [h["table"][0, r, (lens[r] - 1 if not window else max(0, lens[r] - n - window + 1)) // b] for r in range(3)]
            h["vs"] = own.copy()
            h["vs"][at] *= 2.0 ** ratio
            out, lse = _run(h, cache, layer, q, lens, start, count, window)
            _check((fmt, D, chunk, window, ratio), h, q, out, lse, lens, start, count, group, b, fmt, window)
            for r in range(3):
                p = lens[r] - n + np.arange(n)
                first = (lens[r] - 1 if not window else max(0, lens[r] - n - window + 1)) // b * b
                blind = torch.tensor(start[r] + np.flatnonzero(p < first if not window else p - window >= first + b - 1), device="cuda:0", dtype=torch.long)
                assert torch.equal(out[blind], clean[blind]) and torch.equal(lse[blind], clean_lse[blind]), (window, ratio, r)
    cache.close()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("n,group,D", [(1, 1, 64), (2, 7, 128), (3, 16, 256), (80, 2, 128), (66, 2, 192)])
def test_scales_of_tokens_that_hardly_count(fmt, n, group, D):
    """Tokens with next to no weight and value scales 2^10 to 2^120 of the others', before and behind them; scales that fall as the scores
    rise, and the other way round; the least and the largest scales there are."""
    torch = _torch()
    _say("hardly", fmt, n, group, D)
    rng = np.random.default_rng(D + n)
    b, H, blocks = 16, 1, 21
    lens, count, start = np.array([blocks * b - 3]), np.array([n]), np.array([0])
    cache, layer, h = _cache_of(rng, fmt, 1, 1, b, D, H, group, lens[None])
    # a query's first channel and a block's keys' first channel give the block its score: `step` a code
    q = torch.tensor(rng.normal(size=(n, H * group, D)) * 0.002, dtype=torch.bfloat16, device="cuda:0")
    q[:, :, 0] = 1.0
    ids = h["table"][0, 0, :blocks]
    h["ks"][ids] = 1.0
    j = np.arange(blocks)
    cases = []
    for score, e in (
            (np.where(j == 0, -60, 0), np.where(j == 0, 40, 0)), (np.where(j == 20, -60, 0), np.where(j == 20, 60, 0)),
            (np.where(j % 7 == 3, -80, 0), np.where(j % 7 == 3, 70, -30)), (np.where(j % 5 == 0, -20, 0), np.where(j % 5 == 0, 10, 0)),
            (3 * j - 60, -6 * j), (60 - 3 * j, 6 * j), (4 * j - 80, 60 - 6 * j), (0 * j, 6 * j - 60), (0 * j, 60 - 6 * j),
            (np.where(j == 2, -80, 0), np.where(j == 2, 120, 0)), (0 * j, 0 * j - 100), (0 * j, 0 * j + 115)):
        cases.append((score, e))
    for score, e in cases:
        h["k"][ids, 0, :, 0] = ko.encode(np.clip(score.astype(np.float64), -112, 112)[:, None] * np.ones((1, b)), fmt)
        h["vs"][ids] = (2.0 ** e.astype(np.float64)).astype(np.float32)[:, None]
        out, lse = _run(h, cache, layer, q, lens, start, count, scale=1.0)
        _check((fmt, n, group, D, score.tolist(), e.tolist()), h, q, out, lse, lens, start, count, group, b, fmt, scale=1.0)
    cache.close()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("n,group,D", [(1, 1, 64), (2, 7, 128), (70, 2, 128)])
def test_scores_beyond_what_32_bits_tell_apart(fmt, n, group, D):
    """Scores of 2^24 to 2^40, thousands apart, at scales that are no powers of two: the token with the largest has all of the weight."""
    torch = _torch()
    rng = np.random.default_rng(D + n)
    b, L = 16, 333
    lens, count, start = np.array([L]), np.array([n]), np.array([0])
    cache, layer, h = _cache_of(rng, fmt, 1, 1, b, D, 1, group, lens[None])
    ids = h["table"][0, 0, :-(-L // b)]
    h["ks"][ids], h["vs"][ids] = 1.0 / 3.0, (1.0 / 3.0 * np.exp(rng.normal(size=len(ids)) * 0.5))[:, None]
    for e in (18, 26, 34):
        q = torch.zeros(n, group, D, dtype=torch.bfloat16, device="cuda:0")
        q[:, :, 0] = 2.0 ** e
        for best in (3, 100, L - n):  # (seen by all)
            code = rng.integers(-100, 80, (len(ids), 1, b)).astype(np.float64)
            code[best // b, 0, best % b] = 96
            h["k"][ids, :, :, 0] = ko.encode(code, fmt)
            out, lse = _run(h, cache, layer, q, lens, start, count, scale=1.0)
            want = ko.decode(h["v"][ids[best // b], 0, :, best % b], fmt) * float(h["vs"][ids[best // b], 0])
            err = np.abs(out.double().cpu().numpy() - want)
            assert (err <= np.abs(want) * (2.0 ** -8 + 2.0 ** -10)).all(), (fmt, n, e, best)
            assert (np.abs(lse.double().cpu().numpy() / (2.0 ** e * 32) - 1) < 2.0 ** -20).all()
    cache.close()
