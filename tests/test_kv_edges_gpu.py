"""Calls at the limits of what include/br_kv.h allows, on the GPU: windows, strides, scales, lists that name a block twice, streams."""
import weakref

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests import kv_oracle as ko
from tests.test_kv_gpu import _attend_case, _dev, _say, _scattered, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30, 2 ** 20 + 1, 2 ** 20, 129, 128])
@pytest.mark.parametrize("group", [1, 4])
def test_windows_that_hide_nothing(window, group):
    """Up to the largest number that fits, with rows of fewer tokens than queries: whoever is there sees all tokens up to itself."""
    lens, counts = [[20, 3, 40, 0, 100]], [[30, 9, 2, 3, 4]]  # (tables of 8 blocks of 16 tokens)
    _attend_case("window", "int8", "float16", 64, 2, group, 16, lens, counts, window=window)
    _attend_case("window", "fp8", "bfloat16", 128, 1, group, 16, lens, counts, window=window)


@pytest.mark.parametrize("fmt,D,b,H", [("int8", 128, 64, 3), ("fp8", 256, 128, 2), ("int8", 64, 16, 1), ("fp8", 96, 32, 4)])
def test_lists_that_name_a_block_twice(fmt, D, b, H):
    """What such a block then holds is not said; all others hold what they would without it."""
    torch = _torch()
    _say("twice", fmt, D, b, H)
    rng = np.random.default_rng(D)
    N = 60
    cache = kv.KvCache(kv.KvConfig(rows=2, block_tokens=b, n_blocks=N, max_blocks=N, n_kv_heads=H, n_q_heads=H, head_dim=D, fmt=fmt))
    layer = cache.new_layer()
    k = ko.encode(rng.integers(-110, 111, (N, H, b, D)).astype(np.float64), fmt)
    s = np.exp2(rng.integers(-12, 3, (N, H))).astype(np.float32)
    layer.k.copy_(_dev(k)), layer.v.copy_(layer.k.transpose(2, 3)), layer.k_scale.copy_(_dev(s)), layer.v_scale.copy_(_dev(s))
    slot = []
    for i in rng.permutation(N - 2):  # blocks N - 2 and N - 1: again and again, from offsets inside them, between all others
        off = int(rng.integers(0, b - 3))
        slot += list(i * b + np.arange(off, b if rng.random() < 0.5 else off + 3))
        off = int(rng.integers(1, b - 3))
        slot += list((N - 1 - int(rng.integers(0, 2))) * b + np.arange(off, b))
    slot = np.array(slot, np.int32)
    T = len(slot)
    x = (rng.normal(size=(T, H, D)) * np.exp(rng.normal(size=(T, 1, 1)) * 3)).astype(np.float32)
    cache.append_device(layer, _dev(x), _dev(x), _dev(slot))
    ok = slot // b < N - 2
    ko.append(k, s, x[ok], slot[ok], b, fmt)
    for scale, codes in ((layer.k_scale, layer.k), (layer.v_scale, layer.v.transpose(2, 3))):
        assert np.array_equal(scale[:N - 2].cpu().numpy(), s[:N - 2]) and np.array_equal(codes[:N - 2].cpu().numpy(), k[:N - 2])
    cache.close()


def _in_use(shape, dtype):
    """Memory of the current stream that is free again while zeros are still on their way there."""
    torch = _torch()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    x = torch.empty(shape, dtype=dtype, device="cuda:0")
    torch.cuda._sleep(20_000_000)
    x.zero_()


def test_a_cache_on_a_stream_of_its_own():
    """Workspace, layers and step arrays made while another stream is current: what that stream still does in memory that it has given back does not
    reach them, and what they give back is not handed out there while the cache's stream works in it.  Requests at the start may be that stream's."""
    torch = _torch()
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(3)
    W, B, b, N, M = 1, 40, 16, 4096, 60
    lens = rng.integers(1, 900, (W, B))
    table = _scattered(rng, lens, b, N, M)
    cfg = kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=1, head_dim=128)
    dl, dt = _dev(lens, torch.int32), _dev(table)
    _in_use(kv.workspace_bytes(cfg) // 4 + 64, torch.int32)
    cache = kv.KvCache(cfg, lens=dl, table=dt, stream=stream)
    torch.cuda.synchronize()
    assert np.array_equal(cache.lens.cpu().numpy(), lens) and np.array_equal(cache.table.cpu().numpy(), table)
    shape = (N, 1, b, 128)
    _in_use(shape, torch.uint8)
    layer = cache.new_layer()
    with torch.cuda.stream(stream):
        layer.k.fill_(7)
    torch.cuda.synchronize()
    assert bool((layer.k == 7).all())
    _in_use((W, 1 << 21), torch.int32)
    step = cache.alloc_step(1 << 21)
    with torch.cuda.stream(stream):
        step["slot"].fill_(7)
    torch.cuda.synchronize()
    assert bool((step["slot"] == 7).all())
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        layer.k.fill_(9)
    del layer
    mine = torch.empty(shape, dtype=torch.uint8, device="cuda:0").fill_(3)
    torch.cuda.synchronize()
    assert bool((mine == 3).all())
    cache.close()
    # lengths and blocks that the current stream has yet to write
    late, at = torch.zeros_like(dl), torch.full_like(dt, -1)
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    late.copy_(dl), at.copy_(dt)
    cache = kv.KvCache(cfg, lens=late, table=at, stream=stream)
    torch.cuda.synchronize()
    assert np.array_equal(cache.lens.cpu().numpy(), lens) and np.array_equal(cache.table.cpu().numpy(), table)
    cache.close()


def test_requests_of_the_start_are_not_kept():
    """The tensors that a cache begins with are the caller's alone once it has them."""
    torch = _torch()
    cfg = kv.KvConfig(rows=4, n_blocks=8, max_blocks=2)
    lens, table = torch.ones((1, 4), dtype=torch.int32, device="cuda:0"), torch.arange(8, dtype=torch.int32, device="cuda:0").view(1, 4, 2)
    cache = kv.KvCache(cfg, lens=lens, table=table, stream=torch.cuda.Stream())
    refs = weakref.ref(lens), weakref.ref(table)
    del lens, table
    assert refs[0]() is None and refs[1]() is None
    torch.cuda.synchronize()
    assert cache.lens.tolist() == [[1] * 4] and cache.table[0, :, 0].tolist() == [0, 2, 4, 6]
    cache.close()


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
def test_scales_up_to_the_largest(fmt):
    """Earlier scales up to 2^126 are scales, whatever their bits, and stay what an append has made of them; those above are none."""
    torch = _torch()
    D, b = 64, 16
    good = [2.0 ** 124, 2.0 ** 125, 1.5 * 2.0 ** 125, 8.5e37, 8.505e37, float(np.nextafter(np.float32(2.0 ** 126), np.float32(0))), 2.0 ** 126]
    none = [float(np.nextafter(np.float32(2.0 ** 126), np.float32(np.inf))), 1.5 * 2.0 ** 126, 2.0 ** 127, 3.4e38]
    s = np.array(good + none, np.float32)[:, None]
    N = len(s)
    cache = kv.KvCache(kv.KvConfig(rows=2, block_tokens=b, n_blocks=N, max_blocks=4, head_dim=D, fmt=fmt))
    layer = cache.new_layer()
    rng = np.random.default_rng(1)
    k = ko.encode(rng.integers(-110, 111, (N, 1, b, D)).astype(np.float64), fmt)
    layer.k.copy_(_dev(k)), layer.v.copy_(layer.k.transpose(2, 3))
    layer.k_scale.copy_(_dev(s)), layer.v_scale.copy_(_dev(s))
    ks, n = s[:len(good)].copy(), len(good)
    k = k[:n]
    for off in (5, 6, 7):
        x = rng.normal(size=(N, 1, D)).astype(np.float32) * (1.0 if off < 7 else 1e37)
        slot = np.arange(N) * b + off
        cache.append_device(layer, _dev(x), _dev(x), _dev(slot, torch.int32))
        ko.append(k, ks, x[:n], slot[:n], b, fmt)
        for scale, codes in ((layer.k_scale, layer.k), (layer.v_scale, layer.v.transpose(2, 3))):
            assert np.array_equal(scale[:n].cpu().numpy(), ks) and np.array_equal(codes[:n].cpu().numpy(), k), off
            assert bool(torch.isnan(scale[n:]).all()), off
    cache.close()


def test_one_token_of_any_stride():
    """Where there is one token, what lies between it and a next one is nobody's."""
    torch = _torch()
    H, D = 2, 64
    cache = kv.KvCache(kv.KvConfig(rows=2, n_blocks=4, max_blocks=2, n_kv_heads=H, n_q_heads=H, head_dim=D))
    layer = cache.new_layer()
    x = torch.randn(2, H, D, dtype=torch.float16, device="cuda:0")
    far = [torch.as_strided(x[i], (1, H, D), (2 ** 40 + 1, D, 1)) for i in range(2)]
    slot = torch.full((1,), 16, dtype=torch.int32, device="cuda:0")
    cache.append_device(layer, far[0], far[1], slot)
    y = torch.zeros(2, H, D, dtype=torch.float16, device="cuda:0")
    back = [torch.as_strided(y[i], (1, H, D), (2 ** 40 + 1, D, 1)) for i in range(2)]
    cache.read_device(layer, slot, back[0], back[1])
    near = torch.zeros_like(y)
    cache.append_device(layer, x[:1].clone(), x[1:].clone(), slot)
    cache.read_device(layer, slot, near[:1], near[1:])
    assert torch.equal(y, near) and bool((y - x).abs().max() < 0.05)
    cache.close()


def test_a_step_clears_what_a_broken_call_has_left():
    """Counters of delivered pieces that are not zero, as a call leaves them whose lengths were changed under it: after a step the next call is
    right again."""
    torch = _torch()
    rng = np.random.default_rng(7)
    D, b, L = 64, 16, 40000
    N = L // b
    cfg = kv.KvConfig(rows=2, block_tokens=b, n_blocks=N, max_blocks=N, head_dim=D)
    lens, table = _dev([[L, 0]], torch.int32), _dev(_scattered(rng, np.array([[L, 0]]), b, N, N))
    cache = kv.KvCache(cfg, lens=lens, table=table)
    layer = cache.new_layer()
    layer.k.random_(0, 256), layer.v.random_(0, 256), layer.k_scale.fill_(0.01), layer.v_scale.fill_(0.01)
    q = torch.randn(2, 1, D, dtype=torch.float16, device="cuda:0")
    want, out = torch.empty_like(q), torch.zeros_like(q)
    cache.attend_device(layer, q, want)
    zero, step = torch.zeros((1, 2), dtype=torch.int32, device="cuda:0"), cache.alloc_step(4)
    total = kv.workspace_bytes(cfg) // 4
    for left in (1, -1, 1000):
        cache.ws[total - 768:total].fill_(left)  # (the last of the workspace, the counters among them)
        cache.step_device(zero - 1, zero, step)
        for _ in range(2):
            out.zero_()
            cache.attend_device(layer, q, out)
            assert torch.equal(out, want), left
    cache.close()
