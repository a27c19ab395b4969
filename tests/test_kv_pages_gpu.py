"""Blocks that several rows hold, on the GPU: tables, holders, lists and bytes have to be equal to the plain statement's, and every row's tokens to what
was written into them, whoever else holds their blocks."""
import ctypes as C

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests.kv_pages_oracle import SharedTables

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _dev(x):
    return _torch().as_tensor(np.ascontiguousarray(x, np.int32), device="cuda:0")


def _say(*a):
    print(*a, flush=True)


def _same_tables(tag, cache, oracles):
    assert np.array_equal(cache.lens.cpu().numpy(), [o.lens for o in oracles]), (tag, "lens")
    assert np.array_equal(cache.table.cpu().numpy(), [o.table() for o in oracles]), (tag, "table")
    assert np.array_equal(cache.holders.cpu().numpy(), [o.holders() for o in oracles]), (tag, "holders")


def _same_step(tag, out, refs, cap):
    got = {n: x.cpu().numpy() for n, x in out.items()}
    for w, ref in enumerate(refs):
        ref["start"] = [w * cap + x for x in ref["start"]]
        for name, want in ref.items():
            assert np.array_equal(got[name][w], want), (tag, w, name)


def _forks(rng, W, B, lens):
    """Rows that go on from neighbours, from themselves, from anywhere, from nowhere; whole, cut, emptied."""
    frm = np.where(rng.random((W, B)) < 0.5, np.arange(B) // 4 * 4, rng.integers(0, B, (W, B)))
    frm = np.where(rng.random((W, B)) < 0.3, np.arange(B), frm)
    frm = np.where(rng.random((W, B)) < 0.3, rng.choice([-1, -2 ** 31, B, 2 ** 31 - 1], (W, B)), frm)
    cut = np.where(rng.random((W, B)) < 0.4, -1, (rng.random((W, B)) * (lens.max() + 20)).astype(int))
    return frm, np.where(rng.random((W, B)) < 0.1, 0, cut)


TABLES = [  # workers, rows, block, n_blocks, max_blocks, cap, longest request
    (1, 1, 16, 1, 1, 3, 16), (1, 4, 16, 31, 8, 64, 100), (3, 7, 32, 33, 5, 100, 160), (2, 64, 16, 400, 40, 700, 500), (5, 255, 64, 900, 30, 2000, 1500),
    (2, 300, 16, 1025, 64, 0, 900), (1, 1024, 128, 700, 20, 5000, 2000), (1, 40, 16, 262144, 700, 300000, 11000), (300, 13, 32, 64, 9, 77, 200),
]


@pytest.mark.parametrize("case", TABLES, ids=str)
def test_tables(case):
    W, B, b, N, M, cap, longest = case
    _say("tables", case)
    rng = np.random.default_rng(W * 1000 + B)
    cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M, shared=True))
    oracles = [SharedTables(B, b, N, M) for _ in range(W)]
    out = cache.alloc_step(cap)
    for k in range(8):
        keep = np.where(rng.random((W, B)) < 0.6, -1, rng.integers(-2, longest, (W, B)))
        keep = np.where(rng.random((W, B)) < 0.2, 0, keep)
        add = np.where(rng.random((W, B)) < 0.6, 1, np.exp(rng.uniform(0, np.log(longest), (W, B))).astype(int))
        add = np.where(rng.random((W, B)) < 0.1, rng.choice([0, -5, 2 ** 31 - 1, M * b, M * b + 1], (W, B)), add)
        if k == 6:
            keep, add = np.where(rng.random((W, B)) < 0.7, 0, -1), np.zeros((W, B), int)  # many leave
        for x in out.values():
            x.fill_(-77)
        cache.step_device(_dev(keep), _dev(add), out)
        _same_step((case, k), out, [o.step(keep[w], add[w], cap) for w, o in enumerate(oracles)], cap)
        _same_tables((case, k, "step"), cache, oracles)
        n = [N // 2 + 1, 3, 0, N][k % 4]
        if k % 2 == 0 or k == 7:
            moves = cache.alloc_moves(n)
            cache.compact_device(moves)
            refs = [o.compact(n) for o in oracles]
            for name in moves:
                assert np.array_equal(moves[name].cpu().numpy(), [r[name] for r in refs]), (case, k, name)
            _same_tables((case, k, "compact"), cache, oracles)
        lens = np.array([o.lens for o in oracles])
        frm, cut = _forks(rng, W, B, lens)
        cut = None if k == 3 else cut
        cache.fork_device(_dev(frm), None if cut is None else _dev(cut))
        for w, o in enumerate(oracles):
            o.fork(frm[w], None if cut is None else cut[w])
        _same_tables((case, k, "fork"), cache, oracles)
    cache.close()


@pytest.mark.parametrize("case", [(256, 40, 16, 20000, 1024), (256, 1000, 16, 60000, 64), (2, 200, 16, 4000, 12), (4200, 8, 16, 100, 4), (1, 40, 16, 262144, 11000), (5, 16, 32, 3000, 128), (3, 30, 64, 3000, 100)], ids=str)
def test_forks_of_many_entries(case):
    """Every way in which a fork's work is divided: lengths, tables, holders, and each row's last block (by what the next step asks to be copied)."""
    torch = _torch()
    W, B, b, N, M = case
    _say("forks", case)
    g = torch.Generator("cuda").manual_seed(B)
    r = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda:0", dtype=torch.int32)
    place = torch.arange(M, device="cuda:0", dtype=torch.int32)
    lens = r(0, M * b + 1, W, B)
    lens[:, 0], lens[:, 1] = M * b, 0
    table = torch.where(place < ((lens + b - 1) // b)[..., None], r(0, N, W, B, M), -1).int()
    for k in range(0, B - 1, 3):  # (rows that begin alike)
        n = torch.minimum((lens[:, k] + b - 1) // b, (lens[:, k + 1] + b - 1) // b) // 2
        table[:, k + 1] = torch.where(place < n[:, None], table[:, k], table[:, k + 1])
    cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=1, n_q_heads=1, head_dim=64, shared=True), lens=lens, table=table)
    step = cache.alloc_step(4 * B)
    for turn in range(2):
        frm, cut = r(0, B, W, B), r(-100, M * b + 50, W, B)
        own = r(0, 10, W, B)
        frm = torch.where(own < 2, torch.arange(B, device="cuda:0", dtype=torch.int32), torch.where(own == 3, -1, torch.where(own == 4, torch.arange(B, device="cuda:0", dtype=torch.int32) // 3 * 3, frm))).int()
        stays = (frm < 0) | (frm >= B)
        take = torch.where(stays, torch.arange(B, device="cuda:0", dtype=torch.int32), frm).long()
        held = lens.gather(1, take)
        lens2 = torch.where(stays | (cut < 0), held, torch.minimum(held, cut)).int()
        table2 = torch.where(place < ((lens2 + b - 1) // b)[..., None], table.gather(1, take[..., None].expand(-1, -1, M)), -1).int()
        cache.fork_device(frm, cut)
        lens, table = lens2, table2
        torch.cuda.synchronize()
        assert torch.equal(cache.lens, lens) and torch.equal(cache.table, table), (case, turn)
        ids = torch.where(table >= 0, table, N).view(W, -1).long()
        holders = torch.zeros((W, N + 1), dtype=torch.int32, device="cuda:0").scatter_add_(1, ids, torch.ones_like(ids, dtype=torch.int32))[:, :N]
        assert torch.equal(cache.holders, holders), (case, turn)
    cache.step_device(torch.full_like(lens, -1), ((lens > 0) & (lens < M * b)).int(), step)
    torch.cuda.synchronize()
    last = table.gather(2, torch.clamp((lens - 1) // b, min=0)[..., None].long())[..., 0]
    several = holders.gather(1, torch.clamp(last, min=0).long()) > 1
    want = torch.where((lens % b != 0) & several, last, -1)
    assert not bool(step["status"].any()) and torch.equal(step["copy_src"], want.int()), case
    now = torch.zeros((W, N + 1), dtype=torch.int32, device="cuda:0")
    ids = torch.where(cache.table >= 0, cache.table, N).view(W, -1).long()
    now.scatter_add_(1, ids, torch.ones_like(ids, dtype=torch.int32))
    assert torch.equal(cache.holders, now[:, :N]) and torch.equal(step["stats"][:, 1], (now[:, :N] > 0).sum(1)), case
    cache.close()


def test_requests_at_the_start_may_share_blocks():
    """Ids outside the worker's blocks count as none, lengths are clamped, stale entries are not looked at."""
    b, N, M = 16, 40, 6
    lens = [[90, 33, 33, 0, 1000, 20]]
    table = [[[7, 8, 9, 10, 11, 12], [7, 8, 3, 5, 5, 5], [7, 8, 4, -1, -1, -1], [9] * 6, [30, 31, 32, 33, 34, 7], [-3, N, 1, 1, 1, 1]]]
    cache = kv.KvCache(kv.KvConfig(rows=6, block_tokens=b, n_blocks=N, max_blocks=M, shared=True), lens=_dev(lens), table=_dev(table))
    rows = [[7, 8, 9, 10, 11, 12], [7, 8, 3], [7, 8, 4], [], [30, 31, 32, 33, 34, 7], [-1, -1]]
    o = SharedTables(6, b, N, M, [90, 33, 33, 0, 96, 20], [r + [-1] * (M - len(r)) for r in rows])
    _same_tables("start", cache, [o])
    assert cache.holders[0, 7].item() == 4
    out = cache.alloc_step(50)
    # row 5 ends inside a block that does not exist: its token has no place, and nothing is copied
    keep, add = [[90, 18, 33, -1, -1, -1]], [[6, 2, 15, 4, 1, 1]]
    cache.step_device(_dev(keep), _dev(add), out)
    _same_step("start", out, [o.step(keep[0], add[0], 50)], 50)
    _same_tables("start", cache, [o])
    frm = [[5, 0, 5, 1, -1, 2]]
    cache.fork_device(_dev(frm))
    o.fork(frm[0])
    _same_tables("holes", cache, [o])
    moves = cache.alloc_moves(N)
    cache.compact_device(moves)
    ref = o.compact(N)
    assert moves["src"][0].tolist() == ref["src"] and moves["dst"][0].tolist() == ref["dst"]
    _same_tables("holes", cache, [o])
    cache.close()


# -- what the rows hold ---------------------------------------------------------------
def _vectors(tags, H, D):
    """A token's key and value from its number: whole numbers up to 100 and one of 127, which int8 holds as they are with a scale of 1."""
    tags = np.asarray(tags, np.int64).reshape(-1)
    ch = np.arange(H * D)
    x = (tags[:, None] * 7919 + ch * (13 + tags[:, None] % 5)) % 201 - 100
    x[:, ::D] = 127
    x = x.reshape(-1, H, D)
    return x, -x[:, :, ::-1]


class Content:
    """A shared cache with tokens that are numbered, and the numbers that each row should hold."""

    def __init__(self, W, B, b, N, M, H, D, cap, seed, stream=None):
        torch = _torch()
        self.rng, self.dims, self.cap = np.random.default_rng(seed), (W, B, b, N, M, H, D), cap
        self.cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=H, n_q_heads=H, head_dim=D, fmt="int8", shared=True), stream=stream)
        self.layer, self.out = self.cache.new_layer(), self.cache.alloc_step(cap)
        self.layer.k.fill_(99), self.layer.v.fill_(98), self.layer.k_scale.fill_(float("nan")), self.layer.v_scale.fill_(float("nan"))
        self.rows, self.next = [[[] for _ in range(B)] for _ in range(W)], 1
        torch.cuda.synchronize()

    def step(self, keep, add):
        torch = _torch()
        W, B, b, N, M, H, D = self.dims
        self.cache.step_device(_dev(keep), _dev(add), self.out)
        self.cache.copy_device(self.layer, self.out["copy_src"], self.out["copy_dst"])
        count, tags = self.out["count"].cpu().numpy(), np.zeros((W, self.cap), np.int64)
        for w in range(W):
            at = 0
            for r in range(B):
                row = self.rows[w][r]
                if keep[w, r] >= 0:
                    del row[keep[w, r]:]
                new = list(range(self.next, self.next + count[w, r]))
                self.next += len(new)
                row += new
                tags[w, at:at + len(new)] = new
                at += len(new)
        k, v = (torch.tensor(np.ascontiguousarray(x), dtype=torch.float16, device="cuda:0") for x in _vectors(tags, H, D))
        self.cache.append_device(self.layer, k, v, self.out["slot"])

    def fork(self, frm, cut):
        B = self.dims[1]
        self.cache.fork_device(_dev(frm), _dev(cut))
        for w, rows in enumerate(self.rows):
            old = [list(r) for r in rows]
            for r in range(B):
                f, c = int(frm[w, r]), int(cut[w, r])
                if 0 <= f < B:
                    rows[r] = old[f] if c < 0 else old[f][:c]
                    rows[r] = list(rows[r])

    def compact(self, n):
        moves = self.cache.alloc_moves(n)
        self.cache.compact_device(moves)
        self.cache.copy_device(self.layer, moves["src"], moves["dst"])

    def check(self, tag):
        torch = _torch()
        W, B, b, N, M, H, D = self.dims
        lens, table = self.cache.lens.cpu().numpy(), self.cache.table.cpu().numpy()
        n = max(1, max(sum(len(r) for r in rows) for rows in self.rows))
        slot, tags = np.full((W, n), -1, np.int32), np.zeros((W, n), np.int64)
        for w in range(W):
            assert lens[w].tolist() == [len(r) for r in self.rows[w]], (tag, w)
            p = [(r, i) for r in range(B) for i in range(lens[w, r])]
            for at, (r, i) in enumerate(p):
                slot[w, at], tags[w, at] = table[w, r, i // b] * b + i % b, self.rows[w][r][i]
        k, v = (torch.empty((W * n, H, D), device="cuda:0") for _ in range(2))
        self.cache.read_device(self.layer, _dev(slot), k, v)
        wk, wv = _vectors(tags, H, D)
        there = slot.reshape(-1) >= 0
        assert np.array_equal(k.cpu().numpy()[there], wk[there]) and np.array_equal(v.cpu().numpy()[there], wv[there]), tag


CONTENT = [  # workers, rows, block, n_blocks, max_blocks, heads, width
    (1, 8, 16, 60, 12, 1, 64), (2, 13, 32, 50, 8, 3, 96), (3, 9, 64, 30, 5, 2, 128), (1, 17, 128, 30, 3, 5, 192), (2, 6, 16, 40, 20, 2, 256),
]


@pytest.mark.parametrize("case", CONTENT, ids=str)
def test_every_row_keeps_its_own_tokens(case):
    W, B, b, N, M, H, D = case
    _say("content", case)
    c = Content(*case, cap=B * M * b, seed=B)
    rng = c.rng
    for k in range(10):
        room = M * b
        keep = np.where(rng.random((W, B)) < 0.7, -1, rng.integers(0, room, (W, B)))
        add = np.where(rng.random((W, B)) < 0.5, 1, rng.integers(0, room // 2, (W, B)))
        c.step(np.where(rng.random((W, B)) < 0.1, 0, keep), add)
        c.check((case, k, "step"))
        frm, cut = _forks(rng, W, B, np.array([[len(r) for r in rows] for rows in c.rows]))
        c.fork(frm, cut)
        if k % 3 == 1:
            c.compact([N, 2][k % 2])
        c.check((case, k, "fork"))
        c.step(np.full((W, B), -1), np.where(rng.random((W, B)) < 0.7, rng.integers(0, 4, (W, B)), 0))
        c.check((case, k, "write"))
    c.cache.close()


def test_attention_of_rows_that_share_blocks():
    """... is that of rows with blocks of their own, bit for bit."""
    torch = _torch()
    W, B, b, N, M, H, D = 1, 12, 16, 300, 30, 2, 64
    c = Content(W, B, b, N, M, H, D, cap=B * 200, seed=3)
    c.step(np.zeros((W, B), int), np.where(np.arange(B) % 4 == 0, 150 + np.arange(B) * 11, 0)[None])
    c.fork((np.arange(B) // 4 * 4)[None], np.where(np.arange(B) % 2, 130, -1)[None])
    c.step(np.full((W, B), -1), (1 + np.arange(B) % 3)[None])
    lens = c.cache.lens.clone()
    own = kv.KvCache(kv.KvConfig(rows=B, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=H, n_q_heads=H, head_dim=D, fmt="int8"))
    layer, out = own.new_layer(), own.alloc_step(int(lens.sum()))
    own.step_device(_dev(np.zeros((W, B))), lens, out)
    k, v = (torch.tensor(np.ascontiguousarray(x), dtype=torch.float16, device="cuda:0") for x in _vectors([t for r in c.rows[0] for t in r], H, D))
    own.append_device(layer, k, v, out["slot"])
    q = torch.randn((B, H, D), generator=torch.Generator("cuda").manual_seed(1), device="cuda:0").to(torch.bfloat16) / 1024
    one, two = torch.empty_like(q), torch.empty_like(q)
    c.cache.attend_device(c.layer, q, one)
    own.attend_device(layer, q, two)
    assert torch.equal(one, two) and bool(torch.isfinite(one.float()).all()) and one.float().abs().max() > 1
    c.cache.close(), own.close()


# -- copies ---------------------------------------------------------------------------
@pytest.mark.parametrize("case", [(1, 1, 16, 64, 1), (3, 5, 32, 96, 7), (2, 3, 128, 256, 40), (4, 17, 64, 128, 0), (2, 1, 16, 192, 300),
                                  (7, 1, 16, 96, 300), (3, 1, 32, 64, 700), (9, 1, 16, 64, 230), (2, 2, 16, 64, 1100)], ids=str)
def test_copies(case):
    """Bytes and scales of blocks, also from worker to worker; pairs that are none; nothing else changes."""
    torch = _torch()
    W, H, b, D, n = case
    _say("copies", case)
    rng = np.random.default_rng(n)
    N = 2 * n + 3
    cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=2, block_tokens=b, n_blocks=N, max_blocks=2, n_kv_heads=H, n_q_heads=H, head_dim=D))
    layer = cache.new_layer()
    for x in (layer.k, layer.v):
        x.copy_(torch.randint(0, 256, x.shape, dtype=torch.uint8, device="cuda:0"))
    for x in (layer.k_scale, layer.v_scale):
        x.copy_(torch.randint(-2 ** 31, 2 ** 31 - 1, x.shape, dtype=torch.int32, device="cuda:0").view(torch.float32))
    ids = np.stack([rng.permutation(N) for _ in range(W)])
    src, dst = ids[:, :n].copy(), ids[:, n:2 * n].copy()
    workers = rng.integers(0, W, (W, n))
    for bad, where in ((src, 0.1), (dst, 0.1)):
        bad[rng.random((W, n)) < where] = -1
    if n > 6:
        src[0, :3], dst[0, 3:6] = [N, -2 ** 31, 2 ** 31 - 1], [N, 2 ** 31 - 1, -7]
    given = [workers, None] if W > 1 else [None]
    for other in given:
        # (blocks of other workers at the same numbers: sources and destinations of one call are apart)
        s, d = (src, dst) if other is None else (np.where(src >= 0, src % (n + 1), src), np.where((dst >= 0) & (dst < N), n + 1 + dst % (n + 2), dst))
        if other is not None:
            for w in range(W):
                seen = set()
                for j in range(n):
                    if d[w, j] in seen:
                        d[w, j] = -1
                    seen.add(d[w, j])
        want = {k: getattr(layer, k).view(torch.int32 if "scale" in k else torch.uint8).cpu().numpy().reshape(W, N, -1).copy() for k in ("k", "v", "k_scale", "v_scale")}
        before = {k: x.copy() for k, x in want.items()}
        for w in range(W):
            for j in range(n):
                if 0 <= s[w, j] < N and 0 <= d[w, j] < N:
                    for k in want:
                        want[k][w, d[w, j]] = before[k][w if other is None else other[w, j], s[w, j]]
        cache.copy_device(layer, _dev(s), _dev(d), None if other is None else _dev(other))
        for k in want:
            assert np.array_equal(getattr(layer, k).view(torch.int32 if "scale" in k else torch.uint8).cpu().numpy().reshape(W, N, -1), want[k]), (case, k)
    if n and W > 1:  # workers that do not exist: no pair
        kept = layer.k.clone()
        cache.copy_device(layer, _dev(src), _dev(dst), _dev(np.where(workers % 2, -1, W)))
        assert torch.equal(kept, layer.k)
    cache.close()


# -- graphs, streams, refusals -----------------------------------------------------------
def test_captured_and_replayed_on_a_stream_of_its_own():
    """Fork, step, copies, compaction in one graph: replayed with eager calls between, each time as the plain statement has it."""
    torch = _torch()
    W, B, b, N, M = 2, 10, 16, 80, 12
    stream = torch.cuda.Stream()
    c = Content(W, B, b, N, M, 1, 64, cap=B * 40, seed=9, stream=stream)
    oracles = [SharedTables(B, b, N, M) for _ in range(W)]
    frm, cut = np.tile(np.arange(B) // 5 * 5, (W, 1)), np.tile(np.where(np.arange(B) % 5, -1, 70), (W, 1))
    add, keep = np.tile(np.arange(B) % 3, (W, 1)), np.full((W, B), -1)
    dev = [_dev(x) for x in (frm, cut, add, keep)]
    moves = c.cache.alloc_moves(N)
    first = _dev(np.where(np.arange(B) % 5 == 0, 90, 3)[None].repeat(W, 0)), _dev(np.zeros((W, B)))
    torch.cuda.synchronize()

    def run():
        c.cache.fork_device(dev[0], dev[1])
        c.cache.step_device(dev[3], dev[2], c.out)
        c.cache.copy_device(c.layer, c.out["copy_src"], c.out["copy_dst"])
        c.cache.compact_device(moves)
        c.cache.copy_device(c.layer, moves["src"], moves["dst"])

    def plain():
        for w, o in enumerate(oracles):
            o.fork(frm[w], cut[w])
            o.step(keep[w], add[w], c.cap)
            o.compact(N)

    c.cache.step_device(first[1], first[0], c.out)
    for w, o in enumerate(oracles):
        o.step([0] * B, first[0].cpu().numpy()[w], c.cap)
    run(), plain()
    torch.cuda.synchronize()
    _same_tables("eager", c.cache, oracles)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run()
    for k in range(4):
        with torch.cuda.stream(stream):
            graph.replay()
        plain()
        torch.cuda.synchronize()
        _same_tables(("replay", k), c.cache, oracles)
        if k % 2:  # eager work between: some leave, others come
            gone = _dev(np.where(np.arange(B) % 5 == 3, 0, -1)[None].repeat(W, 0))
            torch.cuda.synchronize()
            c.cache.step_device(gone, first[0], c.out)
            for w, o in enumerate(oracles):
                o.step(gone.cpu().numpy()[w], first[0].cpu().numpy()[w], c.cap)
            torch.cuda.synchronize()
            _same_tables(("between", k), c.cache, oracles)
    c.cache.close()


def test_refusals():
    torch = _torch()
    sizes = dict(rows=4, n_blocks=20, max_blocks=4, n_kv_heads=1, n_q_heads=1, head_dim=64)
    one, more = kv.KvCache(kv.KvConfig(**sizes)), kv.KvCache(kv.KvConfig(**sizes, shared=True))
    x = _dev(np.zeros((1, 64)))
    p, lib, layer = x.data_ptr(), one.lib, more.new_layer()
    lens, out = C.byref(kv._Lengths(keep=p, add=p)), C.byref(kv._StepOut(token_cap=0))
    moves = lambda **kw: C.byref(kv._Moves(**{**dict(src=p, dst=p, n=4), **kw}))
    forks = lambda **kw: C.byref(kv._Forks(**{**dict(from_=p), **kw}))
    assert lib.br_kv_step(more.ctx, lens, out) == -1 and lib.br_kv_step_shared(one.ctx, lens, out, moves()) == -1
    assert lib.br_kv_fork(one.ctx, forks()) == -1 and lib.br_kv_compact(one.ctx, moves()) == -1
    assert lib.br_kv_get_shared_layout(one.ctx, C.byref(kv._SharedLayout())) == -1
    for bad in (None, moves(n=3), moves(n=5), moves(src=None), moves(dst=None)):
        assert lib.br_kv_step_shared(more.ctx, lens, out, bad) == -1
    assert lib.br_kv_fork(more.ctx, None) == -1 and lib.br_kv_fork(more.ctx, forks(from_=None)) == -1
    for bad in (None, moves(n=-1), moves(n=2 ** 31 - 256), moves(src=None), moves(dst=None)):
        assert lib.br_kv_compact(more.ctx, bad) == -1 and lib.br_kv_copy(more.ctx, layer.ref, bad) == -1
    assert lib.br_kv_copy(more.ctx, None, moves()) == -1
    for call in (lambda m: lib.br_kv_compact(more.ctx, m), lambda m: lib.br_kv_copy(more.ctx, layer.ref, m)):
        assert call(moves(n=0, src=None, dst=None)) == 0
    torch.cuda.synchronize()
    assert not bool(more.lens.any()) and not bool(x.any())
    one.close(), more.close()
