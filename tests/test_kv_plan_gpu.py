"""What a plan takes together, on the GPU: companies as they stand at the workspace's end, and the attention behind them."""
import ctypes as C

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests.test_kv_gpu import _check_attention, _say, _torch
from tests.test_kv_shared_gpu import _families, _i32, _reference, _shared_cache

pytestmark = pytest.mark.gpu

TILE = 64


def _companies(cache):
    """(worker, rows, tiles held together) of every company of the last plan: eight numbers for each row, the first and the third of them, and four for each
    member, the first of them its row, are the workspace's last two arrays, which begin at multiples of 256 bytes."""
    own = kv._SharedLayout()
    assert cache.lib.br_kv_get_shared_layout(cache.ctx, C.byref(own)) == 0
    W, B = cache.cfg.n_workers, cache.cfg.rows
    up = lambda n: (n + 255) // 256 * 256
    members = own.total_bytes - up(16 * W * B)
    companies = members - up(32 * W * B)
    ws = cache.ws.cpu().numpy()
    members, companies = ws[members // 4:][:4 * W * B].reshape(W * B, 4), ws[companies // 4:][:8 * W * B].reshape(W, B, 8)
    return [(w, [int(r) for r in members[c[1]:c[1] + c[0], 0] - w * B], int(c[2])) for w in range(W) for c in companies[w] if c[0] > 0]


def _plan(tag, lens, lead, blocks, members, alive=None, said=None, b=16, H=2, group=4, D=64):
    """Rows that hold their leader's first `blocks` blocks together, some of which have left since (alive); the companies of the plan, the attention checked."""
    torch = _torch()
    lens, lead = np.asarray(lens), np.asarray(lead)
    W, R = lens.shape
    _say("plan", tag, (W, R), "members", members)
    first, layer, h = _shared_cache(np.random.default_rng(R), "int8", W, R, b, D, H, group, lens, lead, np.full((W, R), blocks))
    if alive is not None:
        lens = np.where(alive, lens, 0)
    cache = kv.KvCache(first.cfg, lens=_i32(lens), table=_i32(h["table"]))
    q = torch.tensor(np.random.default_rng(1).normal(size=(W * R, H * group, D)), dtype=torch.float16, device="cuda:0")
    got = []
    for lists in (False, True):  # rows that have left: without tokens, or without a query as well
        count = np.where(lens > 0, 1, 0) if lists else np.ones((W, R), int)
        start = np.arange(W * R).reshape(W, R)
        out, lse = torch.full_like(q, 3.0), torch.full((W * R, H * group), 3.0, device="cuda:0")
        cache.plan_device(_i32(lead if said is None else said), members, **(dict(start=_i32(start), count=_i32(count)) if lists else {}))
        cache.attend_shared_device(layer, q, out, lse=lse)
        ref = _reference(q.double().cpu().numpy(), h, lens, start.reshape(-1), count.reshape(-1), W, group, b, "int8", 0, None)
        _check_attention((tag, lists), cache, q, out, lse, ref, "float16")
        got.append([c for c in _companies(cache) if lens[c[0], c[1][0]] > 0])
    first.close(), cache.close()
    assert got[0] == got[1], tag
    return got[0]


# one worker by one block, in two launches, and many workers: every way in which what rows have in common is found
@pytest.mark.parametrize("W,R", [(1, 12), (1, 48), (1, 100), (1, 300), (130, 72)], ids=str)
def test_leaders_that_have_left(W, R):
    """The rows that remain hold their first 320 tokens together, and are read together, whoever led them."""
    rng = np.random.default_rng(R)
    F = 6
    lens = 321 + rng.integers(0, 40, (W, R))
    lead = _families(R, F).repeat(W, 0)
    every = sorted((w, list(range(f, min(f + F, R))), 5) for w in range(W) for f in range(0, R, F))
    heads = dict(H=1, group=2) if W > 1 else {}
    assert sorted(_plan("all there", lens, lead, 20, F, **heads)) == every
    alive = np.arange(R)[None].repeat(W, 0) % F != 0
    left = [(w, rows[1:], 5) for w, rows, n in every if len(rows) > 1]
    assert sorted(_plan("leaders gone", lens, lead, 20, F, alive=alive, **heads)) == left
    alive = rng.random((W, R)) < 0.6
    left = [(w, [r for r in rows if alive[w, r]]) for w, rows, n in every]
    left = [(w, rows, 5 if len(rows) > 1 else 0) for w, rows in left if rows]
    got = [(w, rows, n if len(rows) > 1 else 0) for w, rows, n in _plan("some gone", lens, lead, 20, F, alive=alive, **heads)]
    assert sorted(got) == left


def test_a_leader_that_goes_with_others():
    """Row 0 leads rows 1..5 and is itself led by row 6: it is compared with that one, they with each other, and of the other family only the company that it
    has come to holds nothing together."""
    lens, lead = np.full((1, 12), 330), np.array([[0, 0, 0, 0, 0, 0, 6, 6, 6, 6, 6, 6]])
    said = lead.copy()
    said[0, 0] = 6
    for R in (12, 100):
        more = R - 12
        wide = lambda x, fill: np.concatenate([x, fill], 1)
        got = _plan("led", wide(lens, np.full((1, more), 5)), wide(lead, np.arange(12, R)[None]), 20, 6, said=wide(said, np.arange(12, R)[None]))
        got = [c for c in got if c[1][0] < 12]
        assert (0, [1, 2, 3, 4, 5], 5) in got and (0, [9, 10, 11], 5) in got and sum(0 in c[1] for c in got) == 1 and sorted(r for c in got for r in c[1]) == list(range(12)), got


@pytest.mark.parametrize("case", [(1, 16, 4, 64, 4), (1, 16, 16, 128, 2), (2, 40, 8, 192, 4), (1, 100, 4, 64, 4)], ids=str)
def test_a_plan_of_other_rows_is_none(case):
    """A step or a fork behind a plan, eager or replayed: the attention writes nothing until the next plan has run; compaction leaves it as it is."""
    torch = _torch()
    W, R, members, D, group = case
    _say("older plan", case)
    rng = np.random.default_rng(R)
    lens, lead = 150 + rng.integers(0, 100, (W, R)), _families(R, 8).repeat(W, 0)
    one, layer, h = _shared_cache(rng, "int8", W, R, 16, D, 2, group, lens, lead, np.full((W, R), 8))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    cache = kv.KvCache(one.cfg, lens=_i32(lens), table=_i32(h["table"]), stream=side)
    lead, q = _i32(lead), torch.tensor(rng.normal(size=(W * R, 2 * group, D)), dtype=torch.float16, device="cuda:0")
    out, lse = torch.empty_like(q), torch.empty((W * R, 2 * group), device="cuda:0")
    every, none, step, moves = _i32(np.full((W, R), -1)), _i32(np.zeros((W, R))), cache.alloc_step(4), cache.alloc_moves(h["N"])
    torch.cuda.synchronize()

    def attend(tag, planned):
        with torch.cuda.stream(side):
            out.fill_(7.0), lse.fill_(7.0)
        cache.attend_shared_device(layer, q, out, lse=lse)
        torch.cuda.synchronize()
        if not planned:
            assert bool((out == 7.0).all()) and bool((lse == 7.0).all()), tag
            return
        k, v, ks, vs = (x.cpu().numpy() for x in (layer.k, layer.v, layer.k_scale, layer.v_scale))
        now = dict(h, k=k, v=v, ks=ks, vs=vs, table=cache.table.cpu().numpy())
        ref = _reference(q.double().cpu().numpy(), now, cache.lens.cpu().numpy(), np.arange(W * R), np.ones(W * R, np.int64), W, group, 16, "int8", 0, None)
        _check_attention((case, tag), cache, q, out, lse, ref, "float16")

    def stepped():
        cache.step_device(every, none, step)

    def forked():
        cache.fork_device(every)

    cache.plan_device(lead, members)
    attend("first", True)
    graphs = {}
    for what in (stepped, forked):
        what()
        attend(("behind", what.__name__), False)
        cache.plan_device(lead, members)
        attend(("again", what.__name__), True)
        graphs[what] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[what], stream=side):
            what()
        attend(("captured", what.__name__), True)
    planning = torch.cuda.CUDAGraph()
    with torch.cuda.graph(planning, stream=side):
        cache.plan_device(lead, members)
    for what, graph in graphs.items():
        for turn in range(2):
            with torch.cuda.stream(side):
                graph.replay()
            attend(("replayed", what.__name__, turn), False)
            with torch.cuda.stream(side):
                planning.replay()
            attend(("planned", what.__name__, turn), True)
    cache.compact_device(moves)
    cache.copy_device(layer, moves["src"], moves["dst"])
    attend("compact", True)
    one.close(), cache.close()


@pytest.mark.parametrize("W,R,M", [(1, 8, 4), (300, 40, 200), (5000, 2, 4)], ids=str)
def test_every_form_of_a_fork_ends_a_plan(W, R, M):
    torch = _torch()
    _say("forks and plans", W, R, M)
    cache = kv.KvCache(kv.KvConfig(n_workers=W, rows=R, n_blocks=R, max_blocks=M, shared=True), lens=_i32(np.full((W, R), 16)),
                       table=_i32(np.where(np.arange(M) == 0, np.arange(R)[:, None], -1)[None].repeat(W, 0)))
    layer = cache.new_layer()
    for x in (layer.k, layer.v):
        x.fill_(1)
    for x in (layer.k_scale, layer.v_scale):
        x.fill_(1.0)
    q = torch.ones((W * R, 1, 64), dtype=torch.float16, device="cuda:0")
    out, lead = torch.zeros_like(q), _i32(np.zeros((W, R)))
    cache.plan_device(lead, 4)
    cache.attend_shared_device(layer, q, out)
    assert bool((out == 1.0).all())
    cache.fork_device(lead)
    cache.attend_shared_device(layer, q, out.fill_(7.0))
    assert bool((out == 7.0).all())
    cache.plan_device(lead, 4)
    cache.attend_shared_device(layer, q, out)
    assert bool((out == 1.0).all())
    cache.close()
