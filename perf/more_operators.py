"""Measured cases of what a worker does with blocks that several requests hold, and of differential attention over its cache.

Requests that begin alike (samples of one prompt, beams, turns of one talk) hold the same blocks of the 8-bit cache until they
write into them.  A pass is one call, or a few in a row, of a program that keeps such a cache:

  fork     rows take over other rows' tokens by holding their blocks
  branch   rows are forked, get their next tokens (each a block of its own where it would write into one that others hold) and the
           blocks that go with that are copied
  copy     blocks of requests that move from worker to worker
  compact  requests leave, the blocks in use move to the lowest ids, their keys and values with them, requests come
  diff     differential attention: the first map's result less lambda times the second's

Keys of a case:
  kind                  one of the above
  workers, rows         workers, and requests a worker may hold
  block                 tokens of a block
  len_lo, len_hi        cached tokens of a row: spread evenly over the logarithm, in an order drawn from the seed
  idle                  rows that hold nothing
  fork, branch: family  rows that begin alike; how: "samples": a family's rows take over its first one, "beams": each takes over any of
                        them; own: tokens of a row that the others of its family do not hold; cut: the rows keep so many of a hundred of the
                        tokens that they take over (100: all)
  branch: add           tokens that come to each row
  copy: take            requests that each worker gets from another
  compact: leave        share of the rows that leave; room: of a hundred blocks, those that a list of moves has places for
  heads, group, dim     key heads, query heads for each of them, head width (diff: both maps' channels side by side)
  fmt                   "int8" or "fp8" (e4m3); dtype: of queries ("bf16", "f16")
  diff: tokens          query tokens of a row; chunk, chunk_rows: so many of the rows have `chunk` of them instead
        window          tokens that a query sees, itself included; 0: all up to itself
        lam             "head": a lambda for each query head; "token": for each token and query head
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
TOP = {"int8": 127.0, "fp8": 448.0}
STATS = 8


def _case(name, kind, **kw):
    c = dict(kind=kind, workers=1, rows=96, block=16, len_lo=256, len_hi=8192, idle=0, heads=8, dim=128, fmt="int8")
    if kind in ("fork", "branch"):
        c.update(family=8, how="samples", own=0, cut=100)
    if kind == "branch":
        c.update(add=1)
    if kind == "copy":
        c.update(take=1)
    if kind == "compact":
        c.update(leave=0.3, room=100)
    if kind == "diff":
        c.update(group=4, dtype="bf16", tokens=1, chunk=0, chunk_rows=0, window=0, lam="head")
    c.update(kw)
    if kind == "fork":
        del c["heads"], c["dim"], c["fmt"]  # tables only
    return dict(c, name=name) if name else c


def listed():
    return [
        # one worker: every prompt is sampled eight times
        _case("fork_samples", "fork"),
        # beams of all workers of a replay trade places at a step: all rows at once, each family's among themselves
        _case("fork_beams", "fork", workers=512, rows=144, block=64, how="beams", own=300, family=4, idle=4),
        # the first tokens of those samples: each row's last block is its own from here on
        _case("branch_samples", "branch", len_lo=300, len_hi=4000),
        # a few workers with odd sizes; rows go back to a point inside what they share and go on from there with drafted tokens
        _case("branch_ragged", "branch", workers=13, rows=77, block=32, len_lo=1, len_hi=3000, how="beams", own=40, family=5, cut=90, add=5, heads=3, dim=96, fmt="fp8", idle=7),
        # one short request to its neighbour: the smallest call
        _case("copy_short", "copy", workers=2, rows=3, len_lo=100, len_hi=500),
        # requests that change workers when loads are evened out
        _case("copy_requests", "copy", workers=16, rows=6, block=64, len_lo=1024, len_hi=16384, take=2, fmt="fp8"),
        # a worker gives part of its memory away when its requests have become few
        _case("compact_worker", "compact", block=64, leave=0.6, fmt="fp8"),
        # the workers of a batch of small clusters
        _case("compact_workers", "compact", workers=300, rows=31, len_lo=20, len_hi=1000, heads=1, dim=64, room=10),
        # the smallest attention: one short request
        _case("diff_one_short", "diff", rows=1, len_lo=500, len_hi=500),
        # a full worker of the throughput configuration
        _case("diff_batch", "diff", rows=144, block=64, group=8, fmt="fp8", idle=3),
        # four drafted tokens to each request, a sliding window, odd head counts, narrow heads, lambda from the token
        _case("diff_drafts_window", "diff", rows=57, len_lo=5, len_hi=16384, heads=3, group=3, dim=64, dtype="f16", tokens=4, window=1024, lam="token"),
        # two prompts of which a chunk of 512 tokens is run beside the others' decode steps
        _case("diff_chunks", "diff", rows=48, block=128, len_lo=512, fmt="fp8", chunk=512, chunk_rows=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fork", "branch", "copy", "compact", "diff", "diff", "diff"])
    block = rng.choice([16, 32, 64, 128])
    if kind == "fork":
        workers = _log_int(rng, 1, 2048)
        rows = _log_int(rng, 2, min(1024, max(8, 70000 // workers)))
        hi = min(16384, max(64, 100000000 // (workers * rows)))
        return _case(None, kind, workers=workers, rows=rows, block=block, len_lo=_log_int(rng, 1, 60), len_hi=_log_int(rng, 64, hi), idle=rng.randrange(0, 1 + rows // 8),
                     family=rng.randrange(2, 13), how=rng.choice(["samples", "beams"]), own=rng.choice([0, 1, _log_int(rng, 2, 400)]), cut=rng.choice([100, 100, rng.randrange(1, 100)]))
    sizes = dict(block=block, heads=rng.randrange(1, 13), dim=rng.choice([64, 96, 128, 192, 256]), fmt=rng.choice(["int8", "fp8"]))
    cells = sizes["heads"] * sizes["dim"]
    if kind == "diff":
        sizes["group"] = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 12, 16])
        sizes.update(dtype=rng.choice(["bf16", "f16"]), lam=rng.choice(["head", "token"]))
        most = 200000000 // cells
        rows = _log_int(rng, 1, 300)
        hi = _log_int(rng, 16, max(17, min(40960, most // rows)))
        if rng.random() < 0.25:
            chunk = max(2, min(hi // 6, rng.randrange(9, 600), 20000000000 // (hi * cells * sizes["group"])))
            return _case(None, kind, rows=rows, len_lo=max(1, hi // 30), len_hi=hi, chunk=chunk, chunk_rows=1, **sizes)
        return _case(None, kind, rows=rows, len_lo=rng.randrange(5, 6 + min(hi - 10, 300)), len_hi=hi, tokens=rng.choice([1, 1, 1, 2, 5]), window=rng.choice([0, 0, 0, 100, 2048]),
                     idle=rng.randrange(0, 1 + rows // 8), **sizes)
    most = max(2000, 300000000 // cells)  # tokens of all rows together
    workers = _log_int(rng, 2 if kind == "copy" else 1, 200)
    rows = _log_int(rng, 2, max(3, min(300, most // (40 * workers))))
    hi = max(20, min(16384, most // (workers * rows)))
    lens = dict(len_lo=rng.randrange(1, 20), len_hi=_log_int(rng, 20, max(21, hi)))
    idle = rng.randrange(0, 1 + rows // 8)
    if kind == "branch":
        return _case(None, kind, workers=workers, rows=rows, idle=idle, family=rng.randrange(2, 13), how=rng.choice(["samples", "beams"]),
                     own=rng.choice([0, 1, _log_int(rng, 2, 400)]), cut=rng.choice([100, 100, rng.randrange(1, 100)]), add=rng.choice([1, 1, 1, 3, 40]), **lens, **sizes)
    if kind == "copy":
        return _case(None, kind, workers=workers, rows=rows, take=rng.randrange(1, 1 + min(4, rows)), **lens, **sizes)
    return _case(None, kind, workers=workers, rows=rows, idle=idle, leave=rng.uniform(0.05, 0.9), room=rng.choice([100, 50, 50, rng.randrange(1, 30)]), **lens, **sizes)


def _spread(n, lo, hi):
    """n lengths, even over the logarithm of [lo, hi]."""
    return [min(hi, max(lo, int(round(lo * (hi / lo) ** ((k + 0.5) / n))))) for k in range(n)]


def _lengths(case):
    """Cached tokens of the rows of a worker before the call, unordered; of families: rows of one follow each other."""
    n = case["rows"] - case["idle"]
    if "family" not in case:
        return _spread(n, case["len_lo"], case["len_hi"]) + [0] * case["idle"]
    f = case["family"]
    shared = _spread(_up(n, f), case["len_lo"], case["len_hi"])
    return [shared[r // f] + case["own"] for r in range(n)] + [0] * case["idle"]


def _up(x, m):
    return (x + m - 1) // m


def _blocks(case):
    """(blocks of a worker, entries of a row's table)."""
    lens, b = _lengths(case), case["block"]
    if "family" in case:  # (every row may come to have its last blocks for itself, and what it gets beside what it gave up)
        extra = case["own"] + case.get("add", 0)
        firsts = lens[:case["rows"] - case["idle"]:case["family"]]
        return sum(_up(x, b) for x in firsts) + 2 * case["rows"] * (_up(extra, b) + 2), _up(max(lens) + extra, b) + 1
    held = sum(_up(x, b) for x in lens)
    if case["kind"] == "copy":
        return held + sum(_up(x, b) for x in sorted(lens)[-case["take"]:]) + 3, _up(max(lens), b)
    return held + max(4, held // 8), _up(max(lens), b)


def _order(shape, g):
    return torch.rand(shape, generator=g, device=DEVICE).argsort(-1)


def _table(nb, width, n_blocks, g):
    """Rows of nb [W, R] blocks each, scattered over their worker's n_blocks: [W, R, width], -1 behind the last."""
    W, R = nb.shape
    order = _order((W, n_blocks), g).to(torch.int32)
    first = nb.cumsum(1) - nb
    at = torch.arange(width, device=DEVICE)
    where = (first[:, :, None] + at).clamp_(max=n_blocks - 1).view(W, R * width)
    return torch.where(at < nb[:, :, None], order.gather(1, where).view(W, R, width), -1).contiguous()


def _families(case, g):
    """Lengths and tables of rows that hold their family's first blocks together, and the last ones alone."""
    W, R, b, f = case["workers"], case["rows"], case["block"], case["family"]
    n_blocks, width = _blocks(case)
    n = R - case["idle"]
    lens = torch.tensor(_lengths(case), device=DEVICE)
    row = torch.arange(R, device=DEVICE)
    first = torch.where(row < n, row // f * f, row)
    nb = (lens + b - 1) // b
    together = torch.where(row == first, 0, (lens - case["own"]).clamp(min=0) // b)  # blocks that are the first row's
    if case["own"] == 0:
        together = torch.where(row == first, 0, nb)
    alone = _table((nb - together).expand(W, R), width, n_blocks, g)
    at = torch.arange(width, device=DEVICE)
    mine = alone.gather(2, (at - together[:, None]).clamp(0, width - 1).expand(W, R, width))
    table = torch.where(at < together[:, None], alone[:, first], torch.where(at < nb[:, None], mine, -1))
    take = first if case["how"] == "samples" else torch.minimum(first + (torch.rand((W, R), generator=g, device=DEVICE) * f).long(), torch.tensor(max(n - 1, 0), device=DEVICE))
    take = torch.where(row < n, take, -1).expand(W, R)
    cut = torch.where(row < n, _cut(case, lens), 0).expand(W, R)
    i32 = lambda x: x.to(torch.int32).contiguous()
    return dict(lens=i32(lens.expand(W, R)), table=i32(table), take=i32(take), cut=i32(cut))


def _cut(case, lens):
    """Tokens that rows of these lengths keep of what they take over (a family's rows are of one length)."""
    return (lens * case["cut"] + 99) // 100


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    W, R, b, kind = case["workers"], case["rows"], case["block"], case["kind"]
    n_blocks, width = _blocks(case)
    s = dict(case=case, n_blocks=n_blocks)
    if "family" in case:
        s.update(_families(case, g))
    else:
        base = torch.tensor(_lengths(case), device=DEVICE)
        lens = base[_order((W, R), g)]
        s["lens"], s["table"] = lens.to(torch.int32), _table((lens + b - 1) // b, width, n_blocks, g)
    if kind == "branch":
        s["keep"] = torch.full((W, R), -1, dtype=torch.int32, device=DEVICE)
        s["add"] = torch.where(s["take"] >= 0, case["add"], 0).to(torch.int32)
        s["cap"] = R * case["add"]
    if kind == "copy":
        s.update(_moves(s, g))
    if kind == "compact":
        gone = torch.rand((W, R), generator=g, device=DEVICE) < case["leave"]
        s["keep"] = torch.where(gone, 0, -1).to(torch.int32)
        s["add"] = torch.where(gone, s["lens"], 0).contiguous()
        s["none"], s["all"] = torch.zeros_like(s["add"]), torch.full_like(s["keep"], -1)
        s["cap"], s["room"] = sum(_lengths(case)), max(1, n_blocks * case["room"] // 100)
    if kind == "diff":
        _prepare_diff(s, g)
    elif kind != "fork":
        H, D, N = case["heads"], case["dim"], W * n_blocks
        top = 255 if case["fmt"] == "int8" else 127  # (codes below 127 are numbers of either type)
        codes = lambda *shape: torch.randint(0, top, shape, generator=g, device=DEVICE, dtype=torch.uint8)
        s["k"], s["v"] = codes(N, H, b, D), codes(N, H, D, b)
        s["k_scale"], s["v_scale"] = (torch.exp2(torch.randint(-12, 1, (N, H), generator=g, device=DEVICE).float()) for _ in range(2))
    if own:
        _own_cache(s)
    return s


def _moves(s, g):
    """Each worker takes the longest requests of another one: their blocks into free ones of its own."""
    c = s["case"]
    W, R, n_blocks, width = c["workers"], c["rows"], s["n_blocks"], s["table"].shape[2]
    giver = (torch.arange(W, device=DEVICE) + 1 + int(torch.randint(0, W - 1, (1,), generator=g, device=DEVICE)) if W > 1 else torch.zeros(1, device=DEVICE)).long() % W
    rows = s["lens"].argsort(1, descending=True)[:, :c["take"]].long()
    src = s["table"].gather(1, rows[:, :, None].expand(W, c["take"], width))[giver].reshape(W, -1)
    held = torch.zeros((W, n_blocks + 1), dtype=torch.bool, device=DEVICE).scatter_(1, torch.where(s["table"] < 0, n_blocks, s["table"]).view(W, R * width).long(), True)
    free = torch.where(held[:, :n_blocks], 2.0, torch.rand((W, n_blocks), generator=g, device=DEVICE)).argsort(1)
    there = src >= 0
    nth = (there.cumsum(1) - 1).clamp(0, n_blocks - 1)
    dst = torch.where(there, free.gather(1, nth), -1)
    i32 = lambda x: x.to(torch.int32).contiguous()
    return dict(src=i32(src), dst=i32(dst), src_worker=i32(giver[:, None].expand(src.shape)))


def _prepare_diff(s, g):
    c = s["case"]
    H, G, D, b, n_blocks, t = c["heads"], c["group"], c["dim"], c["block"], s["n_blocks"], TYPES[c["dtype"]]
    randn = lambda *shape: torch.randn(shape, generator=g, device=DEVICE)
    # values of a block and head have a size of their own, and a few channels of the keys stand out
    out = torch.where(torch.rand((H, 1, D), generator=g, device=DEVICE) < 0.03, 6.0, 1.0)
    size = torch.exp(0.5 * randn(n_blocks, H, 1, 1))
    k, s["k_scale"] = _encode_blocks(randn(n_blocks, H, b, D) * out, c["fmt"])
    v, s["v_scale"] = _encode_blocks(randn(n_blocks, H, b, D) * size, c["fmt"])
    s["k"], s["v"] = k, v.transpose(2, 3).contiguous()
    del k, v
    lens = s["lens"][0].long()
    count = torch.where(lens > 0, c["tokens"], 0)
    if c["chunk_rows"]:  # the longest rows
        count[lens.argsort(descending=True)[:c["chunk_rows"]]] = c["chunk"]
    s["count"] = count.to(torch.int32)
    s["start"] = (count.cumsum(0) - count).to(torch.int32)
    s["max_count"] = max(c["tokens"], c["chunk"])
    s["T"] = sum(_counts(c))
    s["q"] = randn(s["T"], H * G, D).to(t)
    # what exp(a . b) - exp(c . d) + lambda_0 of trained vectors comes to; from the token: a gate
    s["lam"] = 0.5 + 0.2 * randn(H * G) if c["lam"] == "head" else torch.sigmoid(randn(s["T"], H * G))
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((s["T"], H * G, 2), device=DEVICE)
    s["max_len"] = max(_lengths(c))


def _counts(case):
    n = case["rows"] - case["idle"]
    return [case["chunk"]] * case["chunk_rows"] + [case["tokens"]] * (n - case["chunk_rows"])


def _own_cache(s):
    """The handles that a program with this cache keeps."""
    from paper_2605_06113_amd import kv
    c = s["case"]
    cfg = kv.KvConfig(n_workers=c["workers"], rows=c["rows"], block_tokens=c["block"], n_blocks=s["n_blocks"], max_blocks=s["table"].shape[2], n_kv_heads=c.get("heads", 1),
                      n_q_heads=c.get("heads", 1) * c.get("group", 1), head_dim=c.get("dim", 64), fmt=c.get("fmt", "int8"), shared=c["kind"] != "diff")
    s["cache"] = cache = kv.KvCache(cfg, lens=s["lens"], table=s["table"], device=DEVICE)
    if c["kind"] != "fork":
        s["layer"] = cache.layer(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if c["kind"] in ("branch", "compact"):
        s["step"] = cache.alloc_step(s["cap"])
    if c["kind"] == "compact":
        s["moves"], s["back"] = cache.alloc_moves(s["room"]), cache.alloc_step(s["cap"])


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    kind, cache = s["case"]["kind"], s["cache"]
    if kind == "diff":
        cache.attend_diff_device(s["layer"], s["q"], s["out"], s["lam"], lse=s["lse"], start=s["start"], count=s["count"], max_count=s["max_count"], window=s["case"]["window"])
        return dict(out=s["out"], lse=s["lse"])
    if kind in ("fork", "branch"):
        cache.fork_device(s["take"], s["cut"] if s["case"]["cut"] < 100 or kind == "branch" else None)
        if kind == "fork":
            return dict(lens=cache.lens, table=cache.table, holders=cache.holders)
        cache.step_device(s["keep"], s["add"], s["step"])
        cache.copy_device(s["layer"], s["step"]["copy_src"], s["step"]["copy_dst"])
        return dict(s["step"], lens=cache.lens, table=cache.table, holders=cache.holders, **_memory(s))
    if kind == "copy":
        cache.copy_device(s["layer"], s["src"], s["dst"], src_worker=s["src_worker"])
        return _memory(s)
    cache.step_device(s["keep"], s["none"], s["step"])
    cache.compact_device(s["moves"])
    cache.copy_device(s["layer"], s["moves"]["src"], s["moves"]["dst"])
    cache.step_device(s["all"], s["add"], s["back"])
    return dict(first=s["step"]["stats"], **s["moves"], back=s["back"], lens=cache.lens, table=cache.table, holders=cache.holders, **_memory(s))


def _memory(s):
    """A layer's bytes, those of the scales as whole numbers too: nothing is computed with them, so they have to be equal."""
    return dict(k=s["k"], v=s["v"], k_scale=s["k_scale"].view(torch.int32), v_scale=s["v_scale"].view(torch.int32))


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "diff":
        return _plain_diff(s)
    if kind in ("fork", "branch"):
        _plain_fork(s, s["cut"] if c["cut"] < 100 or kind == "branch" else None)
        if kind == "fork":
            return dict(lens=s["lens"], table=s["table"], holders=_holders(s))
        step = _plain_step(s, s["keep"], s["add"])
        _plain_copy(s, step["copy_src"], step["copy_dst"])
        return dict(step, lens=s["lens"], table=s["table"], holders=_holders(s), **_memory(s))
    if kind == "copy":
        _plain_copy(s, s["src"], s["dst"], s["src_worker"])
        return _memory(s)
    first = _plain_step(s, s["keep"], s["none"])["stats"]
    moves = _plain_compact(s)
    _plain_copy(s, moves["src"], moves["dst"])
    back = _plain_step(s, s["all"], s["add"])
    return dict(first=first, **moves, back=back, lens=s["lens"], table=s["table"], holders=_holders(s), **_memory(s))


# -- plain forms of the tables ---------------------------------------------------
def _holders(s):
    """Rows that hold each block: [W, n_blocks]."""
    W, n_blocks = len(s["table"]), s["n_blocks"]
    at = torch.where(s["table"] < 0, n_blocks, s["table"]).view(W, -1).long()
    return torch.zeros((W, n_blocks + 1), dtype=torch.int32, device=DEVICE).scatter_add_(1, at, torch.ones_like(at, dtype=torch.int32))[:, :n_blocks].contiguous()


def _plain_fork(s, cut):
    lens, table, take, b = s["lens"], s["table"], s["take"].long(), s["case"]["block"]
    W, R, width = table.shape
    forked = (take >= 0) & (take < R)
    source = torch.where(forked, take, torch.arange(R, device=DEVICE))
    new = lens.gather(1, source)
    if cut is not None:
        new = torch.where(forked & (cut >= 0), torch.minimum(new, cut), new)
    rows = table.gather(1, source[:, :, None].expand(W, R, width))
    gone = torch.arange(width, device=DEVICE) >= ((new + b - 1) // b)[:, :, None]
    table.copy_(torch.where(forked[:, :, None] & gone, -1, rows))
    lens.copy_(new)


def _plain_step(s, keep, add):
    c, lens, table = s["case"], s["lens"], s["table"]
    (W, R), b, width, n_blocks, cap = lens.shape, c["block"], table.shape[2], s["n_blocks"], s["cap"]
    at = torch.arange(width, device=DEVICE)
    keep = torch.where(keep < 0, lens, torch.minimum(keep, lens))
    add = add.clamp(min=0).long()
    have = (keep + b - 1) // b
    table[at >= have[:, :, None]] = -1
    held = _holders(s)
    status = torch.zeros_like(keep)

    def refuse(which, why):
        status[which] = why
        add[which] = 0

    # a row that would write into a block that others hold too takes another in its place
    last = table.gather(2, (have - 1).clamp(min=0).long()[:, :, None])[:, :, 0]
    inside = (keep % b > 0) & (last >= 0) & (held.gather(1, last.clamp(min=0).long()) > 1)

    def needed():
        own_block = inside & (add > 0)
        return own_block, (keep + add + b - 1) // b - have + own_block

    refuse((add > 0) & ((keep + add + b - 1) // b > width), 2)
    refuse((add > 0) & (add.cumsum(1) > cap), 3)
    free = held == 0
    need = needed()[1]
    refuse((need > 0) & (need.cumsum(1) > free.sum(1, keepdim=True)), 1)
    instead, need = needed()
    # the k-th block that is taken is the k-th lowest free one
    rank = free.int().cumsum(1, dtype=torch.int32) - 1
    ids = torch.full((W, n_blocks + 1), -1, dtype=torch.int32, device=DEVICE)
    ids.scatter_(1, torch.where(free, rank, n_blocks).long(), torch.arange(n_blocks, dtype=torch.int32, device=DEVICE).expand(W, n_blocks))
    first = need.cumsum(1) - need
    begin = have - instead.to(torch.int32)
    new = (at >= begin[:, :, None]) & (at < (begin + need)[:, :, None])
    k = (first - begin)[:, :, None] + at
    table.copy_(torch.where(new, ids.gather(1, k.clamp(0, n_blocks).view(W, R * width)).view(W, R, width), table))
    total = add.sum(1)
    start = add.cumsum(1) - add
    j = torch.arange(cap, device=DEVICE).expand(W, cap).contiguous()
    row = torch.searchsorted(add.cumsum(1), j, right=True).clamp_(max=R - 1)
    pos = keep.gather(1, row) + j - start.gather(1, row)
    mine = j < total[:, None]
    pos = torch.where(mine, pos, 0)
    slot = table.view(W, R * width).gather(1, row * width + pos // b) * b + pos % b
    lens.copy_((keep + add).to(torch.int32))
    n_used = (_holders(s) > 0).sum(1)
    stats = torch.stack([lens.sum(1), n_used, n_blocks - n_used, (lens > 0).sum(1), total, (status > 0).sum(1), (status == 1).sum(1), need.sum(1)], 1)
    start = start + cap * torch.arange(W, device=DEVICE)[:, None]
    fresh = table.gather(2, (have - 1).clamp(min=0).long()[:, :, None])[:, :, 0]
    i32 = lambda x: x.to(torch.int32)
    return dict(slot=i32(torch.where(mine, slot, -1)), pos=i32(torch.where(mine, pos, -1)), start=i32(start), count=i32(add), status=status, stats=stats,
                copy_src=torch.where(instead, last, -1), copy_dst=torch.where(instead, fresh, -1))


def _plain_copy(s, src, dst, src_worker=None):
    N = s["n_blocks"]
    worker = torch.arange(len(src), device=DEVICE)[:, None].expand(src.shape)
    there = (src >= 0) & (dst >= 0)
    to = (worker * N + dst)[there]
    at = ((worker if src_worker is None else src_worker.long()) * N + src)[there]
    for name in ("k", "v", "k_scale", "v_scale"):
        s[name][to] = s[name][at]


def _plain_compact(s):
    table, n_blocks, room = s["table"], s["n_blocks"], s["room"]
    W = len(table)
    used = _holders(s) > 0
    n_used = used.sum(1, keepdim=True)
    ids = torch.arange(n_blocks, device=DEVICE)
    out = used & (ids >= n_used)  # highest first, to the lowest free ones
    into = ~used & (ids < n_used)
    src = torch.full((W, room + 1), -1, dtype=torch.int32, device=DEVICE)
    dst = src.clone()
    k_out = out.flip(1).cumsum(1).flip(1) - 1
    k_in = into.cumsum(1) - 1
    whole = ids.to(torch.int32).expand(W, n_blocks)
    src.scatter_(1, torch.where(out, k_out, room).clamp(max=room), whole)
    dst.scatter_(1, torch.where(into, k_in, room).clamp(max=room), whole)
    src, dst = src[:, :room].contiguous(), dst[:, :room].contiguous()
    to = whole.clone()
    moved = out & (k_out < room)
    to = torch.where(moved, dst.gather(1, k_out.clamp(0, room - 1)), to)
    table.copy_(torch.where(table >= 0, to.gather(1, table.clamp(min=0).view(W, -1).long()).view(table.shape), -1))
    return dict(src=src, dst=dst)


# -- 8 bits -----------------------------------------------------------------------
def _encode_blocks(x, fmt):
    """x [N, H, ...]: bytes, and the scales [N, H], powers of two."""
    scale = torch.exp2(torch.ceil(torch.log2(x.abs().flatten(2).amax(2).clamp(min=2.0 ** -60) / TOP[fmt])))
    y = x / scale.view(*scale.shape, *[1] * (x.dim() - 2))
    y = y.clamp(-TOP[fmt], TOP[fmt])
    return (y.round().to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)).view(torch.uint8), scale


def _value(code, fmt):
    return code.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()


# -- plain form of the attention ----------------------------------------------------
def _plain_diff(s):
    """The rows with a chunk, if any, and the others, each padded to their largest."""
    c = s["case"]
    q = s["q"].float()
    out, lse = torch.empty_like(q), torch.empty((*q.shape[:2], 2), device=DEVICE)
    by_count = s["lens"][0].argsort(descending=True)
    if c["chunk_rows"]:
        _padded(s, by_count[:c["chunk_rows"]], c["chunk"], q, out, lse)
    _padded(s, by_count[c["chunk_rows"]:c["rows"] - c["idle"]], c["tokens"], q, out, lse)
    return dict(out=out.to(s["q"].dtype), lse=lse)


def _padded(s, rows, n, q, out, lse):
    """Differential attention of n query tokens of each of the given rows."""
    c = s["case"]
    b, H, G, D, R = c["block"], c["heads"], c["group"], c["dim"], len(rows)
    if not R:
        return
    nb, half = _up(s["max_len"], b), D // 2
    blocks = s["table"][0, rows, :nb].clamp(min=0).long()
    k = (_value(s["k"][blocks], c["fmt"]) * s["k_scale"][blocks][..., None, None]).permute(0, 2, 1, 3, 4).reshape(R * H, nb * b, D)
    token = s["start"][rows].long()[:, None] + torch.arange(n, device=DEVICE)
    qs = q[token].view(R, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(R * H, n * G, D)
    j = torch.arange(nb * b, device=DEVICE)
    p = (s["lens"][0, rows].long()[:, None] - n + torch.arange(n, device=DEVICE))[:, None, :, None, None]
    seen = (j <= p) & (j > p - c["window"]) if c["window"] else j <= p
    maps = []
    for m in range(2):
        part = slice(m * half, (m + 1) * half)
        score = torch.bmm(qs[:, :, part].contiguous(), k[:, :, part].transpose(1, 2).contiguous()).view(R, H, n, G, nb * b) / math.sqrt(half)
        score = score.masked_fill_(~seen, -math.inf)
        top = score.amax(-1, keepdim=True)
        e = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
        del score
        total = e.sum(-1, keepdim=True)
        maps.append(e / torch.where(total > 0, total, 1.0))
        lse[..., m][token] = (top + total.log()).view(R, H, n, G).permute(0, 2, 1, 3).reshape(R, n, H * G)
        del e
    del k, qs
    lam = (s["lam"][token] if c["lam"] == "token" else s["lam"].expand(R, n, H * G)).view(R, n, H, G).permute(0, 2, 1, 3)
    weight = maps[0] - lam[..., None] * maps[1]
    del maps
    v = (_value(s["v"][blocks], c["fmt"]) * s["v_scale"][blocks][..., None, None]).permute(0, 2, 1, 4, 3).reshape(R * H, nb * b, D)
    o = torch.bmm(weight.reshape(R * H, n * G, nb * b), v)
    out[token] = o.view(R, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(R, n, H * G, D)


# -- the definition in 64 bits ----------------------------------------------------------
def exact(case, seed):
    if case["kind"] != "diff":
        return None  # whole numbers, and bytes that are copied
    s = prepare(case, seed)
    b, H, G, D, fmt = case["block"], case["heads"], case["group"], case["dim"], case["fmt"]
    if sum(n * x for n, x in zip(_counts(case), sorted(_lengths(case), reverse=True))) * H * G * D > 6e11:
        return None
    out = torch.zeros((s["T"], H * G, D), dtype=torch.float64, device=DEVICE)
    lse = torch.full((s["T"], H * G, 2), -math.inf, dtype=torch.float64, device=DEVICE)
    for r, (n, length, t0) in enumerate(zip(s["count"].tolist(), s["lens"][0].tolist(), s["start"].tolist())):
        if not n:
            continue
        ids = s["table"][0, r, :_up(length, b)].long()
        k = (_value(s["k"][ids], fmt).double() * s["k_scale"][ids].double()[..., None, None]).transpose(0, 1).reshape(H, -1, D)[:, :length]
        v = (_value(s["v"][ids], fmt).double() * s["v_scale"][ids].double()[..., None, None]).permute(1, 0, 3, 2).reshape(H, -1, D)[:, :length].contiguous()
        q = s["q"][t0:t0 + n].double().view(n, H, G, D).permute(1, 0, 2, 3).reshape(H, n * G, D)
        i, j = torch.arange(length - n, length, device=DEVICE)[:, None], torch.arange(length, device=DEVICE)
        hidden = j > i
        if case["window"]:
            hidden = hidden | (j <= i - case["window"])
        lam = s["lam"].double()
        lam = (lam[t0:t0 + n] if case["lam"] == "token" else lam.expand(n, H * G)).view(n, H, G).permute(1, 0, 2).reshape(H, n * G, 1)
        for m, (qm, km) in enumerate(zip(q.chunk(2, -1), k.chunk(2, -1))):
            z = torch.matmul(qm.contiguous(), km.transpose(1, 2).contiguous()).view(H, n, G, length) * (D // 2) ** -0.5
            z = z.masked_fill(hidden[:, None], -math.inf)
            w = torch.logsumexp(z, -1)
            a = torch.exp(z - torch.where(torch.isinf(w), 0.0, w)[..., None]).reshape(H, n * G, length)
            o = torch.matmul(a, v) * (1.0 if m == 0 else -lam)
            out[t0:t0 + n] += o.view(H, n, G, D).transpose(0, 1).reshape(n, H * G, D)
            lse[t0:t0 + n, :, m] = w.permute(1, 0, 2).reshape(n, H * G)
    return dict(out=out, lse=lse)


# -- what a pass cannot do without ------------------------------------------------------
def work(case):
    lens, b, W, R = _lengths(case), case["block"], case["workers"], case["rows"]
    kind = case["kind"]
    if kind in ("fork", "branch"):
        n = R - case["idle"]
        kept = [(x * case["cut"] + 99) // 100 for x in lens[:n]]
        entries = sum(_up(x, b) for x in kept)
        own_rows = sum(_up(x, b) for x in kept[::case["family"]])  # of a block that several rows hold: one count, read and written
        table = 16 * R + 8 * entries + 8 * own_rows
        if kind == "fork":
            return dict(bytes=W * table, flops=0)
        instead = sum(x % b > 0 for x in kept)  # blocks that go with a row's next token
        cells = 2 * case["heads"] * (case["dim"] * b + 4)
        return dict(bytes=W * (table + 40 * R + 8 * R * case["add"] + _blocks(case)[0] / 8 + 2 * instead * cells), flops=0)
    cells = case["heads"] * case["dim"]
    if kind == "copy":
        moved = W * sum(_up(x, b) for x in sorted(lens)[-case["take"]:])
        return dict(bytes=moved * (12 + 4 * (cells * b + 4 * case["heads"])), flops=0)
    if kind == "compact":
        held, stay = sum(_up(x, b) for x in lens), (1 - case["leave"])
        n_blocks = _blocks(case)[0]
        moved = min(stay * held * (1 - stay * held / n_blocks), max(1, n_blocks * case["room"] // 100))  # blocks in use at or above their number, of those scattered evenly
        # lens, keep, add of two steps and their outputs; places in the token lists; a bit a block; entries read, cleared and written; moves
        return dict(bytes=W * (2 * 28 * R + 16 * sum(lens) + n_blocks / 2 + 8 * held + moved * (8 + 4 * (cells * b + 4 * case["heads"]))), flops=0)
    counts = _counts(case)
    read = pairs = 0
    for n, x in zip(counts, sorted(lens, reverse=True)):
        seen = [min(p + 1, case["window"] or p + 1) for p in range(max(0, x - n), x)]
        pairs += sum(seen)
        read += min(x, (case["window"] or x) + n - 1)
    scales = 2 * 4 * case["heads"] * read / b
    per_token = case["group"] * (2 * cells * 2 + 8 * case["heads"]) + (4 * case["heads"] * case["group"] if case["lam"] == "token" else 0)
    # two maps over half of the channels each, one product with the values
    return dict(bytes=2 * cells * read + scales + sum(counts) * per_token, flops=4 * cells * case["group"] * pairs)
