"""A step of rows that hold blocks together, captured and replayed on the GPU: every row's tokens are read back and have to be those that were written for it, and the
attention is that of these tokens, written down without any sharing, in 64 bits, each output with its own bound."""
import math

import numpy as np
import pytest

from paper_2605_06113_amd import kv
from tests import test_kv_pages_gpu as pages
from tests.test_kv_gpu import _check_attention, _say, _torch
from tests.test_kv_shared_gpu import _families, _i32

pytestmark = pytest.mark.gpu


class Rows(pages.Content):
    """Numbered tokens in a shared cache with query heads, on a stream of its own."""

    def __init__(self, dims, group, cap, stream):
        torch = _torch()
        W, B, b, N, M, H, D = dims
        self.dims, self.group, self.cap = dims, group, cap
        cfg = kv.KvConfig(n_workers=W, rows=B, block_tokens=b, n_blocks=N, max_blocks=M, n_kv_heads=H, n_q_heads=H * group, head_dim=D, fmt="int8", shared=True)
        self.cache = kv.KvCache(cfg, stream=stream)
        self.layer, self.out = self.cache.new_layer(), self.cache.alloc_step(cap)
        self.layer.k.fill_(99), self.layer.v.fill_(98), self.layer.k_scale.fill_(float("nan")), self.layer.v_scale.fill_(float("nan"))
        self.rows, self.next = [[[] for _ in range(B)] for _ in range(W)], 1
        torch.cuda.synchronize()

    def attention(self, q, window):
        """What _check_attention compares with, from the numbers of each row's tokens alone."""
        W, B, b, N, M, H, D = self.dims
        T, Hq = q.shape[:2]
        out, lse, A, S, Z = np.zeros((T, Hq, D)), np.full((T, Hq), -math.inf), np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros((T, Hq, D))
        for w in range(W):
            for r, tags in enumerate(self.rows[w]):
                k, v = (x.astype(np.float64) for x in pages._vectors(tags[-window:] if window else tags, H, D))
                t = w * B + r
                for hq in range(Hq if tags else 0):
                    kh, vh = k[:, hq // self.group], v[:, hq // self.group]
                    s = D ** -0.5 * (kh @ q[t, hq])
                    e = np.exp(s - s.max())
                    out[t, hq], A[t, hq], Z[t, hq] = e @ vh / e.sum(), e @ np.abs(vh) / e.sum(), np.abs(vh).sum(0)
                    lse[t, hq], S[t, hq] = s.max() + math.log(e.sum()), (D ** -0.5 * (np.abs(kh) @ np.abs(q[t, hq]))).max()
        return out, lse, A, S, Z


@pytest.mark.parametrize("case", [  # workers, rows, block, blocks, entries, heads, width, query heads each, family, members, window
    (1, 12, 16, 400, 60, 2, 64, 4, 4, 4, 0), (2, 9, 32, 200, 30, 1, 128, 8, 3, 3, 0), (1, 16, 64, 120, 14, 2, 96, 2, 8, 16, 0), (1, 10, 16, 400, 60, 1, 192, 16, 5, 4, 0),
    (1, 12, 128, 60, 7, 1, 256, 4, 6, 6, 0), (1, 70, 16, 2500, 60, 1, 64, 3, 7, 7, 0), (1, 12, 16, 400, 60, 2, 64, 4, 4, 4, 130)], ids=str)
def test_steps_of_families(case):
    """Samples go back to their prompt now and then, get a token each, write into what they held together: one graph, replayed with eager work between."""
    torch = _torch()
    *dims, group, F, members, window = case
    W, B, b, N, M, H, D = dims
    _say("families' steps", case)
    side, rng = torch.cuda.Stream(), np.random.default_rng(B + D)
    c = Rows(dims, group, max(B, B * 300), side)
    one_each = c.cache.alloc_step(B)
    lead, every, one = _families(B, F).repeat(W, 0), np.full((W, B), -1), np.ones((W, B), int)
    cut = np.where(np.arange(B) % F, 230, -1)[None].repeat(W, 0)
    dev = [_i32(x) for x in (lead, cut, every, one)]
    x = torch.zeros((2, W * B, H, D), dtype=torch.float16, device="cuda:0")
    q, out, lse = torch.zeros((W * B, H * group, D), dtype=torch.bfloat16, device="cuda:0"), torch.zeros((W * B, H * group, D), dtype=torch.bfloat16, device="cuda:0"), torch.zeros((W * B, H * group), device="cuda:0")
    torch.cuda.synchronize()

    def run():
        c.cache.fork_device(dev[0], dev[1])
        c.cache.step_device(dev[2], dev[3], one_each)
        c.cache.copy_device(c.layer, one_each["copy_src"], one_each["copy_dst"])
        c.cache.append_device(c.layer, x[0], x[1], one_each["slot"])
        c.cache.plan_device(dev[0], members, start=one_each["start"], count=one_each["count"])
        c.cache.attend_shared_device(c.layer, q, out, lse=lse, window=window)

    def prepare():
        """The next tokens and queries, and the rows as they will be."""
        for rows in c.rows:
            old = [list(r) for r in rows]
            for r in range(B):
                rows[r] = old[r // F * F][:230] if r % F else old[r]
        tags = []
        for rows in c.rows:
            for row in rows:
                row.append(c.next), tags.append(c.next)
                c.next += 1
        for k, part in enumerate(pages._vectors(tags, H, D)):
            x[k].copy_(torch.tensor(np.ascontiguousarray(part), dtype=torch.float16))
        # (scores of a few units apart: keys go up to 127)
        q.copy_(torch.tensor(rng.normal(size=q.shape) / 40, dtype=torch.bfloat16))
        out.fill_(3.0), lse.fill_(3.0)

    def check(tag):
        assert not bool(one_each["status"].any()), tag
        c.check((case, tag))
        _check_attention((case, tag), c.cache, q, out, lse, c.attention(q.double().cpu().numpy(), window), "bfloat16")

    with torch.cuda.stream(side):
        c.step(np.zeros((W, B), int), np.where(np.arange(B) % F, 3, 170 + 7 * (np.arange(B) // F))[None].repeat(W, 0))
        prepare()
        run()
        check("eager")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    with torch.cuda.stream(side):
        for turn in range(4):
            prepare()
            graph.replay()
            check(("replay", turn))
            if turn == 1:  # one prompt is done, its samples go on; another begins in its row
                keep = every.copy()
                keep[:, 0] = 0
                c.step(keep, np.where(np.arange(B) == 0, 200, np.where(np.arange(B) % F == 1, 20, 0))[None].repeat(W, 0))
                c.compact(N)
                c.check((case, "between"))
    c.cache.close()
