"""Routed requests on their workers: the router binds requests, the workers hold their tokens in 8-bit caches and attend over them.

    python examples/decode_workers.py [--steps 64] [--heads 2] [--group 4] [--fmt fp8] [--policy]

One cluster of G data-parallel workers (all on this GPU).  Each decode step:
  1. the round: BR-0 binds waiting requests to workers (binding.Router);
  2. their prompts' keys and values move into the workers' caches (kv.KvCache: tables, append), requests that have finished
     leave them;
  3. every active request decodes a token: its key and value go into the cache, its query attends over all of it;
  4. the router's decode step.
The cached tokens of a worker are the load L_g that the router balances: both are compared in every step.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class Rows:
    """Which request sits in which row of which worker, on the host: what a worker's scheduler keeps."""

    def __init__(self, G: int, B: int):
        self.rem = np.zeros((G, B), np.int64)   # decode steps to run; 0: free
        self.gone = np.zeros((G, B), bool)      # finished, tokens still cached

    def admit(self, g: int, out_len: int) -> int:
        row = int(np.flatnonzero(self.rem[g] == 0)[0])
        self.rem[g, row] = max(1, out_len)
        return row


def run(steps: int = 64, G: int = 4, B: int = 16, heads: int = 2, group: int = 4, dim: int = 128, fmt: str = "fp8", block: int = 16, seed: int = 0, rate: float = 2.0,
        prompt_hi: int = 512, policy: bool = False):
    """One dict per step: loads of the workers, requests, the time of the step's attention in ms."""
    import torch
    from paper_2605_06113_amd import binding, kv, workloads as wl

    cfg = wl.config("c1", G=G, B=B, max_wait=64, token_cap=0, token_watermark=0, arrival_rate=rate, prompt_hi=prompt_hi, out_mu=float(np.log(30.0)), out_hi=200,
                    init_active_total=0, init_waiting=0, seed=seed)
    router = binding.Router(cfg)
    trace = wl.arrival_trace(cfg, steps=steps)
    width = -(-(prompt_hi + 201) // block)
    blocks = B * width
    cache = kv.KvCache(kv.KvConfig(n_workers=G, rows=B, block_tokens=block, n_blocks=blocks, max_blocks=width, n_kv_heads=heads, n_q_heads=heads * group, head_dim=dim, fmt=fmt))
    layer = cache.new_layer()
    prompts, decode = cache.alloc_step(B * prompt_hi), cache.alloc_step(B)
    rows, length = Rows(G, B), {}
    rng = torch.Generator("cuda").manual_seed(seed)
    randn = lambda n, h: torch.randn((n, h, dim), generator=rng, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    q_out = torch.empty((G * B, heads * group, dim), dtype=torch.bfloat16, device="cuda")
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    dev = lambda a: torch.as_tensor(np.ascontiguousarray(a, np.int32)).to("cuda")
    log = []
    for k in range(steps):
        arr = trace.step(k)
        for i in range(int(arr.count[0])):
            length[int(arr.id[0, i])] = (int(arr.s[0, i]), int(arr.o[0, i]))
        # 1. the round
        out = router.route_baseline(arr, binding.POLICY["rr"]) if policy else router.route_step(arr, scores=False)
        load = router.state()["L"][0]
        # 2. finished requests leave, prompts come
        keep, add = np.where(rows.gone, 0, -1), np.zeros((G, B), np.int64)
        rows.gone[:] = False
        for pos in np.flatnonzero(out["assign"][0] >= 0):
            g, (s, o) = int(out["assign"][0, pos]), length[int(out["assign_id"][0, pos])]
            add[g, rows.admit(g, o)] = s
        cache.step_device(dev(keep), dev(add), prompts)
        n = G * prompts["slot"].shape[1]
        if add.any():
            cache.append_device(layer, randn(n, heads), randn(n, heads), prompts["slot"])
        held = prompts["stats"].cpu().numpy()
        assert (held[:, kv.ST["refused"]] == 0).all() and (held[:, kv.ST["tokens"]] == load).all(), "a worker's cached tokens are its load"
        # 3. a token for every active request
        active = rows.rem > 0
        cache.step_device(dev(np.full((G, B), -1)), dev(active), decode)
        cache.append_device(layer, randn(G * B, heads), randn(G * B, heads), decode["slot"])
        q = randn(G * B, heads * group)
        begin.record()
        cache.attend_device(layer, q, q_out, start=decode["start"], count=decode["count"])
        end.record()
        # 4. the router's decode step
        router.advance(1)
        rows.rem[active] -= 1
        rows.gone = active & (rows.rem == 0)
        after = router.state()["L"][0]
        cached = cache.lens.cpu().numpy()
        assert (np.where(rows.gone, 0, cached).sum(1) == after).all()
        end.synchronize()
        used = torch.zeros(G * B, dtype=torch.bool, device="cuda")
        used[(decode["start"][decode["count"] > 0]).long()] = True
        assert bool(torch.isfinite(q_out[used].float()).all())
        log.append(dict(step=k, loads=after.tolist(), requests=int(active.sum()), ms=begin.elapsed_time(end)))
    router.close(), cache.close()
    return log


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--heads", type=int, default=2)
    ap.add_argument("--group", type=int, default=4)
    ap.add_argument("--fmt", choices=("fp8", "int8"), default="fp8")
    ap.add_argument("--policy", action="store_true", help="round robin instead of BR-0")
    a = ap.parse_args()
    log = run(steps=a.steps, heads=a.heads, group=a.group, fmt=a.fmt, policy=a.policy)
    for r in log[:: max(1, len(log) // 16)]:
        print(f"step {r['step']:4d}  requests {r['requests']:3d}  loads {r['loads']}  spread {max(r['loads']) - min(r['loads']):6d}  attention {r['ms'] * 1e3:7.1f} us")
    print(f"mean spread {np.mean([max(r['loads']) - min(r['loads']) for r in log]):.0f} tokens, mean attention {1e3 * np.mean([r['ms'] for r in log]):.1f} us")


if __name__ == "__main__":
    main()
