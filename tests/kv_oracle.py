"""Plain implementations of what include/br_kv.h defines, in whole numbers and 64 bits, one request at a time."""
import math

import numpy as np

TOP = {"int8": 127.0, "fp8": 448.0}
LEAST = -100


def _e4m3_values():
    v = np.zeros(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        x = math.nan if e == 15 and m == 7 else (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
        v[c] = -x if s else x
    return v


E4M3 = _e4m3_values()


def decode(codes, fmt):
    codes = np.asarray(codes, np.uint8)
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[codes]


def encode(x, fmt):
    """To the nearest value of the format, ties to even codes; |x| <= TOP."""
    x = np.asarray(x, np.float64)
    if fmt == "int8":
        return np.rint(x).astype(np.int8).view(np.uint8)
    pos = E4M3[:127]  # codes 0..126 ascend
    a = np.abs(x)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def scale_for(top, fmt):
    if top == 0:
        return 2.0 ** LEAST
    e = math.ceil(math.log2(top / TOP[fmt]))
    while top > TOP[fmt] * 2.0 ** e:
        e += 1
    while top <= TOP[fmt] * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** max(e, LEAST)


class Tables:
    """One worker's block tables (br_kv_step), row by row."""

    def __init__(self, rows, block, n_blocks, max_blocks, lens=None, table=None):
        self.B, self.b, self.N, self.M = rows, block, n_blocks, max_blocks
        self.lens = [0] * rows if lens is None else [int(x) for x in lens]
        self.rows = [[] for _ in range(rows)] if table is None else [[int(x) for x in t[:self.up(n)]] for t, n in zip(table, self.lens)]

    def up(self, n):
        return -(-n // self.b)

    def step(self, keep, add, cap):
        B = self.B
        kp = [n if k < 0 else min(int(k), n) for k, n in zip(keep, self.lens)]
        want, status = [max(0, int(a)) for a in add], [0] * B
        for r in range(B):
            del self.rows[r][self.up(kp[r]):]
        for r in range(B):
            if want[r] and self.up(kp[r] + want[r]) > self.M:
                want[r], status[r] = 0, 2
        asked = 0
        for r in range(B):
            asked += want[r]
            if want[r] and asked > cap:
                want[r], status[r] = 0, 3
        used = {i for row in self.rows for i in row if i >= 0}
        free = [i for i in range(self.N) if i not in used]
        needed = 0
        for r in range(B):
            need = self.up(kp[r] + want[r]) - self.up(kp[r])
            needed += need
            if need and needed > len(free):
                want[r], status[r] = 0, 1
        slot, pos, start, taken = [], [], [], 0
        for r in range(B):
            start.append(len(slot))
            for p in range(kp[r], kp[r] + want[r]):
                if p // self.b == len(self.rows[r]):
                    self.rows[r].append(free[taken])
                    taken += 1
                i = self.rows[r][p // self.b]
                slot.append(i * self.b + p % self.b if i >= 0 else -1)
                pos.append(p)
            self.lens[r] = kp[r] + want[r]
        n = len(slot)
        n_used = sum(i >= 0 for row in self.rows for i in row)
        stats = [sum(self.lens), n_used, self.N - n_used, sum(x > 0 for x in self.lens), n, sum(x > 0 for x in status), sum(x == 1 for x in status), taken]
        return dict(slot=slot + [-1] * (cap - n), pos=pos + [-1] * (cap - n), start=start, count=want, status=status, stats=stats)

    def table(self):
        return np.array([row + [-1] * (self.M - len(row)) for row in self.rows], np.int32)


def append(k, scale, x, slot, block_tokens, fmt):
    """x [T, H, D] (any float) into k [blocks, H, b, D] (codes), scale [blocks, H], in place."""
    T, H, _ = x.shape
    t = 0
    while t < T:
        s = int(slot[t])
        n = 1
        if s < 0 or s >= k.shape[0] * block_tokens:
            t += 1
            continue
        while t + n < T and (s + n) % block_tokens and int(slot[t + n]) == s + n:
            n += 1
        blk, off = divmod(s, block_tokens)
        for h in range(H):
            y = x[t:t + n, h].astype(np.float64)
            old = float(scale[blk, h])
            if not np.isfinite(y).all() or (off and not math.isfinite(old)):
                scale[blk, h], k[blk, h, off:off + n] = math.nan, 0
                continue
            now = scale_for(np.abs(y).max(), fmt)
            if off:
                now = max(now, 2.0 ** math.ceil(math.log2(old)) if old > 0 else 0.0)
                k[blk, h, :off] = encode(decode(k[blk, h, :off], fmt) * (old / now), fmt)
            scale[blk, h] = now
            k[blk, h, off:off + n] = encode(y / now, fmt)
        t += n


def attend(q, k, v, ks, vs, table, lens, start, count, group, block, fmt, window=0, scale=None, n_tokens=None):
    """q [T, Hq, D]; k [blocks, H, b, D], v [blocks, H, D, b] codes; table [R, M], lens [R] of one worker.
    Returns (out, lse, A, S, Z) in 64 bits; A: sums of weights times magnitudes, S: the largest sum of magnitudes of a score's terms, Z: sums of
    magnitudes of codes, times the largest scale of the row's values."""
    T, Hq, D = q.shape
    H = Hq // group
    scale = D ** -0.5 if scale is None else scale
    out, lse = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan)
    A, S, Z = np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros((T, Hq, D))
    q = np.asarray(q, np.float64)
    N = k.shape[0]
    for r in range(len(lens)):
        L = min(max(int(lens[r]), 0), table.shape[1] * block)
        nb = -(-L // block)
        ids = np.asarray(table[r][:nb], np.int64)
        ok = (ids >= 0) & (ids < N)
        safe = np.where(ok, ids, 0)
        kk = (decode(k[safe], fmt) * ks[safe].astype(np.float64)[:, :, None, None]).transpose(1, 0, 2, 3).reshape(H, nb * block, D)[:, :L]
        vv = (decode(v[safe], fmt) * vs[safe].astype(np.float64)[:, :, None, None]).transpose(1, 0, 3, 2).reshape(H, nb * block, D)[:, :L]
        vc = np.abs(decode(v[safe], fmt)).transpose(1, 0, 3, 2).reshape(H, nb * block, D)[:, :L]
        vtop = np.nanmax(np.abs(vs[safe][ok]).astype(np.float64), axis=0, initial=0.0)
        there = np.repeat(ok, block)[:L]
        for i in range(int(count[r])):
            t, p = int(start[r]) + i, L - int(count[r]) + i
            if t < 0 or t >= T:
                continue
            j = np.arange(L)
            see = there & (j <= p)
            if window:
                see &= j > p - window
            for hq in range(Hq):
                h = hq // group
                if not see.any():
                    out[t, hq], lse[t, hq] = 0.0, -math.inf
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (kk[h][see] @ q[t, hq])
                    S[t, hq] = np.max(abs(scale) * (np.abs(kk[h][see]) @ np.abs(q[t, hq])))
                    m = s.max()
                    w = np.exp(s - m)
                    out[t, hq] = (w @ vv[h][see]) / w.sum()
                    Z[t, hq] = vtop[h] * vc[h][see].sum(0)
                    A[t, hq] = (w @ np.abs(vv[h][see])) / w.sum()
                    lse[t, hq] = m + math.log(w.sum()) if np.isfinite(m) else math.nan
    return out, lse, A, S, Z
