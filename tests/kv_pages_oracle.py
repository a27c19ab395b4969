"""Plain statement of what include/br_kv.h says of blocks that several rows hold: one worker's tables, row by row."""
from collections import Counter

from tests import kv_oracle as ko


class SharedTables(ko.Tables):
    def holders(self):
        c = Counter(i for row in self.rows for i in row if i >= 0)
        return [c[i] for i in range(self.N)]

    def fork(self, frm, length=None):
        rows, lens = [list(r) for r in self.rows], list(self.lens)
        for r in range(self.B):
            f = int(frm[r])
            if not 0 <= f < self.B:
                continue
            n = lens[f]
            if length is not None and length[r] >= 0:
                n = min(n, int(length[r]))
            self.lens[r], self.rows[r] = n, rows[f][:self.up(n)]

    def step(self, keep, add, cap):
        B = self.B
        kp = [n if k < 0 else min(int(k), n) for k, n in zip(keep, self.lens)]
        want, status = [max(0, int(a)) for a in add], [0] * B
        for r in range(B):
            del self.rows[r][self.up(kp[r]):]
        held = self.holders()
        inside = [kp[r] % self.b > 0 and self.rows[r][-1] >= 0 and held[self.rows[r][-1]] > 1 for r in range(B)]
        for r in range(B):
            if want[r] and self.up(kp[r] + want[r]) > self.M:
                want[r], status[r] = 0, 2
        asked = 0
        for r in range(B):
            asked += want[r]
            if want[r] and asked > cap:
                want[r], status[r] = 0, 3
        free = [i for i in range(self.N) if not held[i]]
        needed = 0
        for r in range(B):
            need = self.up(kp[r] + want[r]) - self.up(kp[r]) + (inside[r] and want[r] > 0)
            needed += need
            if need and needed > len(free):
                want[r], status[r] = 0, 1
        slot, pos, start, taken = [], [], [], 0
        src, dst = [-1] * B, [-1] * B
        for r in range(B):
            start.append(len(slot))
            if want[r] and inside[r]:
                src[r], dst[r] = self.rows[r][-1], free[taken]
                self.rows[r][-1] = free[taken]
                taken += 1
            for p in range(kp[r], kp[r] + want[r]):
                if p // self.b == len(self.rows[r]):
                    self.rows[r].append(free[taken])
                    taken += 1
                i = self.rows[r][p // self.b]
                slot.append(i * self.b + p % self.b if i >= 0 else -1)
                pos.append(p)
            self.lens[r] = kp[r] + want[r]
        n, n_used = len(slot), sum(x > 0 for x in self.holders())
        stats = [sum(self.lens), n_used, self.N - n_used, sum(x > 0 for x in self.lens), n, sum(x > 0 for x in status), sum(x == 1 for x in status), taken]
        return dict(slot=slot + [-1] * (cap - n), pos=pos + [-1] * (cap - n), start=start, count=want, status=status, stats=stats, copy_src=src, copy_dst=dst)

    def compact(self, n):
        held = self.holders()
        u = sum(x > 0 for x in held)
        out = [i for i in range(self.N - 1, u - 1, -1) if held[i]]
        into = [i for i in range(u) if not held[i]]
        assert len(out) == len(into)
        pairs = list(zip(out, into))[:n]
        to = dict(pairs)
        self.rows = [[to.get(i, i) for i in row] for row in self.rows]
        more = [-1] * (n - len(pairs))
        return dict(src=[a for a, _ in pairs] + more, dst=[b for _, b in pairs] + more)
