"""Plain statement of differential attention over the 8-bit cache (include/br_kv.h), in 64 bits."""
import numpy as np

from tests import kv_oracle as ko


def attend_diff(q, k, v, ks, vs, table, lens, start, count, lam, group, block, fmt, window=0, scale=None):
    """As kv_oracle.attend; lam [T, Hq].  The map of a half of the channels is that of queries that are 0 in the other.
    Returns out, lse [T, Hq, 2], and of each map [2]: o, A, S, Z of kv_oracle.attend."""
    half = q.shape[2] // 2
    scale = half ** -0.5 if scale is None else scale
    maps = []
    for m in range(2):
        one = np.zeros_like(q)
        one[..., m * half:(m + 1) * half] = q[..., m * half:(m + 1) * half]
        maps.append(ko.attend(one, k, v, ks, vs, table, lens, start, count, group, block, fmt, window=window, scale=scale))
    o1, o2 = maps[0][0], maps[1][0]
    lse = np.stack([maps[0][1], maps[1][1]], -1)
    nothing = (lse[..., 0] == -np.inf)[..., None]
    with np.errstate(invalid="ignore"):
        out = np.where(nothing, 0.0, o1 - np.asarray(lam, np.float64)[..., None] * o2)
    return dict(out=out, lse=lse, o=np.stack([o1, o2]), A=np.stack([m[2] for m in maps]), S=np.stack([m[3] for m in maps]), Z=np.stack([m[4] for m in maps]))
