"""The 8-bit cache and the logits functions in 64 bits, from their definitions; nothing here calls the library."""
import math

import numpy as np
import torch


def e4m3_round(x):
    """float64 -> the nearest e4m3 value, ties to even; |x| <= 448."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    return np.rint(x / step) * step


def scale_for(top):
    """Smallest power of two s >= 2^-100 with top <= 448 s."""
    if top == 0:
        return 2.0 ** -100
    m, e = math.frexp(top)              # top = m 2^e, m in [0.5, 1); 448 = 0.875 x 2^9
    return 2.0 ** max(-100, e - 9 + (1 if m > 0.875 else 0))


class Cache:
    """[layers, heads, capacity, d] values of one of K and V as the cache holds them, block by block."""

    def __init__(self, layers, heads, capacity, d, block):
        self.values = np.zeros((layers, heads, capacity, d))
        self.scale = np.zeros((layers, heads, -(-capacity // block)))
        self.block = block

    def write(self, rows, start):
        """rows [layers, heads, n, d]; a row of None entries (NaN in `skip`) is not supported here: see `append`."""
        self.append(rows, start, list(range(rows.shape[2])))

    def append(self, src, start, path):
        """Rows path[i] of src enter at start + i; an entry outside src is skipped."""
        n, block = len(path), self.block
        if n == 0:
            return
        ok = [0 <= r < src.shape[2] for r in path]
        for y in range(src.shape[0]):
            for h in range(src.shape[1]):
                for b in range(start // block, (start + n - 1) // block + 1):
                    lo, hi = max(start, b * block), min(start + n, (b + 1) * block)
                    fresh = [(p, path[p - start]) for p in range(lo, hi) if ok[p - start]]
                    x = np.array([src[y, h, r] for _, r in fresh]) if fresh else np.zeros((0, src.shape[3]))
                    finite = np.abs(x[np.isfinite(x)])
                    scale = scale_for(finite.max() if finite.size else 0.0)
                    if b * block < start:
                        scale = max(scale, self.scale[y, h, b])
                        old = self.values[y, h, b * block:start]
                        self.values[y, h, b * block:start] = e4m3_round(old / scale) * scale
                    self.scale[y, h, b] = scale
                    for (p, _), row in zip(fresh, x):
                        v = np.where(np.isinf(row), np.sign(row) * 448.0 * scale, row)
                        self.values[y, h, p] = np.where(np.isnan(v), np.nan, e4m3_round(np.nan_to_num(v) / scale) * scale)


def visible(parent):
    n = len(parent)
    seen = np.zeros((n, n), dtype=bool)
    for i in range(n):
        if 0 <= parent[i] < i:
            seen[i] = seen[parent[i]]
        seen[i, i] = True
    return seen


def attention(q, k, v, k_tree, v_tree, parent, scale, row_chunks=None):
    """q [T, Hq, d], k / v [Hkv, L, d] float64 -> out [T, Hq, d], lse [Hq, T], magnitude [T, Hq] of what is summed (largest
    column of sum p |v|), spread [Hq, T] (largest scale sum |q k|), scores of every row [T, chunks]."""
    t, hq, d = q.shape
    hkv, n = k.shape[0], k.shape[1]
    g = hq // hkv
    seen = torch.from_numpy(visible(parent))
    out, mag = torch.zeros(t, hq, d, dtype=torch.float64), torch.zeros(t, hq, dtype=torch.float64)
    lse, spread = torch.zeros(hq, t, dtype=torch.float64), torch.zeros(hq, t, dtype=torch.float64)
    mass = torch.zeros(t, n, dtype=torch.float64)
    for h in range(hq):
        keys = torch.cat([k[h // g], k_tree[h // g]])
        vals = torch.cat([v[h // g], v_tree[h // g]])
        s = q[:, h] @ keys.T * scale
        s[:, n:][~seen] = -math.inf
        lse[h] = torch.logsumexp(s, dim=1)
        p = torch.exp(s - lse[h][:, None])
        out[:, h] = p @ vals
        mag[:, h] = (p @ vals.abs()).amax(dim=1)
        spread[h] = (q[:, h].abs() @ keys.abs().T).amax(dim=1) * scale
        mass += p[:, :n]
    scores = None
    if row_chunks:
        scores = torch.stack([c.mean(dim=1) for c in (mass / hq).split(row_chunks, dim=1)], dim=1)
    return out, lse, mag, spread, scores


def random_tree(n, rng):
    return np.array([-1] + [int(rng.integers(-1, i)) for i in range(1, n)], dtype=np.int32)
