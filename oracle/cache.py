"""Oracle for the language model's key/value cache -- test infrastructure.

A pruned sequence leaves the keys and values of its kept tokens in a cache that
later tokens read (the cache whose size the pruning cuts, section "Efficiency
Analysis").  Plain float64 forms of

* the head norms and the rotation by positions of several axes;
* the 4-bit format of a cached block of 32 values;
* a paged cache: rows in, rows out;
* causal attention over it, with a sliding window and first tokens that stay
  visible, key/value heads shared by query heads.

Everything is written one row, one head or one block at a time.
"""
import math

import numpy as np

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def rope_axes(sections, interleaved: bool):
    """The position axis of each rotated pair."""
    if not interleaved:
        return [a for a, s in enumerate(sections) for _ in range(s)]
    left, out = list(sections), []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                out.append(a)
    return out


def qk_norm_rope(x, pos, g, rot: int, sections, interleaved=False, theta=10000.0, eps=1e-6):
    """x [R, H, d], pos [axes, R]: each head divided by its root mean square
    and scaled by g [d] (None: left as it is), then pairs (i, i + rot/2)
    turned by pos[axis(i)] theta^(-2i/rot)."""
    x = np.asarray(x, np.float64).copy()
    if g is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(g, np.float64)
    out = x.copy()
    for i, a in enumerate(rope_axes(sections, interleaved)):
        t = np.asarray(pos[a], np.float64) * float(theta) ** (-2.0 * i / rot)
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        out[..., i] = x[..., i] * c - x[..., i + rot // 2] * s
        out[..., i + rot // 2] = x[..., i + rot // 2] * c + x[..., i] * s
    return out


def mxfp4_block(x):
    """Codes (0..15) and scale byte of 32 values."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return [0] * len(x), 255
    big, e = float(np.max(np.abs(x))), -126
    while big > 7.0 * 2.0 ** e and e < 125:   # 6 * 2^125 is the largest value that bf16 holds of the levels'
        e += 1
    codes = []
    for v in x:
        y = abs(v) / 2.0 ** e
        off = [abs(y - lv) for lv in LEVELS]
        near = [c for c in range(8) if off[c] == min(off)]
        c = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
        codes.append(c | (8 if math.copysign(1.0, v) < 0 else 0))
    return codes, e + 127


def mxfp4_values(codes, scale: int):
    if scale == 255:
        return np.full(len(codes), np.nan)
    return np.array([(-1.0 if c & 8 else 1.0) * LEVELS[c & 7] * 2.0 ** (scale - 127) for c in codes])


def mxfp4_rows(x):
    """What the 4-bit cache holds for rows x [..., d]."""
    x = np.asarray(x, np.float64)
    flat = x.reshape(-1, 32)
    return np.stack([mxfp4_values(*mxfp4_block(b)) for b in flat]).reshape(x.shape)


class PagedCache:
    """Pages of `page` tokens; each token's K and V are [heads, d] rows."""

    def __init__(self, n_pages: int, page: int, table, mxfp4=False):
        self.n_pages, self.page, self.table, self.mxfp4, self.rows = n_pages, page, table, mxfp4, {}

    def place(self, b: int, j: int):
        if j < 0 or j >= len(self.table[b]) * self.page:
            return None
        p = int(self.table[b][j // self.page])
        return (p, j % self.page) if 0 <= p < self.n_pages else None

    def length(self, b: int, lens) -> int:
        return max(0, min(int(lens[b]), len(self.table[b]) * self.page))

    def append(self, lens, off, k, v):
        for b in range(len(off) - 1):
            n = off[b + 1] - off[b]
            for i in range(n):
                at = self.place(b, self.length(b, lens) - n + i)
                if at is not None:
                    r = off[b] + i
                    self.rows[at] = tuple(mxfp4_rows(x[r]) if self.mxfp4 else np.asarray(x[r], np.float64) for x in (k, v))

    def token(self, b: int, j: int, lens):
        at = self.place(b, j) if 0 <= j < self.length(b, lens) else None
        return None if at is None else self.rows.get(at)

    def attention(self, lens, off, q, scale: float, window=0, sinks=0):
        """(out, spread): out [rows, heads, d] and sum_j p_j |v_j| of the same
        shape, against which rounding errors are measured."""
        q = np.asarray(q, np.float64)
        out, spread = np.zeros_like(q), np.zeros_like(q)
        for b in range(len(off) - 1):
            n, L = off[b + 1] - off[b], self.length(b, lens)
            held = {j: self.token(b, j, lens) for j in range(L)} if n else {}
            for i in range(n):
                me = L - n + i
                see = [j for j in range(0, me + 1)
                       if held[j] is not None and (window == 0 or me - j < window or j < sinks)]
                if not see:
                    continue
                K = np.stack([held[j][0] for j in see])
                V = np.stack([held[j][1] for j in see])
                G = q.shape[1] // K.shape[1]
                for h in range(q.shape[1]):
                    z = K[:, h // G] @ q[off[b] + i, h] * scale
                    p = np.exp(z - z.max())
                    p /= p.sum()
                    out[off[b] + i, h] = p @ V[:, h // G]
                    spread[off[b] + i, h] = p @ np.abs(V[:, h // G])
        return out, spread
