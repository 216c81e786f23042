"""The key/value cache and the head rotation on the GPU against the cache
oracle (float64), on the same stored inputs.

Bars, from the arithmetic.  u = eps/2 of a type (bf16 2^-8, float32 2^-24).
Rotation: two float32 products and a sum, the norm's sum of head_dim squares
(half of its relative error goes through the root), the angle's float32 rest (a
few 2^-24 of a turn) and one rounding to the type: u |y| + 32 * 2^-24 * (|a| + |b|)
with (a, b) the normed pair.  Rows in and out of the cache: exact, both formats
(a 4-bit value is a function of the bf16 inputs, and fits bf16).  Attention: a
probability enters the second product rounded to bf16 (u), its score carries at
most (head_dim + 2) 2^-24 sum |q k| scale, and the output is rounded once: with
spread = sum p |v|,
  u |o| + spread (u + 2 * score error + 2^-14),
where 2^-14 covers the exponential (1 ulp of its argument's range, |z| < 2^8) and
the float32 sums.
"""
import numpy as np
import pytest
import torch

import oracle.cache as oc
from gpu_util import announce, device

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _mp():
    import paper_2608_06411_amd as mp
    return mp


def _f64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------- rotation
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,Hq,Hk,dh,rot,sec,mixed,norm", [
    (1, 32, 32, 128, 128, [64], False, False),
    (7, 28, 4, 128, 128, [16, 24, 24], False, True),
    (65, 5, 1, 128, 64, [3, 20, 9], True, True),
    (130, 3, 3, 64, 64, [8, 12, 12], True, False),
    (33, 14, 2, 64, 16, [1, 2, 3, 2], True, True),
    (5, 1, 1, 128, 48, [0, 24], False, True),
    (3, 200, 40, 64, 32, [16], False, True),
    (4500, 9, 2, 128, 128, [16, 24, 24], True, True),
])
def test_rotation(dtype, R, Hq, Hk, dh, rot, sec, mixed, norm):
    mp, dev = _mp(), device()
    announce(f"rotation {dtype} R {R} heads {Hq}/{Hk} x {dh} rot {rot} {sec}")
    g = torch.Generator().manual_seed(R + rot)
    q = torch.randn(R, Hq, dh, generator=g).to(dtype).to(dev)
    k = (3 * torch.randn(R, Hk, dh, generator=g)).to(dtype).to(dev)
    pos = torch.randint(-5, 70000, (len(sec), R), generator=g, dtype=torch.int32).to(dev)
    qn, kn = ((1 + 0.2 * torch.randn(2, dh, generator=g)).to(dtype).to(dev).unbind(0)) if norm else (None, None)
    rp = mp.RopeParams(dh, rot_dim=rot, sections=sec, interleaved=mixed, theta=50000.0, eps=1e-5)
    got = mp.map_qk_norm_rope(rp, q, k, pos, qn, kn)
    for x, w, y in ((q, qn, got[0]), (k, kn, got[1])):
        w = None if w is None else _f64(w)
        want = oc.qk_norm_rope(_f64(x), _f64(pos), w, rot, sec, mixed, 50000.0, 1e-5)
        # the pair's magnitudes: the rotation of |a| + |b| is bounded by their sum
        a = np.abs(oc.qk_norm_rope(_f64(x), 0 * _f64(pos), w, rot, sec, mixed, 50000.0, 1e-5))
        mag = a.copy()
        mag[..., :rot] = np.tile(a[..., :rot // 2] + a[..., rot // 2:rot], 2)
        assert (np.abs(_f64(y) - want) <= U[dtype] * np.abs(want) + 32 * 2.0 ** -24 * mag).all()


def test_rotation_in_place_in_a_wider_row_and_far_positions():
    """q and k as parts of one qkv row, turned in place (v stays), positions near
    the end of int32: as far as float64 angles go (2^31 turns to 2^-20)."""
    mp, dev = _mp(), device()
    announce("rotation in place")
    g = torch.Generator().manual_seed(3)
    R, Hq, Hk, dh = 37, 6, 2, 128
    qkv = torch.randn(R, (Hq + 2 * Hk) * dh, generator=g).to(dev)
    before = qkv.clone()
    q, k = qkv[:, :Hq * dh].view(R, Hq, dh), qkv[:, Hq * dh:(Hq + Hk) * dh].view(R, Hk, dh)
    pos = torch.randint(2 ** 31 - 1000, 2 ** 31 - 1, (R,), generator=g, dtype=torch.int64).to(torch.int32).to(dev)
    want = oc.qk_norm_rope(_f64(q), _f64(pos)[None], None, dh, [64])
    out = mp.map_qk_norm_rope(mp.RopeParams(dh), q, k, pos, q_out=q, k_out=k)
    assert out[0] is q and out[1] is k
    # float64 angles: 2^31 * 2^-53 in the oracle's and half a turn's share in ours
    assert np.abs(_f64(q) - want).max() <= 2.0 ** -18
    assert torch.equal(qkv[:, (Hq + Hk) * dh:], before[:, (Hq + Hk) * dh:])
    none = mp.map_qk_norm_rope(mp.RopeParams(dh), q[:0], k[:0], pos[:0])
    assert none[0].shape == (0, Hq, dh) and none[1].shape == (0, Hk, dh)


def test_rotation_keeps_what_it_does_not_turn():
    """Values past rot_dim pass as they are, infinities and NaN among them."""
    mp, dev = _mp(), device()
    announce("rotation, values that pass")
    x = torch.randn(4, 2, 128, device=dev).bfloat16()
    x[1, 0, 100], x[2, 1, 40] = float("inf"), float("nan")
    pos = torch.arange(4, dtype=torch.int32, device=dev)
    q, _ = mp.map_qk_norm_rope(mp.RopeParams(128, rot_dim=32), x, x, pos)
    assert torch.equal(q[..., 32:].view(torch.int16), x[..., 32:].view(torch.int16))
    assert torch.isfinite(q[..., :32]).all()


# ------------------------------------------------------------- the cache
class Batch:
    """Sequences with `past` tokens and n new ones in a shuffled pool, the same
    on the GPU and in the oracle."""

    def __init__(self, kind, dh, heads, page, n, past, seed=0, spare=3, wide=0, fill=None):
        mp, dev = _mp(), device()
        g = torch.Generator().manual_seed(seed)
        self.n, self.past, self.B, self.heads, self.dh = n, past, len(n), heads, dh
        lens = [a + b for a, b in zip(n, past)]
        width = max(max(-(-x // page) for x in lens), 1) + wide
        n_pages = self.B * width + spare
        self.table = torch.randperm(n_pages, generator=g)[:self.B * width].view(self.B, width).to(torch.int32)
        self.cache = mp.KVCache(n_pages, page, heads, dh, kind, device=dev)
        if fill is not None:  # what no token has written yet
            for t in (self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale):
                if t is not None:
                    t.fill_(fill if t.dtype == torch.bfloat16 else 255)
        self.oracle = oc.PagedCache(n_pages, page, self.table.tolist(), kind == "mxfp4")
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.off = [0] + np.cumsum(n).tolist()
        self.g = g
        self.dev = dev
        at = torch.tensor(past, dtype=torch.int32)
        po = [0] + np.cumsum(past).tolist()
        if po[-1]:
            self._append(self.rows(po[-1]), self.rows(po[-1]), at, po)

    def rows(self, T, heads=None, scale=1.0):
        x = torch.randn(T, heads or self.heads, self.dh, generator=self.g) * scale
        return x.bfloat16()

    def _append(self, k, v, lens, off):
        _mp().map_cache_append(self.cache, self.table.to(self.dev), lens.to(self.dev), k.to(self.dev), v.to(self.dev), off)
        self.oracle.append(lens.tolist(), off, _f64(k), _f64(v))

    def append(self, k=None, v=None):
        k = self.rows(self.off[-1]) if k is None else k
        v = self.rows(self.off[-1]) if v is None else v
        self._append(k, v, self.lens, self.off)

    def attend(self, q, window=0, sinks=0, scale=None, **kw):
        return _mp().map_cache_attention(self.cache, self.table.to(self.dev), self.lens.to(self.dev), q.to(self.dev), self.off,
                                         scale=scale, window=window, sinks=sinks, **kw)

    def check(self, q, window=0, sinks=0, scale=None, got=None):
        got = _f64(self.attend(q, window, sinks, scale) if got is None else got)[:self.off[-1]]
        s = scale or self.dh ** -0.5
        want, spread = self.oracle.attention(self.lens.tolist(), self.off, _f64(q)[:self.off[-1]], s, window, sinks)
        qk = np.abs(_f64(q)).sum(-1).max() * max([np.abs(r[0]).max() for r in self.oracle.rows.values()] or [0.0])
        du = (self.dh + 2) * 2.0 ** -24 * s * qk
        bar = U[torch.bfloat16] * (np.abs(want) + spread) + spread * (2 * du + 2.0 ** -14)
        off = np.abs(got - want) - bar
        assert (off <= 0).all(), (np.argwhere(off > 0)[:4].tolist(), float(off.max()), float(np.nanmax(np.abs(got))))
        return got


KINDS = ["bf16", "mxfp4"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,heads,page,n,past", [
    (128, 4, 16, [1, 1, 1], [0, 15, 16]),
    (64, 3, 64, [5, 0, 70, 1], [60, 3, 100, 0]),
    (128, 1, 128, [200], [129]),
    (64, 9, 32, [33, 31, 32, 1], [0, 1, 31, 64]),
])
def test_rows_in_and_out(kind, dh, heads, page, n, past):
    mp = _mp()
    announce(f"cache rows {kind} {heads} x {dh} pages of {page}, {n} behind {past}")
    b = Batch(kind, dh, heads, page, n, past, seed=dh + page)
    k, v = b.rows(b.off[-1], scale=5.0), b.rows(b.off[-1])
    b.append(k, v)
    off = [0] + np.cumsum(b.lens.tolist()).tolist()
    got = mp.map_cache_read(b.cache, b.table.to(b.dev), b.lens.to(b.dev), off)
    for s in range(b.B):
        for j in range(int(b.lens[s])):
            for x, want in zip(got, b.oracle.token(s, j, b.lens.tolist())):
                np.testing.assert_array_equal(_f64(x[off[s] + j]), want)
    # by slots: the last, the first, one twice, one that is not there, and stored elsewhere
    slots, where = [], []
    for s in range(b.B):
        L = int(b.lens[s])
        pick = [L - 1, 0, L // 2, L // 2, L, -1] if L else [0]
        slots += pick
        where += [(s, j) for j in pick]
    so = [0] + np.cumsum([6 if int(x) else 1 for x in b.lens]).tolist()
    gk, gv = mp.map_cache_read(b.cache, b.table.to(b.dev), b.lens.to(b.dev), so, slots=torch.tensor(slots, dtype=torch.int32, device=b.dev))
    for r, (s, j) in enumerate(where):
        want = b.oracle.token(s, j, b.lens.tolist())
        for x, i in ((gk, 0), (gv, 1)):
            np.testing.assert_array_equal(_f64(x[r]), np.zeros((heads, dh)) if want is None else want[i])


def test_four_bit_rounding_everywhere():
    """Every bf16 value at and beside the borders between levels, both signs,
    at the lowest, an ordinary and a high scale; scales at both sides of 7 * 2^e;
    zero blocks, infinities and NaN: bit for bit."""
    mp, dev = _mp(), device()
    announce("4-bit rounding")
    blocks = []
    for e in (-126, -125, -130, -4, 0, 60, 125):
        for top in (6.0, 7.0, 4.0, 3.515625, 7.03125):
            pts = [x * (1 + d / 128) for x in (0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5) for d in (-1, 0, 1)] + [0.0, -0.0]
            for i in range(0, len(pts), 15):
                part = (pts[i:i + 15] + [0.0] * 15)[:15]
                blocks.append(torch.tensor([top] + [s * p for p in part for s in (1, -1)] + [-top * 0.99], dtype=torch.float64) * 2.0 ** e)
    blocks += [torch.zeros(32).double(), torch.full((32,), float("inf")).double(), torch.tensor([1.0] * 31 + [float("nan")]).double(),
               torch.tensor([3.38e38] + [1.0] * 31).double(), torch.tensor([2.0 ** -133] + [0.0] * 31).double()]
    x = torch.stack(blocks).to(torch.bfloat16)
    x = torch.cat([x, x[:(-len(x)) % 4]]).view(-1, 1, 128)
    cache = mp.KVCache(len(x) // 16 + 1, 16, 1, 128, "mxfp4", device=dev)
    table = torch.arange(len(x) // 16 + 1, dtype=torch.int32, device=dev)[None]
    lens = torch.tensor([len(x)], dtype=torch.int32, device=dev)
    mp.map_cache_append(cache, table, lens, x.to(dev), x.to(dev), [0, len(x)])
    want = [oc.mxfp4_block(b) for b in _f64(x).reshape(-1, 32)]
    codes, scales = (t.reshape(-1, w)[:len(x)].cpu().numpy() for t, w in ((cache.k, 64), (cache.k_scale, 4)))
    np.testing.assert_array_equal(scales.reshape(-1), [w[1] for w in want])
    np.testing.assert_array_equal(np.stack([codes & 15, codes >> 4], -1).reshape(-1, 32), [w[0] for w in want])
    assert torch.equal(cache.k, cache.v) and torch.equal(cache.k_scale, cache.v_scale)
    k, v = mp.map_cache_read(cache, table, lens, [0, len(x)])
    np.testing.assert_array_equal(_f64(k).reshape(-1, 32), np.stack([oc.mxfp4_values(*w) for w in want]))
    assert torch.equal(k.view(torch.int16), v.view(torch.int16))


def test_bad_pages_and_lengths():
    """Entries that are no page, lengths past the table and below zero: rows
    dropped or zero, other pages untouched, rows behind the last sequence too."""
    mp, dev = _mp(), device()
    announce("bad pages")
    for kind in KINDS:
        b = Batch(kind, 64, 2, 16, [20, 30, 6], [0, 0, 0], seed=5)
        b.table[0, 1], b.table[1, 0], b.table[2, 0] = -1, b.cache.n_pages, 2 ** 31 - 1
        b.oracle.table = b.table.tolist()
        before = [t.clone() for t in (b.cache.k, b.cache.v)]
        b.append()
        used = {int(b.table[0, 0]), int(b.table[1, 1])}
        for t, old in zip((b.cache.k, b.cache.v), before):
            for p in range(b.cache.n_pages):
                assert p in used or torch.equal(t[p], old[p])
        q = b.rows(b.off[-1] + 9, heads=4)
        out = torch.full((b.off[-1] + 9, 4, 64), 7.0, dtype=torch.bfloat16, device=dev)
        b.attend(q, out=out)
        b.check(q, got=out)
        assert (out[b.off[-1]:] == 7).all() and not out[b.off[2]:b.off[3]].any()
        for lens in ([1000, 3, -4], [20, 30, 6]):
            b.lens = torch.tensor(lens, dtype=torch.int32)
            b.check(q)
            k, v = mp.map_cache_read(b.cache, b.table.to(dev), b.lens.to(dev), b.off)
            for s in range(3):
                for i in range(b.n[s]):
                    want = b.oracle.token(s, i, lens)
                    np.testing.assert_array_equal(_f64(v[b.off[s] + i]), np.zeros((2, 64)) if want is None else want[1])


# ------------------------------------------------------------- attention
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,heads,G,page,n,past,window,sinks", [
    (128, 2, 1, 16, [1, 1, 1, 1], [0, 1, 63, 64], 0, 0),          # single tokens, the first of a sequence among them
    (128, 1, 7, 64, [1, 1, 0, 1], [15, 130, 40, 257], 0, 0),
    (64, 3, 4, 32, [1, 2, 5], [700, 333, 90], 0, 0),
    (128, 2, 3, 16, [3, 6, 4], [200, 17, 0], 33, 5),              # a few rows, window edges inside tiles
    (64, 1, 8, 128, [9, 1], [300, 1000], 64, 64),
    (128, 1, 1, 32, [17, 70, 1, 33], [0, 0, 0, 50], 0, 0),        # prompts
    (128, 2, 2, 64, [130, 64], [31, 0], 0, 0),
    (64, 2, 5, 16, [150, 65, 129], [0, 100, 3], 40, 4),
    (128, 1, 16, 128, [40, 20], [90, 5], 7, 200),                 # more first tokens than the window is long
    (64, 4, 1, 16, [300], [0], 1, 0),                             # a row sees itself alone
    (128, 1, 24, 16, [1, 2], [100, 150], 0, 0),                   # more heads than one tile of 16
])
def test_attention(kind, dh, heads, G, page, n, past, window, sinks):
    announce(f"cache attention {kind} {heads * G}/{heads} x {dh} pages of {page}, {n} behind {past}, window {window}, {sinks} first")
    b = Batch(kind, dh, heads, page, n, past, seed=dh + page + G, wide=2, fill=float("nan"))
    b.append()
    b.check(b.rows(b.off[-1], heads=heads * G, scale=1.5), window, sinks)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,past,window,sinks,scale", [
    ([1], [5000], 0, 0, None), ([1, 1], [4095, 2049], 1000, 4, 0.3), ([3], [3000], 0, 0, 2.0), ([260], [1500], 0, 0, None),
    ([70], [2000], 500, 10, None),
])
def test_attention_behind_a_long_cache(kind, n, past, window, sinks, scale):
    """Few rows over many tokens (the work is split along the cache and joined)."""
    announce(f"cache attention {kind}, {n} behind {past}")
    b = Batch(kind, 128, 1, 32, n, past, seed=n[0] + past[0], wide=3, fill=float("nan"))
    b.append()
    b.check(b.rows(b.off[-1], heads=2), window, sinks, scale)


@pytest.mark.parametrize("n", [[1, 1], [4, 6], [90, 40]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("kind", KINDS)
def test_what_a_row_does_not_see_adds_nothing(kind, n, bad):
    """NaN and infinities in tokens that are outside a row's window, or after it:
    the rows that see them not are what they are without them."""
    announce(f"cache attention {kind}, {bad} in hidden places, rows {n}")
    past, window, sinks = [100, 70], 20, 3
    for where in ("keys", "values"):
        b = Batch(kind, 64, 2, 16, n, past, seed=n[0])
        k, v = b.rows(b.off[-1]), b.rows(b.off[-1])
        b.append(k, v)
        q = b.rows(b.off[-1], heads=4)
        clean = _f64(b.attend(q, window, sinks))
        # sequence 0's token 50 (outside each window of [1, 1]) and its last row's own token
        x = k if where == "keys" else v
        x[n[0] - 1, 1, 5] = bad
        b.append(k, v)
        page, place = int(b.table[0, 50 // 16]), 50 % 16
        pool = b.cache.k if where == "keys" else b.cache.v
        if kind == "bf16":
            pool[page, 0, place, 9] = bad
        else:
            (b.cache.k_scale if where == "keys" else b.cache.v_scale)[page, 0, place, 0] = 255
        got = _f64(b.attend(q, window, sinks))
        for i in range(n[0]):
            me = past[0] + i
            for h in range(4):
                hit = (me - 50 < window and h // 2 == 0) or (i == n[0] - 1 and h // 2 == 1)
                if not hit:
                    np.testing.assert_array_equal(got[i, h], clean[i, h])
                elif where == "values":
                    assert not np.isfinite(got[i, h]).all()
        np.testing.assert_array_equal(got[n[0]:], clean[n[0]:])


@pytest.mark.parametrize("n", [[1, 1], [5], [80]])
@pytest.mark.parametrize("kind", KINDS)
def test_scores_far_apart(kind, n):
    """Scores over hundreds (one token takes all), all equal, and rising through
    the sequence, so that the running maximum moves at every block."""
    announce(f"cache attention {kind}, scores far apart, rows {n}")
    past = [900] * len(n)
    b = Batch(kind, 64, 1, 16, n, past, seed=7)
    rise = torch.linspace(0, 64, 16).bfloat16()
    k = b.rows(sum(past))
    k[:, 0, 0] = rise[torch.arange(sum(past)) % 900 // 64 % 16]
    b._append(k, b.rows(sum(past)), torch.tensor(past, dtype=torch.int32), [900 * i for i in range(len(n) + 1)])
    b.append()
    q = b.rows(b.off[-1], heads=2)
    q[:, :, 0] = 40.0
    b.check(q)
    b.check(-q)
    b.check(torch.zeros_like(q))
    b.check(q, scale=3.0)


def test_strided_rows_streams_and_repeats():
    """q, k and v as parts of one row, out inside a wider one, on another stream,
    twice: the same bits."""
    mp, dev = _mp(), device()
    announce("cache, strided rows on a stream")
    for kind in KINDS:
        b = Batch(kind, 128, 2, 16, [3, 1, 40], [50, 600, 20], seed=9)
        qkv = b.rows(b.off[-1], heads=10).to(dev)
        q, k, v = qkv[:, :6], qkv[:, 6:8], qkv[:, 8:]
        s = torch.cuda.Stream()
        wide = torch.zeros(b.off[-1], 8, 128, dtype=torch.bfloat16, device=dev)
        table, lens = b.table.to(dev), b.lens.to(dev)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            mp.map_cache_append(b.cache, table, lens, k, v, b.off)
            mp.map_cache_attention(b.cache, table, lens, q, b.off, out=wide[:, 1:7])
            again = mp.map_cache_attention(b.cache, table, lens, q.contiguous(), mp.SeqOffsets(b.off))
        s.synchronize()
        b.oracle.append(b.lens.tolist(), b.off, _f64(k), _f64(v))
        b.check(q, got=wide[:, 1:7])
        assert torch.equal(wide[:, 1:7], again) and not wide[:, 0].any() and not wide[:, 7].any()


def test_a_captured_step_follows_lengths_and_pages():
    """A decode step captured once and replayed while the lengths grow and a
    sequence moves to other pages: each replay equals the eager step."""
    mp, dev = _mp(), device()
    announce("cache, captured step")
    for kind in KINDS:
        b = Batch(kind, 128, 2, 16, [1, 1, 1], [30, 200, 0], seed=11, wide=8)
        rp = mp.RopeParams(128, sections=[16, 24, 24])
        qkv, pos = torch.zeros(3, 12, 128, dtype=torch.bfloat16, device=dev), torch.zeros(3, 3, dtype=torch.int32, device=dev)
        table, lens, off = b.table.to(dev), b.lens.to(dev), mp.SeqOffsets(b.off)
        norm = (1 + 0.1 * torch.randn(128, device=dev)).bfloat16()
        ws = mp.cache_attention_workspace(b.cache, off, 8, table)
        out = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device=dev)

        def step():
            q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
            rq, rk = mp.map_qk_norm_rope(rp, q, k, pos, norm, norm)
            mp.map_cache_append(b.cache, table, lens, rk, v, off)
            mp.map_cache_attention(b.cache, table, lens, rq, off, window=150, sinks=4, out=out, workspace=ws)

        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        g = torch.Generator().manual_seed(1)
        for t in range(6):
            qkv.copy_(torch.randn(3, 12, 128, generator=g).bfloat16())
            pos.copy_(torch.randint(0, 900, (3, 3), generator=g, dtype=torch.int32))
            lens += 17
            if t == 3:  # sequence 0 in other pages: its tokens move with it
                spare = [p for p in range(b.cache.n_pages) if p not in set(table.flatten().tolist())]
                old = int(table[0, 0])
                for pool in (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale):
                    if pool is not None:
                        pool[spare[0]] = pool[old]
                table[0, 0] = spare[0]
            graph.replay()
            torch.cuda.synchronize()
            replayed = out.clone()
            out.zero_()
            step()
            torch.cuda.synchronize()
            assert torch.equal(out, replayed), (kind, t)


def test_long_pool_offsets():
    """A pool past 4 GiB: pages at its end are where they should be."""
    mp, dev = _mp(), device()
    announce("cache, pool past 4 GiB")
    heads, page, dh = 32, 128, 128
    n_pages = (5 << 30) // (heads * page * dh * 2)
    cache = mp.KVCache(n_pages, page, heads, dh, "bf16", device=dev)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device=dev)
    n = 300
    lens = torch.tensor([n], dtype=torch.int32, device=dev)
    g = torch.Generator(device=dev).manual_seed(2)
    k, v, q = (torch.randn(n, heads, dh, generator=g, device=dev).bfloat16() for _ in range(3))
    mp.map_cache_append(cache, table, lens, k, v, [0, n])
    gk, gv = mp.map_cache_read(cache, table, lens, [0, n])
    assert torch.equal(gk, k) and torch.equal(gv, v)
    for rows in (1, 100):
        o = mp.map_cache_attention(cache, table, lens, q[:rows], [0, rows])
        for h in (0, 31):
            z = q[:rows, h].double() @ k[:, h].double().T.contiguous() / dh ** 0.5
            hide = torch.arange(n, device=dev)[None] > (n - rows + torch.arange(rows, device=dev))[:, None]
            p = torch.softmax(z.masked_fill(hide, -float("inf")), 1)
            want, spread = p @ v[:, h].double(), p @ v[:, h].double().abs()
            assert ((o[:, h].double() - want).abs() <= U[torch.bfloat16] * (want.abs() + spread) + spread * 2.0 ** -10).all()


def test_a_decoder_layers_attention_from_the_cache():
    """The calls as a program strings them together: a layer's prefill in two
    parts and single tokens through the cache, against map_decoder_layer over the
    whole sequences (its RMSNorm, products and SwiGLU by torch in float32)."""
    mp, dev = _mp(), device()
    announce("decoder layer from the cache")
    d, H, ff, lens_all = 256, 2, 512, [70, 45]
    g = torch.Generator().manual_seed(4)
    w = {"attn_norm": 1 + 0.1 * torch.randn(d, generator=g), "w_qkv": 0.05 * torch.randn(3 * d, d, generator=g),
         "w_o": 0.05 * torch.randn(d, d, generator=g), "ffn_norm": 1 + 0.1 * torch.randn(d, generator=g),
         "w_gate_up": 0.05 * torch.randn(2 * ff, d, generator=g), "w_down": 0.05 * torch.randn(d, ff, generator=g)}
    w = {k: x.bfloat16().to(dev) for k, x in w.items()}
    X = torch.randn(sum(lens_all), d, generator=g).bfloat16().to(dev)
    pos = torch.cat([torch.sort(torch.randperm(3000, generator=g)[:n]).values for n in lens_all]).to(torch.int32).to(dev)
    want = mp.map_decoder_layer(mp.DecoderWeights(**w, n_heads=H), X, pos, [0, 70, 115])
    f = {k: x.float() for k, x in w.items()}

    def norm(x, weight):
        return (x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight).bfloat16().float()

    cache = mp.KVCache(20, 16, H, 128, "bf16", device=dev)
    table = torch.tensor([[3, 9, 1, 0, 12], [5, 2, 19, 7, -1]], dtype=torch.int32, device=dev)
    rp, got, have = mp.RopeParams(128), torch.empty_like(X), [0, 0]
    for part in ([33, 12], [36, 32], [1, 1]):
        rows = torch.cat([torch.arange(s + h, s + h + n) for s, h, n in zip((0, 70), have, part)]).to(dev)
        have = [h + n for h, n in zip(have, part)]
        off, lens = [0, part[0], sum(part)], torch.tensor(have, dtype=torch.int32, device=dev)
        x = X[rows].float()
        qkv = (norm(x, f["attn_norm"]) @ f["w_qkv"].T).bfloat16().view(len(rows), 3 * H, 128)
        q, k = mp.map_qk_norm_rope(rp, qkv[:, :H], qkv[:, H:2 * H], pos[rows])
        mp.map_cache_append(cache, table, lens, k, qkv[:, 2 * H:], off)
        o = mp.map_cache_attention(cache, table, lens, q, off)
        x1 = (x + o.reshape(len(rows), d).float() @ f["w_o"].T).bfloat16().float()
        gu = norm(x1, f["ffn_norm"]) @ f["w_gate_up"].T
        act = (torch.nn.functional.silu(gu[:, :ff]) * gu[:, ff:]).bfloat16().float()
        got[rows] = (x1 + act @ f["w_down"].T).bfloat16()
    # the same stored bf16 intermediates by other sums: the layer's own bar
    du, dw = (got.double() - X.double()), (want.double() - X.double())
    assert float((du - dw).norm() / dw.norm()) <= 1e-2


# ------------------------------------------------ how a call is divided
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,heads,G,page,n,past,window,sinks", [
    (64, 2, 2, 16, [1, 3, 1, 0, 2], [3000, 5, 0, 700, 1200], 0, 0),       # stretches over sequences of very different lengths
    (128, 1, 7, 64, [5, 1, 4], [900, 2500, 0], 0, 0),                     # ... over tiles of 16 of 35 (row, head) pairs
    (128, 2, 4, 32, [9, 16, 1], [1500, 40, 600], 300, 20),                # ... and a window's two ranges
    (64, 1, 3, 128, [1, 40, 2, 130], [2000, 1800, 600, 0], 0, 0),         # single tokens and prompts in one call
    (128, 1, 2, 16, [17, 1], [1400, 1300], 200, 4),
])
def test_attention_divided(kind, dh, heads, G, page, n, past, window, sinks):
    announce(f"cache attention divided {kind} {heads * G}/{heads} x {dh}, {n} behind {past}, window {window}")
    b = Batch(kind, dh, heads, page, n, past, seed=sum(past) + dh, wide=5, fill=float("nan"))
    b.append()
    q = b.rows(b.off[-1], heads=heads * G, scale=1.5)
    b.check(q, window, sinks)
    # a length past the table, one of zero, one of a sequence shorter than its rows
    b.lens = b.lens.clone()
    b.lens[0], b.lens[1] = 2 ** 30, min(2, int(b.lens[1]))
    b.oracle.rows.update({(p, s): (np.zeros((heads, dh)), np.zeros((heads, dh)))
                          for p, s in [(int(b.table[0, j // page]), j % page) for j in range(n[0] + past[0], b.table.shape[1] * page)]})
    for t, w in ((b.cache.k, 0), (b.cache.v, 0), (b.cache.k_scale, 127), (b.cache.v_scale, 127)):
        if t is not None:
            for j in range(n[0] + past[0], b.table.shape[1] * page):
                t[int(b.table[0, j // page]), :, j % page] = w
    b.check(q, window, sinks)


@pytest.mark.parametrize("kind", KINDS)
def test_hidden_values_in_long_caches(kind):
    """NaN between the first tokens and the windows, and in the last row's own
    token, where the few rows' blocks lie in several stretches."""
    announce(f"cache attention {kind}, NaN hidden in a long cache")
    b = Batch(kind, 64, 1, 16, [5, 1], [1500, 900], seed=21)
    k, v = b.rows(6), b.rows(6)
    b.append(k, v)
    q = b.rows(6, heads=2)
    clean = _f64(b.attend(q, 400, 3))
    v[4, 0, 7] = float("nan")
    b.append(k, v)
    page, place = int(b.table[0, 700 // 16]), 700 % 16
    if kind == "bf16":
        b.cache.v[page, 0, place, 9] = float("inf")
        b.cache.k[page, 0, place, 3] = float("nan")
    else:
        b.cache.v_scale[page, 0, place, 0] = b.cache.k_scale[page, 0, place, 1] = 255
    got = _f64(b.attend(q, 400, 3))
    assert not np.isfinite(got[4]).all()
    np.testing.assert_array_equal(got[[0, 1, 2, 3, 5]], clean[[0, 1, 2, 3, 5]])


def test_prompt_behind_more_blocks_than_pages_held():
    """A prompt's tokens past 256 blocks of 64 (the table's entries are brought
    256 blocks at a time), with as many heads as keep the tokens in one part."""
    mp, dev = _mp(), device()
    announce("cache prompt past 256 blocks")
    past, n, H, dh = 16500, 20, 512, 64
    for kind in KINDS:
        g = torch.Generator(device=dev).manual_seed(5)
        cache = mp.KVCache(140, 128, 1, dh, kind, device=dev)
        table = torch.randperm(140, generator=torch.Generator().manual_seed(1))[None, :130].to(torch.int32).to(dev)
        lens = torch.tensor([past + n], dtype=torch.int32, device=dev)
        k, v = (torch.randn(past + n, 1, dh, generator=g, device=dev).bfloat16() for _ in range(2))
        mp.map_cache_append(cache, table, lens, k, v, [0, past + n])
        k, v = mp.map_cache_read(cache, table, lens, [0, past + n])
        q = torch.randn(n, H, dh, generator=g, device=dev).bfloat16()
        for window, sinks in ((0, 0), (16400, 70)):
            o = mp.map_cache_attention(cache, table, lens, q, [0, n], window=window, sinks=sinks)
            at = past + torch.arange(n, device=dev)[:, None]
            j = torch.arange(past + n, device=dev)[None]
            hide = (j > at) | ((at - j >= window) & (j >= sinks) if window else j < 0)
            for h in (0, 255, 511):
                z = (q[:, h].double() @ k[:, 0].double().T.contiguous()) / dh ** 0.5
                p = torch.softmax(z.masked_fill(hide, -float("inf")), 1)
                want, spread = p @ v[:, 0].double(), p @ v[:, 0].double().abs()
                assert ((o[:, h].double() - want).abs() <= U[torch.bfloat16] * (want.abs() + spread) + spread * 2.0 ** -10).all()


def test_two_calls_at_once():
    """Two streams, two workspaces, one cache: both calls' results are what each
    gives alone."""
    mp, dev = _mp(), device()
    announce("cache, two calls at once")
    b = Batch("mxfp4", 128, 2, 32, [1, 2, 1], [2500, 900, 40], seed=31)
    c = Batch("bf16", 128, 2, 32, [40, 1], [1200, 3000], seed=32)
    b.append()
    c.append()
    qs = [b.rows(4, heads=4).to(dev), c.rows(41, heads=4).to(dev)]
    alone = [b.attend(qs[0]), c.attend(qs[1])]
    args = [(x.cache, x.table.to(dev), x.lens.to(dev), q, mp.SeqOffsets(x.off)) for x, q in ((b, qs[0]), (c, qs[1]))]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(8):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                outs[i].append(mp.map_cache_attention(*args[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(o, alone[i]) for o in outs[i])
