"""Attention over the cache and the head norms: what rounding and range may and may
not move; attention in every form a call can take: a tile a workgroup, stretches, a
prompt, a prompt in parts.

Bars.  A row's probabilities above the fraction line add up to what is below it
(prompts) or to that but for 2^-17 (few rows), so values that are all equal come
back as they are: the float32 sums of T terms are off by T 2^-24 each, together
under the 2^-9 that moves a bfloat16 number for T < 8000.  Elsewhere, with u = 2^-8
and spread = sum p |v|, a probability's rounding and the output's: u (|o| + spread)
+ spread 2^-14 for the exponentials and the sums; the far scores are single
products, exact in float32.
"""
import numpy as np
import pytest
import torch

import oracle.cache as oc
from gpu_util import announce, device
from test_gpu_cache import KINDS, U, Batch, _f64, _mp

pytestmark = pytest.mark.gpu

# new rows and tokens before them: 16 rows or fewer, with a short table a tile a
# workgroup, else in stretches; more rows, in parts behind a long cache
FORMS = {"tile": ([1, 1], [290, 301]), "stretches": ([3, 1], [3000, 700]), "prompt": ([150], [300]), "parts": ([40], [2500])}


class Held(Batch):
    """A batch whose oracle holds what the cache gives back for the rows put in
    (their rounding to 4 bits has tests of its own)."""

    def _append(self, k, v, lens, off):
        _mp().map_cache_append(self.cache, self.table.to(self.dev), lens.to(self.dev), k.to(self.dev), v.to(self.dev), off)
        self.hold(lens, off)

    def hold(self, lens, off):
        """The last rows of each sequence, as the cache has them."""
        slots = [int(lens[s]) - off[s + 1] + r for s in range(self.B) for r in range(off[s], off[s + 1])]
        k, v = (_f64(x) for x in _mp().map_cache_read(self.cache, self.table.to(self.dev), lens.to(self.dev), off,
                                                      slots=torch.tensor(slots, dtype=torch.int32, device=self.dev)))
        for s in range(self.B):
            for r in range(off[s], off[s + 1]):
                self.oracle.rows[self.oracle.place(s, slots[r])] = (k[r], v[r])


def _batch(kind, form, dh=128, heads=2, seed=0):
    n, past = FORMS[form]
    return Held(kind, dh, heads, 16, n, past, seed=seed)


def _store(b, k, v):
    """All of each sequence's tokens at once: k and v by (sequence, token)."""
    lens = b.lens.tolist()
    off = [0] + np.cumsum(lens).tolist()
    b._append(torch.cat([k(s, lens[s]) for s in range(b.B)]), torch.cat([v(s, lens[s]) for s in range(b.B)]), b.lens, off)


def _near(got, want, spread):
    bar = U[torch.bfloat16] * (np.abs(want) + spread) + spread * 2.0 ** -14
    off = np.abs(got - want) - bar
    assert (off <= 0).all(), (np.argwhere(~(off <= 0))[:4].tolist(), float(np.abs(got).max()))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", FORMS)
def test_a_row_over_equal_values_gives_that_value(kind, form):
    """Token 0 at a score of zero, token 257 at one a little above it (the
    running maximum then stays where it is), all others far below."""
    announce(f"equal values, {kind}, {form}")
    b = _batch(kind, form, seed=1)
    g = torch.Generator().manual_seed(2)

    def keys(s, n):
        k = torch.zeros(n, 2, 128)
        k[:, :, 1] = -1.0
        k[[0, 257], :, 1] = 0.0
        k[257, :, 0] = 1.0
        return k.bfloat16()

    row = (torch.randint(0, 2, (1, 2, 128), generator=g) * 2 - 1).float().bfloat16()
    _store(b, keys, lambda s, n: row.expand(n, 2, 128).contiguous())
    q = torch.zeros(b.off[-1], 64, 128)
    q[:, :, 0] = 3.0 + 2.9 * torch.rand(b.off[-1], 64, generator=g)
    q[:, :, 1] = 4096.0
    got = b.attend(q.bfloat16(), scale=float(np.log(2.0)))
    want = row.repeat_interleave(32, 1).expand(b.off[-1], 64, 128)
    assert torch.equal(got.cpu(), want.contiguous())


@pytest.mark.parametrize("wide", [0, 40])
def test_few_rows_weigh_by_more_than_bfloat16(wide):
    """Two tokens with opposite values and nearly equal weights, whose difference
    a probability's rounding to 8 bits would move by more than the output's
    rounding: the weights carry 2^-17.  In tiles and, behind a wide table, stretches."""
    announce(f"nearly equal weights, table {wide} pages wider")
    b = Held("bf16", 128, 1, 16, [1] * 32, [1] * 32, seed=9, wide=wide)
    g = torch.Generator().manual_seed(9)

    def keys(s, n):
        k = torch.zeros(n, 1, 128)
        k[1, 0, 0] = 0.5 * torch.rand(1, generator=g)
        return k.bfloat16()

    def values(s, n):
        v = torch.randn(1, 1, 128, generator=g).bfloat16()
        return torch.cat([v, -v])

    _store(b, keys, values)
    q = torch.zeros(32, 8, 128)
    q[:, :, 0] = torch.rand(32, 8, generator=g) - 0.5
    q = q.bfloat16()
    want, spread = b.oracle.attention(b.lens.tolist(), b.off, _f64(q), 1.0)
    du = 130 * 2.0 ** -24 * 0.25  # |q k| <= 1/4
    off = np.abs(_f64(b.attend(q, scale=1.0)) - want) - U[torch.bfloat16] * np.abs(want) - spread * (2.0 ** -17 + 2 * du + 2.0 ** -14)
    assert (off <= 0).all(), float(off.max())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("first", [64, 1 << 30])
def test_values_whose_sum_passes_float32(kind, form, first):
    """Values at the end of their range, of one sign a channel: their sum is
    infinite in float32, their mean is not.  In all tokens, or in the first ones
    only, so that some waves' and some parts' sums are finite."""
    announce(f"large values, {kind}, {form}, the first {first}")
    b = _batch(kind, form, seed=3)
    g = torch.Generator().manual_seed(4)
    sign = (torch.randint(0, 2, (1, 2, 128), generator=g) * 2 - 1).double()

    def values(s, n):
        v = (1.2e38 + 2.1e38 * torch.rand(n, 2, 128, generator=g).double()) * sign
        v[first:] = torch.randn(max(n - first, 0), 2, 128, generator=g).double()
        return v.bfloat16()

    _store(b, lambda s, n: b.rows(n), values)
    q = b.rows(b.off[-1], heads=4)
    got = b.attend(q)
    assert torch.isfinite(got).all()
    b.check(q, got=got)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", FORMS)
def test_large_values_beside_hidden_ones(kind, form):
    """... and a NaN in the last row's own token, which the other rows do not see."""
    announce(f"large values beside a hidden NaN, {kind}, {form}")
    b = _batch(kind, form, seed=5)
    g = torch.Generator().manual_seed(6)

    def values(s, n):
        v = (1.2e38 + 2.1e38 * torch.rand(n, 2, 128, generator=g).double()).bfloat16()
        if s == 0:
            v[n - 1, :, 5] = float("nan")
        return v

    _store(b, lambda s, n: b.rows(n), values)
    q = b.rows(b.off[-1], heads=4)
    last = b.n[0] - 1
    got = b.attend(q)
    assert torch.isnan(got[last, :, 5]).all()
    keep = [r for r in range(b.off[-1]) if r != last]
    assert torch.isfinite(got[keep]).all()
    want, spread = b.oracle.attention(b.lens.tolist(), b.off, _f64(q), 128 ** -0.5)
    du = 130 * 2.0 ** -24 * 128 ** -0.5 * np.abs(_f64(q)).sum(-1).max() * max(np.abs(r[0]).max() for r in b.oracle.rows.values())
    bar = U[torch.bfloat16] * (np.abs(want) + spread) + spread * (2 * du + 2.0 ** -14)
    assert (np.abs(_f64(got) - want) <= bar)[keep].all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("far", [20, 27, 31, 36, 60])
def test_far_scores(kind, form, far):
    """Scores of plus and minus 1.77 times 2^far: half of the tokens share each
    row's weight, whatever their score times log2(e) rounds to."""
    announce(f"scores of 2^{far}, {kind}, {form}")
    b = _batch(kind, form, seed=far)
    g = torch.Generator().manual_seed(far)

    def keys(s, n):
        k = torch.zeros(n, 2, 128)
        k[:, :, 0] = (torch.randint(0, 2, (n, 2), generator=g) * 2 - 1) * 1.5 * 2.0 ** (far // 2)
        return k.bfloat16()

    _store(b, keys, lambda s, n: b.rows(n))
    q = torch.zeros(b.off[-1], 4, 128)
    q[:, :, 0] = 151 / 128 * 2.0 ** (far - far // 2)
    q[::2, 1, 0] *= -1.0
    q = q.bfloat16()
    for scale in (1.0, 0.7):
        want, spread = b.oracle.attention(b.lens.tolist(), b.off, _f64(q), float(np.float32(scale)))
        _near(_f64(b.attend(q, scale=scale)), want, spread)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size,eps", [(1e-30, 0.0), (1e-22, 1e-38), (1e18, 1e-6), (3e25, 1e-6), (1e38, 0.0)])
def test_norms_whose_squares_pass_float32(dtype, size, eps):
    """Heads whose sum of squares is infinite or zero in float32, among ordinary
    ones; their norms are neither."""
    mp, dev = _mp(), device()
    announce(f"norms of heads of {size}, eps {eps}, {dtype}")
    g = torch.Generator().manual_seed(7)
    R, Hq, Hk, dh, rot = 9, 10, 3, 128, 64
    q, k = torch.randn(R, Hq, dh, generator=g).double(), torch.randn(R, Hk, dh, generator=g).double()
    q[::2, 1::3] *= size / 3
    k[1::2] *= size / 3
    q, k = q.to(dtype).to(dev), k.to(dtype).to(dev)
    pos = torch.randint(0, 5000, (1, R), generator=g, dtype=torch.int32).to(dev)
    qn, kn = ((1 + 0.2 * torch.randn(2, dh, generator=g)).to(dtype).to(dev)).unbind(0)
    got = mp.map_qk_norm_rope(mp.RopeParams(dh, rot_dim=rot, eps=eps), q, k, pos, qn, kn)
    eps = float(np.float32(eps))
    for x, w, y in ((q, qn, got[0]), (k, kn, got[1])):
        want = oc.qk_norm_rope(_f64(x), _f64(pos), _f64(w), rot, [rot // 2], eps=eps)
        a = np.abs(oc.qk_norm_rope(_f64(x), 0 * _f64(pos), _f64(w), rot, [rot // 2], eps=eps))
        mag = a.copy()
        mag[..., :rot] = np.tile(a[..., :rot // 2] + a[..., rot // 2:rot], 2)
        assert (np.abs(_f64(y) - want) <= U[dtype] * np.abs(want) + 32 * 2.0 ** -24 * mag).all()


def test_norms_of_zero_and_of_what_is_not_finite():
    """A head of zeros stays zero; one that holds an infinity or a NaN is the
    formula's, and its neighbours are what they are without it."""
    mp, dev = _mp(), device()
    announce("norms of zeros and infinities")
    x = torch.randn(4, 6, 64, generator=torch.Generator().manual_seed(8)).to(dev)
    w, pos, rp = torch.ones(64, device=dev), torch.arange(4, dtype=torch.int32, device=dev), mp.RopeParams(64)
    clean, _ = mp.map_qk_norm_rope(rp, x, x, pos, w, w)
    y = x.clone()
    y[0, 1] = 0.0
    y[2, 3, 7], y[3, 0, 5] = float("inf"), float("nan")
    got, _ = mp.map_qk_norm_rope(rp, y, y, pos, w, w)
    assert not got[0, 1].any() and torch.isnan(got[3, 0]).all()
    assert torch.isnan(got[2, 3, [7, 39]]).all() and not got[2, 3, [0, 6, 8, 31, 38, 40, 63]].any()
    same = torch.ones(4, 6, dtype=torch.bool)
    same[0, 1] = same[2, 3] = same[3, 0] = False
    assert torch.equal(got[same], clean[same])


@pytest.mark.parametrize("form", list(FORMS) + ["three parts", "five parts"])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_visible_infinity_is_the_rows_value(form, sign):
    """An infinite value in the last row's own token, among equal scores: that
    row's channel is infinite, whatever waves, stretches and parts join."""
    announce(f"a visible infinity, {form}, {sign}")
    n, past = FORMS.get(form) or ([40], [1700 if form == "three parts" else 2700])
    b = Held("bf16", 128, 2, 16, n, past, seed=12)

    def values(s, length):
        v = b.rows(length)
        if s == 0:
            v[length - 1, 1, 77] = sign * float("inf")
        return v

    _store(b, lambda s, length: torch.zeros(length, 2, 128).bfloat16(), values)
    got = b.attend(b.rows(b.off[-1], heads=4)).cpu()
    bad = torch.zeros(got.shape, dtype=torch.bool)
    bad[n[0] - 1, 2:, 77] = True
    assert (got[bad] == sign * float("inf")).all() and torch.isfinite(got[~bad]).all()
