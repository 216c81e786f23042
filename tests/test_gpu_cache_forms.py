"""Attention over the cache in the forms a call can take: many sequences at
once, tiles for every place on the card, pages given back behind a window,
divided prompts with hidden values, blocks past the held table entries, replays
whose pages move.  Against the cache oracle, with its tests' bars, or with inputs
whose results are known exactly: a row whose keys give one token all the weight
returns that token's values as they are."""
import numpy as np
import pytest
import torch

from gpu_util import announce, device
from test_gpu_cache import KINDS, U, _f64, _mp
from test_gpu_cache_values import Held as Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
def test_as_many_sequences_as_a_call_takes(kind):
    """256 sequences: single tokens, a few rows, prompts in two parts (the last
    ones at the end of the batch) and empty ones, in stretches over all of them."""
    announce(f"256 sequences, {kind}")
    g = np.random.default_rng(1)
    n = g.choice([0, 1, 1, 1, 2, 5, 16], 256).tolist()
    past = g.integers(0, 300, 256).tolist()
    for s in (0, 3, 70, 129, 200, 255):
        n[s], past[s] = int(g.integers(17, 60)), int(g.integers(0, 900))
    past[64] = past[190] = 1000
    b = Batch(kind, 64, 1, 16, n, past, seed=41, wide=5)
    b.append()
    b.check(b.rows(b.off[-1], heads=2, scale=1.5))
    b.check(b.rows(b.off[-1], heads=2), 100, 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,heads,G", [(128, 16, 1), (64, 16, 3)])
def test_a_tile_for_each_place_and_ragged_lengths(kind, dh, heads, G):
    """More tiles than the card holds at a time, lengths a hundred times apart."""
    announce(f"640 tiles, {kind}, {heads * G}/{heads} x {dh}")
    n = [1] * 37 + [3, 1, 2]
    past = [(7 * s * s + 3) % 90 for s in range(38)] + [1900, 700]
    b = Batch(kind, dh, heads, 32, n, past, seed=42, fill=float("nan"))
    b.append()
    b.check(b.rows(b.off[-1], heads=heads * G))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,past", [([1, 3], [3000, 1500]), ([40, 25], [2500, 1700]), ([1, 2], [400, 300])])
def test_pages_given_back_behind_a_window(kind, n, past):
    """Entries of pages that no row sees any token of are -1, the pages in
    another sequence's hands (NaN here): the same bits as before."""
    announce(f"pages given back, {kind}, {n} behind {past}")
    window, sinks = 250, 20
    b = Batch(kind, 128, 1, 16, n, past, seed=43)
    b.append()
    q = b.rows(b.off[-1], heads=3)
    before = b.attend(q, window, sinks)
    for s in range(2):
        for t in range(2, (past[s] - window + 1) // 16):
            p = int(b.table[s, t])
            for pool in (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale):
                if pool is not None:
                    pool[p] = float("nan") if pool.dtype == torch.bfloat16 else 255
            b.table[s, t] = -1
    b.oracle.table = b.table.tolist()
    after = b.attend(q, window, sinks)
    assert (b.table < 0).sum() > (10 if past[0] > 1000 else 5) and torch.equal(before, after)
    b.check(q, window, sinks, got=after)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("where", ["keys", "values"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_hidden_values_in_a_divided_prompt(kind, where, bad):
    """A token that only the first rows' windows reach, in an early part, and the
    last row's own, in the last one: the rows that do not see them keep their bits."""
    announce(f"divided prompt, {bad} in hidden {where}, {kind}")
    past, n, window, sinks = 3000, 40, 1500, 3
    b = Batch(kind, 64, 1, 16, [n, 20], [past, 800], seed=44)
    k, v = b.rows(60), b.rows(60)
    b.append(k, v)
    q = b.rows(60, heads=2)
    clean = b.attend(q, window, sinks)
    early = past - window + 1 + 10  # row i sees it for i <= 10
    (k if where == "keys" else v)[n - 1, 0, 7] = bad
    b.append(k, v)
    page, place = int(b.table[0, early // 16]), early % 16
    if kind == "bf16":
        (b.cache.k if where == "keys" else b.cache.v)[page, 0, place, 9] = bad
    else:
        (b.cache.k_scale if where == "keys" else b.cache.v_scale)[page, 0, place, 0] = 255
    got = b.attend(q, window, sinks)
    keep = list(range(11, n - 1)) + list(range(n, 60))
    assert torch.equal(got[keep], clean[keep])
    if where == "values":
        assert not torch.isfinite(got[:11, :, 9]).any() and not torch.isfinite(got[n - 1, :, 7]).any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,heads,past", [(20, 512, 16500), (20, 64, 16500), (2, 64, 16500), (1, 64, 500), (70, 64, 900)])
def test_each_block_counts(kind, rows, heads, past):
    """Past 256 blocks of 64 tokens in one part, in several, in stretches, and
    behind short caches.  Head h's query gives all the weight to one token, chosen
    at blocks' and pages' ends: its values come back.  With queries of zero each
    16 tokens' share of the mean shows in a channel of its own."""
    mp, dev = _mp(), device()
    announce(f"each block counts, {kind}, {rows} rows of {heads} heads behind {past}")
    dh, page, T = 64, 16, past + rows
    g = torch.Generator().manual_seed(past + heads)
    width = -(-T // page)
    cache = mp.KVCache(width + 3, page, 1, dh, kind, device=dev)
    table = torch.randperm(width + 3, generator=g)[None, :width].to(torch.int32).to(dev)
    lens = torch.tensor([T], dtype=torch.int32, device=dev)
    ends = [x for blk in (0, 1, 2, 7, 15, 16, 63, 127, 128, 254, 255, 256, 257) for x in (64 * blk, 64 * blk + 63)]
    pick = sorted({x for x in ends + [past - 1, past, 31, 32, 47, 48] if x <= past})
    pick = torch.tensor(pick + torch.randint(0, past + 1, (64 - len(pick),), generator=g).tolist())
    k = torch.zeros(T, 1, dh)
    for c, t in enumerate(pick.tolist()):
        k[t, 0, c] = 4.0
    v = torch.randn(T, 1, dh, generator=g)
    mp.map_cache_append(cache, table, lens, k.bfloat16().to(dev), v.bfloat16().to(dev), [0, T])
    held = mp.map_cache_read(cache, table, lens, [0, T])[1].cpu()
    q = torch.zeros(rows, heads, dh)
    for h in range(heads):
        q[:, h, h % dh] = 1024.0  # (a score of 512 above the others': they weigh 2^-738)
    q = q.bfloat16().to(dev)
    for window, sinks in ((0, 0), (past - 5, 70)):
        o = mp.map_cache_attention(cache, table, lens, q, [0, rows], window=window, sinks=sinks).cpu()
        for h in range(heads):
            token = pick[h % dh]
            same = (pick == token).nonzero().flatten()[0]
            for i in range(rows):
                me = past + i
                if window == 0 or me - token < window or token < sinks:
                    assert torch.equal(o[i, h], held[token, 0]), (h, i, int(token), int(same))
    at = torch.arange(T)
    mark = torch.nn.functional.one_hot(at // 16 % dh, dh).float()[:, None]
    mp.map_cache_append(cache, table, lens, k.bfloat16().to(dev), mark.bfloat16().to(dev), [0, T])
    for window, sinks in ((0, 0), (past - 5, 70)):
        o = mp.map_cache_attention(cache, table, lens, torch.zeros_like(q), [0, rows], window=window, sinks=sinks)
        me = past + torch.arange(rows)[:, None]
        see = (at[None] <= me) & ((me - at[None] < window) | (at[None] < sinks) if window else at[None] >= 0)
        want = (see.double() @ mark[:, 0].double() / see.sum(1, keepdim=True))[:, None].numpy()
        # (weights of one, sums of whole numbers: the division and the output's rounding)
        assert (np.abs(_f64(o) - want) <= (U[torch.bfloat16] + 2.0 ** -20) * want).all()


def test_scale_bytes_of_the_smallest_values():
    """Every code under every scale byte, read back, and attention over the
    smallest ones, whose values bfloat16 holds as subnormal numbers."""
    mp, dev = _mp(), device()
    announce("scale bytes 0 .. 255")
    cache = mp.KVCache(16, 16, 1, 64, "mxfp4", device=dev)
    codes = torch.arange(16, dtype=torch.uint8).repeat(4)
    packed = codes[0::2] | (codes[1::2] << 4)
    cache.k[:] = packed.to(dev)
    cache.v[:] = packed.flip(0).to(dev)
    byte = torch.arange(256, dtype=torch.uint8)
    for s in (cache.k_scale, cache.v_scale):
        s.view(256, 2)[:] = byte[:, None].to(dev)
    table = torch.arange(16, dtype=torch.int32, device=dev)[None]
    lens = torch.tensor([256], dtype=torch.int32, device=dev)
    k, v = (_f64(x)[:, 0] for x in mp.map_cache_read(cache, table, lens, [0, 256]))
    level = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
    value = np.concatenate([level, -level])
    with np.errstate(over="ignore"):
        for x, c in ((k, codes.numpy()), (v, np.stack([packed.flip(0).numpy() & 15, packed.flip(0).numpy() >> 4], -1).reshape(-1))):
            want = value[c][None] * 2.0 ** (np.arange(256)[:, None] - 127.0)
            np.testing.assert_array_equal(x[:253], want[:253])  # (6 * 2^126 is past bfloat16)
            assert np.isnan(x[255]).all()
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device=dev)
    for first, many in ((0, 16), (0, 48), (16, 16)):  # equal weights over tokens of bytes first .. first + many - 1
        t = table[:, first // 16:].contiguous()
        got = _f64(mp.map_cache_attention(cache, t, torch.tensor([many], dtype=torch.int32, device=dev), q, [0, 1]))
        want, spread = v[first:first + many].mean(0), np.abs(v[first:first + many]).mean(0)
        # a subnormal result is off by half of 2^-133
        assert (np.abs(got - want) <= U[torch.bfloat16] * np.abs(want) + 2.0 ** -20 * spread + 2.0 ** -134).all()


@pytest.mark.parametrize("kind", KINDS)
def test_replays_follow_pages_that_move(kind):
    """A captured step while the lengths grow, a sequence moves to another page
    and the old one turns to NaN: eager and replayed alike, and as the oracle."""
    mp, dev = _mp(), device()
    announce(f"captured step, pages that move, {kind}")
    b = Batch(kind, 128, 2, 16, [1, 1, 2], [30, 900, 0], seed=45, wide=3)
    table, lens, off = b.table.to(dev), b.lens.to(dev), mp.SeqOffsets(b.off)
    ws = mp.cache_attention_workspace(b.cache, off, 8, table)
    qkv, out = torch.zeros(4, 12, 128, dtype=torch.bfloat16, device=dev), torch.zeros(4, 8, 128, dtype=torch.bfloat16, device=dev)

    def step():
        mp.map_cache_append(b.cache, table, lens, qkv[:, 8:10], qkv[:, 10:], off)
        mp.map_cache_attention(b.cache, table, lens, qkv[:, :8], off, window=700, sinks=4, out=out, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    step_rows = torch.tensor([1, 1, 2], dtype=torch.int32)
    for t in range(5):
        rows = b.rows(4, heads=12)
        qkv.copy_(rows)
        if t:
            b.lens = b.lens + step_rows
            lens += step_rows.to(dev)
        if t in (2, 4):  # tokens 0 .. 15 of sequence t / 2 - 1 move
            s = t // 2 - 1
            spare = [p for p in range(b.cache.n_pages) if p not in set(b.table.flatten().tolist())][0]
            old = int(b.table[s, 0])
            for pool in (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale):
                if pool is not None:
                    pool[spare] = pool[old]
                    pool[old] = float("nan") if pool.dtype == torch.bfloat16 else 255
            b.oracle.rows.update({(spare, i): b.oracle.rows[(old, i)] for i in range(16) if (old, i) in b.oracle.rows})
            b.table[s, 0] = table[s, 0] = spare
            b.oracle.table = b.table.tolist()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        b.hold(b.lens, b.off)
        replayed = out.clone()
        b.check(rows[:, :8], 700, 4, got=replayed)
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, replayed), t


@pytest.mark.parametrize("n,past", [([1, 40, 2, 33, 16, 0, 50], [700, 1500, 3, 0, 200, 5, 600]), ([16] * 6 + [17], [100] * 6 + [2000])])
@pytest.mark.parametrize("kind", KINDS)
def test_divided_prompts_among_few_rows(kind, n, past):
    """The prompts' parts are joined, the few rows between them written once; a
    workspace of the size asked for is enough, and what lies behind it stays."""
    mp, dev = _mp(), device()
    announce(f"divided prompts among few rows, {kind}, {n}")
    b = Batch(kind, 128, 1, 32, n, past, seed=46, wide=8)
    b.append()
    q = b.rows(b.off[-1], heads=4).to(dev)
    size = mp.cache_attention_workspace(b.cache, b.off, 4, b.table).numel()
    room = torch.full((size + 4096 + 256,), 0xA5, dtype=torch.uint8, device=dev)
    at = -room.data_ptr() % 256
    got = b.attend(q, workspace=room[at:at + size])
    b.check(q, got=got)
    assert (room[at + size:] == 0xA5).all() and (room[:at] == 0xA5).all()
