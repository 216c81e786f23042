"""Refusals of the cache calls and of the head rotation, on the host: the C
entry points return a status and the binding raises before anything is enqueued
(no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2608_06411_amd as mp
from paper_2608_06411_amd import binding as bd

P = ctypes.c_void_p
A = 0x10000  # an aligned address that nothing reads


def _cache(**kw):
    c = bd.map_cache(A, A, A, A, bd.MAP_CACHE_BF16, 10, 16, 4, 128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _off(*vals):
    return (ctypes.c_int32 * len(vals))(*vals)


def _rows(call, c=None, dt=bd.MAP_BF16, B=2, table=A, max_pages=3, lens=A, k=A, ldk=512, v=A, ldv=512, off=(0, 2, 5)):
    c = _cache() if c is None else c
    o = None if off is None else _off(*off)
    if call == "append":
        return bd.lib().map_cache_append(ctypes.byref(c), dt, B, P(table), max_pages, P(lens), P(k), ldk, P(v), ldv, o, None)
    return bd.lib().map_cache_read(ctypes.byref(c), dt, B, P(table), max_pages, P(lens), None, o, P(k), ldk, P(v), ldv, None)


BAD_CACHE = [dict(type=2), dict(n_pages=0), dict(page=48), dict(page=8), dict(page=256), dict(n_kv_heads=0), dict(n_kv_heads=257),
             dict(head_dim=96), dict(head_dim=32), dict(k=None), dict(v=A + 8),
             dict(type=bd.MAP_CACHE_MXFP4, k_scale=None), dict(type=bd.MAP_CACHE_MXFP4, v_scale=A + 4)]


@pytest.mark.parametrize("call", ["append", "read"])
def test_rows_calls_refuse(call):
    inv = bd.MAP_ERR_INVALID_ARG
    for bad in BAD_CACHE:
        assert _rows(call, _cache(**bad)) == inv, bad
    for bad in [dict(dt=9), dict(B=0), dict(B=bd.MAP_CACHE_MAX_BATCH + 1), dict(table=None), dict(lens=None), dict(max_pages=0),
                dict(max_pages=1 << 27), dict(k=None), dict(v=None), dict(k=A + 2), dict(ldk=511), dict(ldk=520 + 4), dict(ldv=508),
                dict(off=None), dict(off=(1, 2, 5)), dict(off=(0, 3, 2)), dict(off=(0, 0, bd.MAP_CACHE_MAX_ROWS + 1))]:
        assert _rows(call, **bad) == inv, bad
    assert _rows(call, dt=bd.MAP_F32) == bd.MAP_ERR_UNSUPPORTED
    assert _rows(call, off=(0, 0, 0)) == bd.MAP_OK  # no rows: nothing to enqueue


def _attend(c=None, dt=bd.MAP_BF16, B=2, heads=8, table=A, max_pages=3, lens=A, q=A, ldq=1024, off=(0, 2, 5), scale=0.1, window=0,
            sinks=0, out=A, ldo=1024, ws=A, nbytes=1 << 40):
    c = _cache() if c is None else c
    o = None if off is None else _off(*off)
    return bd.lib().map_cache_attention(ctypes.byref(c), dt, B, heads, P(table), max_pages, P(lens), P(q), ldq, o, scale, window,
                                        sinks, P(out), ldo, P(ws), nbytes, None)


def test_attention_refuses():
    inv = bd.MAP_ERR_INVALID_ARG
    for bad in BAD_CACHE:
        assert _attend(_cache(**bad)) == inv, bad
    for bad in [dict(dt=9), dict(B=0), dict(B=257), dict(heads=0), dict(heads=6), dict(heads=1028), dict(table=None), dict(lens=None),
                dict(max_pages=0), dict(q=None), dict(q=A + 8), dict(out=None), dict(ldq=1016), dict(ldq=1028), dict(ldo=1000),
                dict(off=None), dict(off=(0, 3, 2)), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(window=-1), dict(sinks=-1)]:
        assert _attend(**bad) == inv, bad
    assert _attend(dt=bd.MAP_F32) == bd.MAP_ERR_UNSUPPORTED
    need = bd.lib().map_cache_attention_workspace(ctypes.byref(_cache()), 2, 8, 3, _off(0, 2, 5))
    assert need >= 256
    for ws, nbytes in ((None, need), (A + 16, need), (A, need - 1)):
        assert _attend(ws=ws, nbytes=nbytes) == bd.MAP_ERR_WORKSPACE
    assert _attend(off=(0, 0, 0)) == bd.MAP_OK


def _rope(dt=bd.MAP_BF16, R=3, heads=4, kv=2, q=A, ldq=512, k=A, ldk=256, pos=A, ldpos=3, qn=None, kn=None, qo=2 * A, ldqo=512,
          ko=2 * A, ldko=256, **kw):
    rp = bd.map_rope(128, 128, 2, 0, (ctypes.c_int32 * 4)(20, 44, 0, 0), 10000.0, 1e-6)
    for name, v in kw.items():
        setattr(rp, name, (ctypes.c_int32 * 4)(*v) if name == "sections" else v)
    return bd.lib().map_qk_norm_rope(ctypes.byref(rp), dt, R, heads, kv, P(q), ldq, P(k), ldk, P(pos), ldpos, P(qn), P(kn), P(qo),
                                     ldqo, P(ko), ldko, None)


def test_rotation_refuses():
    for bad in [dict(dt=5), dict(R=-1), dict(R=bd.MAP_CACHE_MAX_ROWS + 1, ldpos=1 << 21), dict(heads=0), dict(kv=0), dict(heads=1025),
                dict(q=None), dict(k=None), dict(pos=None), dict(qo=None), dict(ko=None), dict(q=A + 8), dict(qn=A + 2), dict(ldq=504),
                dict(ldq=516), dict(ldk=248), dict(ldqo=500), dict(ldko=252), dict(ldpos=2), dict(head_dim=96), dict(rot_dim=24),
                dict(rot_dim=144), dict(rot_dim=0), dict(n_axes=0), dict(n_axes=5), dict(sections=(20, 43, 0, 0)),
                dict(sections=(-1, 65, 0, 0)), dict(theta=0.0), dict(theta=float("nan")), dict(eps=-1.0),
                dict(qo=A, ldqo=520)]:
        assert _rope(**bad) == bd.MAP_ERR_INVALID_ARG, bad
    assert _rope(R=0, ldpos=0) == bd.MAP_OK


# ------------------------------------------------ the binding, on CPU tensors
def _cpu(kind="bf16", B=2, rows=5, heads=8):
    c = mp.KVCache(10, 16, 4, 128, kind, device="cpu")
    return dict(cache=c, table=torch.zeros(B, 3, dtype=torch.int32), lens=torch.zeros(B, dtype=torch.int32),
                q=torch.zeros(rows, heads, 128, dtype=torch.bfloat16), k=torch.zeros(rows, 4, 128, dtype=torch.bfloat16),
                off=[0, 2, 5])


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_binding_refuses(kind):
    bf = torch.bfloat16
    good = _cpu(kind)

    def append(**kw):
        d = dict(good, **kw)
        mp.map_cache_append(d["cache"], d["table"], d["lens"], d["k"], d.get("v", d["k"]), d["off"])

    def read(**kw):
        d = dict(good, **kw)
        mp.map_cache_read(d["cache"], d["table"], d["lens"], d["off"], slots=d.get("slots"), k_out=d.get("k_out"))

    def attend(**kw):
        d = dict(good, **kw)
        mp.map_cache_attention(d["cache"], d["table"], d["lens"], d["q"], d["off"], window=d.get("window", 0), out=d.get("out"))

    for call in (append, read, attend):
        for bad, match in [(dict(table=torch.zeros(2, 3, dtype=torch.int64)), "table"), (dict(table=torch.zeros(3, 3, dtype=torch.int32)), "table"),
                           (dict(table=torch.zeros(2, 6, dtype=torch.int32)[:, ::2]), "table"),
                           (dict(lens=torch.zeros(3, dtype=torch.int32)), "lens"), (dict(off=[0, 3, 2]), "offsets"), (dict(off=[1, 3, 5]), "offsets"),
                           (dict(cache=None), "KVCache"), (dict(), "ROCm device")]:
            with pytest.raises((ValueError, TypeError), match=match):
                call(**bad)
    for bad, match in [(dict(k=torch.zeros(4, 4, 128, dtype=bf)), "k"), (dict(k=torch.zeros(5, 4, 128)), "k"), (dict(v=torch.zeros(5, 4, 64, dtype=bf)), "v"),
                       (dict(k=torch.zeros(5, 4, 256, dtype=bf)[..., ::2]), "strides"), (dict(k=torch.zeros(5, 4, 132, dtype=bf)[..., :128]), "strides"),
                       (dict(k=torch.zeros(5, 516, dtype=bf)[:, :512].view(5, 4, 128)), "strides")]:
        with pytest.raises(ValueError, match=match):
            append(**bad)
    with pytest.raises(ValueError, match="slots"):
        read(slots=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="k_out"):
        read(k_out=torch.zeros(5, 4, 128))
    with pytest.raises(ValueError, match="heads"):
        attend(q=torch.zeros(5, 6, 128, dtype=bf))
    with pytest.raises(ValueError, match="negative"):
        attend(window=-2)
    with pytest.raises(ValueError, match="out"):
        attend(out=torch.zeros(5, 8, 64, dtype=bf))
    with pytest.raises(ValueError, match="page"):
        mp.KVCache(4, 24, 4, 128, kind, device="cpu")
    with pytest.raises(ValueError, match="head_dim"):
        mp.KVCache(4, 16, 4, 96, kind, device="cpu")
    with pytest.raises(ValueError, match="kind"):
        mp.KVCache(4, 16, 4, 64, "int4", device="cpu")


def test_binding_refuses_bad_rotations():
    rp = mp.RopeParams(128, sections=[16, 24, 24])
    q, k, pos = torch.zeros(5, 4, 128), torch.zeros(5, 2, 128), torch.zeros(3, 5, dtype=torch.int32)
    for bad, match in [(dict(q=torch.zeros(5, 4, 64)), "heads of 64"), (dict(k=torch.zeros(4, 2, 128)), "k"), (dict(pos=pos[:2]), "pos"),
                       (dict(pos=pos.long()), "pos"), (dict(k=k.bfloat16()), "k"), (dict(q_norm=torch.zeros(64)), "q_norm"),
                       (dict(q=q.half()), "dtype"), (dict(q_out=torch.zeros(5, 4, 128).bfloat16()), "q_out"), (dict(), "ROCm device")]:
        with pytest.raises((ValueError, TypeError), match=match):
            mp.map_qk_norm_rope(rp, **dict(dict(q=q, k=k, pos=pos), **bad))
    for sec in ([64, 1], [], [10, 10, 10, 10, 24], [-1, 65]):
        with pytest.raises(ValueError, match="sections"):
            mp.RopeParams(128, sections=sec)


def test_attention_workspace_grows_with_the_table():
    # The calls with a window run on the workspace of their table: one for a longer table serves a shorter view of it,
    # up to the longest table that is allowed (2^30 tokens, whose blocks over 64 tiles pass an int's count).
    off = _off(*range(9))  # eight single tokens
    for kind in (bd.MAP_CACHE_BF16, bd.MAP_CACHE_MXFP4):
        c = _cache(type=kind, page=128, n_kv_heads=16)
        sizes = [bd.lib().map_cache_attention_workspace(ctypes.byref(c), 8, 16, 1 << w, off) for w in range(24)]
        assert sizes[0] > 0 and sizes == sorted(sizes)
        assert bd.lib().map_cache_attention_workspace(ctypes.byref(c), 8, 16, (1 << 23) + 1, off) == 0


def test_binding_refuses_rows_that_differ():
    rp, pos = mp.RopeParams(64), torch.zeros(5, dtype=torch.int32)
    with pytest.raises(ValueError, match="6 rows"):  # (its last row would come back unwritten)
        mp.map_qk_norm_rope(rp, torch.zeros(5, 4, 64), torch.zeros(6, 2, 64), pos)


@pytest.mark.parametrize("bad", [dict(window=1 << 31), dict(sinks=(1 << 32) + 4), dict(sinks=-1)])
def test_binding_refuses_sizes_past_an_int(bad):
    d = _cpu("bf16")
    with pytest.raises(ValueError, match="31 bits"):
        mp.map_cache_attention(d["cache"], d["table"], d["lens"], d["q"], d["off"], **bad)


@pytest.mark.parametrize("few", [1, 16])
@pytest.mark.parametrize("prompts", [[17], [40, 100]])
def test_attention_workspace_holds_the_prompts_rows_alone(few, prompts):
    # The parts of divided prompts are for the prompts' rows: sequences of few rows beside them need no room there.
    def size(n):
        off = [0]
        for x in n:
            off.append(off[-1] + x)
        return bd.lib().map_cache_attention_workspace(ctypes.byref(_cache(n_kv_heads=8, page=64)), len(n), 32, 512, _off(*off))

    alone, beside = size(prompts), size([few] * 100 + prompts[:1] + [few] * 150 + prompts[1:])
    assert alone > 1 << 20
    assert beside <= alone + size([few] * 250)


@pytest.mark.parametrize("of,current", [("cuda:1", 0), ("cuda:0", 0), ("cuda:2", 1), ("cpu", 0)])
def test_attention_workspace_is_sized_on_the_caches_device(monkeypatch, of, current):
    # The division, and with it the size, follows the current device's compute units: it has to be the cache's.
    seen, now = [], [current]

    class Guard:
        def __init__(self, device):
            self.to = torch.device(device).index

        def __enter__(self):
            self.was, now[0] = now[0], self.to

        def __exit__(self, *_):
            now[0] = self.was

    class Lib:
        @staticmethod
        def map_cache_attention_workspace(*_):
            seen.append(now[0])
            return 512

    cache = _cpu()["cache"]
    cache.device = torch.device(of)
    monkeypatch.setattr(bd, "lib", lambda: Lib)
    monkeypatch.setattr(bd, "_workspace", lambda nbytes, device: (nbytes, device))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", Guard)
    got = mp.cache_attention_workspace(cache, [0, 2, 5], 8, torch.zeros(2, 3, dtype=torch.int32))
    assert got == (512, cache.device) and now == [current]
    assert seen == [current if of == "cpu" else cache.device.index]


@pytest.mark.parametrize("missing", ["k_scale", "v_scale"])
@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_from_tensors_refuses_one_scale(kind, missing):
    c, s = mp.KVCache(2, 16, 1, 64, kind, device="cpu"), torch.zeros(2, 1, 16, 2, dtype=torch.uint8)
    with pytest.raises((ValueError, TypeError), match="scale"):
        mp.KVCache.from_tensors(c.k, c.v, **{"v_scale" if missing == "k_scale" else "k_scale": s})
    again = mp.KVCache.from_tensors(c.k, c.v, c.k_scale, c.v_scale)
    assert again.kind == kind and again.head_dim == 64
