"""The calls around the language model's key/value cache whose speed is measured.

Three kinds of pass, each through the library's Python entry points when
``own`` is set, and in elementary torch operations otherwise:

  rope    map_qk_norm_rope: RMS norms of the query and key heads and the
          rotation by positions of one to three axes (time, height, width)
  store   map_cache_append of new keys and values to their pages, then
          map_cache_read of the same slots (what the cache now holds for them)
  attend  map_cache_attention over the pages, for single tokens, for a few
          rows behind a long cache and for whole prompts

The cache is a pool of pages; a sequence's table names its pages in order.
Pages hold bfloat16, or four bits a value with one power of two for each 32
values along the head (MXFP4).  Inputs are drawn on the GPU from the seed:
keys have a few channels of larger spread, as they do behind a rotation, pages
lie in the pool in random order, and positions are those of a question behind
a grid of image or video tokens.
"""
import math

import torch

own = False
DEV = "cuda"
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


def listed():
    return [
        # Four sequences' next token: the rotation of a decode step, the smallest call.
        dict(name="rope_step_4", kind="rope", dtype="bf16", R=4, Hq=28, Hkv=4, Dh=128, rot=128, axes=3, mixed=False, norm=True),
        # One image pruned to 160 tokens and its question (224 rows) in float32, half of each head rotated.
        dict(name="rope_224_f32", kind="rope", dtype="f32", R=224, Hq=32, Hkv=32, Dh=128, rot=64, axes=2, mixed=True, norm=False),
        # Eight clips of 4608 video tokens with their questions: three axes and head norms, the largest prompt.
        dict(name="rope_video_37600", kind="rope", dtype="bf16", R=37600, Hq=28, Hkv=4, Dh=128, rot=128, axes=3, mixed=False, norm=True),
        # A decode step's keys and values of 16 sequences into 4-bit pages.
        dict(name="store_step_16_mxfp4", kind="store", cache="mxfp4", B=16, n_lo=1, n_hi=1, past_lo=100, past_hi=3000, Hkv=32, Dh=128, page=16),
        # Four unpruned images with ragged questions into bfloat16 pages.
        dict(name="store_4x2944_bf16", kind="store", cache="bf16", B=4, n_lo=2896, n_hi=3008, past_lo=0, past_hi=0, Hkv=32, Dh=128, page=64),
        # Eight video clips with their questions behind a short system prompt into 4-bit pages.
        dict(name="store_8x4700_mxfp4", kind="store", cache="mxfp4", B=8, n_lo=4640, n_hi=4736, past_lo=11, past_hi=45, Hkv=8, Dh=128, page=32),
        # The next token of one pruned sequence: latency.
        dict(name="attend_step_1_pruned", kind="attend", cache="bf16", B=1, n_lo=1, n_hi=1, past_lo=230, past_hi=260, Hq=32, Hkv=32, Dh=128, page=64, window=0, sinks=0),
        # The next token of 16 unpruned sequences: the cache that the pruning avoids.
        dict(name="attend_step_16_bf16", kind="attend", cache="bf16", B=16, n_lo=1, n_hi=1, past_lo=2896, past_hi=3008, Hq=32, Hkv=32, Dh=128, page=64, window=0, sinks=0),
        # The next token of 32 long conversations over 4-bit pages with shared heads.
        dict(name="attend_step_32_mxfp4", kind="attend", cache="mxfp4", B=32, n_lo=1, n_hi=1, past_lo=4096, past_hi=32768, Hq=28, Hkv=4, Dh=128, page=64, window=0, sinks=0),
        # A few guessed tokens of eight sequences, through a sliding window with four first tokens.
        dict(name="attend_draft_8_window", kind="attend", cache="bf16", B=8, n_lo=3, n_hi=6, past_lo=6000, past_hi=12000, Hq=32, Hkv=8, Dh=64, page=16, window=4096, sinks=4),
        # The prompt of one unpruned image and its question.
        dict(name="attend_prompt_2944", kind="attend", cache="bf16", B=1, n_lo=2944, n_hi=2944, past_lo=0, past_hi=0, Hq=32, Hkv=32, Dh=128, page=64, window=0, sinks=0),
        # Two video prompts over 4-bit pages, each row seeing two frames back and the first 64 tokens.
        dict(name="attend_video_2x4700", kind="attend", cache="mxfp4", B=2, n_lo=4640, n_hi=4736, past_lo=11, past_hi=45, Hq=28, Hkv=4, Dh=128, page=32, window=1152, sinks=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _largest(total, limit):
    return max(1, int(limit // max(1, total)))


def draw(rng):
    kind = rng.choice(("rope", "store", "attend", "attend"))
    Dh = rng.choice((64, 128, 128))
    Hkv = rng.choice((1, 2, 4, 8, 32))
    page = rng.choice((16, 32, 64, 128))
    if kind == "rope":
        rot = rng.choice((Dh, Dh, Dh // 2))
        Hq = Hkv * rng.choice((1, 2, 7) if Hkv < 32 else (1,))
        # at most the values of the listed video case, in bytes
        dtype = rng.choice(("bf16", "bf16", "f32"))
        R = min(_log_int(rng, 1, 40000), _largest((Hq + Hkv) * Dh * (2 if dtype == "bf16" else 4), 3.0e8))
        return dict(kind="rope", dtype=dtype, R=R, Hq=Hq, Hkv=Hkv, Dh=Dh, rot=rot, axes=rng.choice((1, 2, 3)),
                    mixed=rng.random() < 0.5, norm=rng.random() < 0.6)
    cache = rng.choice(("bf16", "mxfp4"))
    if kind == "store":
        n = _log_int(rng, 1, 4736)
        B = min(_log_int(rng, 1, 64), _largest(n * Hkv * Dh, 4.5e7))
        return dict(kind="store", cache=cache, B=B, n_lo=max(1, n - n // 3), n_hi=n, past_lo=0, past_hi=rng.choice((0, 40, 3000)),
                    Hkv=Hkv, Dh=Dh, page=page)
    Hq = Hkv * rng.choice((1, 2, 4, 7) if Hkv < 32 else (1,))
    form = rng.choice(("step", "step", "few", "prompt"))
    n = 1 if form == "step" else _log_int(rng, 2, 64) if form == "few" else _log_int(rng, 64, 2944)
    past = _log_int(rng, 1, 32768) if form != "prompt" else rng.choice((0, 0, _log_int(rng, 1, 2000)))
    B = _log_int(rng, 1, 64)
    B = min(B, _largest((past + n) * Hkv * Dh, 1.9e8), _largest((past + n) * n * Hq * Dh, 3.5e10))
    window = rng.choice((0, 0, _log_int(rng, 1, 8192)))
    return dict(kind="attend", cache=cache, B=B, n_lo=max(1, n - n // 3), n_hi=n, past_lo=max(0, past // 2), past_hi=past, Hq=Hq,
                Hkv=Hkv, Dh=Dh, page=page, window=window, sinks=rng.choice((0, 4, 64)) if window else 0)


# ------------------------------------------------------------------ sizes
def _lengths(case):
    """Each sequence's new rows and its tokens so far, from the case alone."""
    B = case["B"]
    n = [case["n_lo"] + (b * 37 + 11) % (case["n_hi"] - case["n_lo"] + 1) for b in range(B)]
    past = [case["past_lo"] + (b * 7919 + 5003) % (case["past_hi"] - case["past_lo"] + 1) for b in range(B)]
    return n, past


def _seen(i, case):
    """How many tokens the row at index i of its sequence sees."""
    w, s = case["window"], case["sinks"]
    return i + 1 if w == 0 or i < w else w + min(s, i + 1 - w)


def _sections(rot, axes):
    half = rot // 2
    if axes == 1:
        return [half]
    if axes == 2:
        return [half // 2, half - half // 2]
    t = half // 4
    return [t, (half - t) // 2, half - t - (half - t) // 2]


def _token_bytes(cache, Dh):
    """One token's key (or value) of one head."""
    return 2 * Dh if cache == "bf16" else Dh // 2 + Dh // 32


def work(case):
    if case["kind"] == "rope":
        heads, es = case["Hq"] + case["Hkv"], 2 if case["dtype"] == "bf16" else 4
        values = case["R"] * heads * case["Dh"]
        return {"bytes": 2 * values * es + 4 * case["R"] * case["axes"] + (2 * case["Dh"] * es if case["norm"] else 0),
                "flops": (9 if case["norm"] else 3) * values}
    n, past = _lengths(case)
    if case["kind"] == "store":
        rows = sum(n) * case["Hkv"]
        return {"bytes": 2 * rows * (4 * case["Dh"] + 2 * _token_bytes(case["cache"], case["Dh"])), "flops": 0}
    tokens = pairs = 0
    for r, p in zip(n, past):
        first = _seen(p, case)
        tokens += min(p + r, first + r - 1 if case["window"] else p + r)
        full = range(p, p + r)
        pairs += sum(_seen(i, case) for i in full) if case["window"] else r * p + r * (r + 1) // 2
    return {"bytes": 2 * tokens * case["Hkv"] * _token_bytes(case["cache"], case["Dh"]) + 2 * sum(n) * case["Hq"] * case["Dh"] * 2,
            "flops": 4 * case["Dh"] * case["Hq"] * pairs}


# ----------------------------------------------------------------- inputs
def _normal(g, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _positions(g, R, axes):
    """Question tokens behind a grid: time, height and width of each row."""
    r = torch.arange(R, device=DEV)
    t, y, x = r // 576, (r // 24) % 24, r % 24
    start = int(torch.randint(0, 300, (1,), generator=g, device=DEV))
    rows = torch.stack([r, y, x] if axes == 1 else [y, x, t] if axes == 2 else [t, y, x])[:axes] + start
    return rows.to(torch.int32).contiguous()


def _spread(g, Dh):
    c = torch.ones(Dh, device=DEV)
    c[torch.randint(0, Dh, (4,), generator=g, device=DEV)] = 4.0
    return c


def _quantise(x):
    """bf16 values [..., Dh] -> codes [..., Dh / 2] (two to a byte, the even
    one low) and scale bytes [..., Dh / 32]: 2^e is the smallest power of two
    with max <= 7 * 2^e, values go to the nearest level, ties to the even
    code; a block with an infinity or a NaN has scale byte 255."""
    f = x.float().unflatten(-1, (-1, 32))
    big = f.abs().amax(-1)
    m, ex = torch.frexp(torch.where(torch.isfinite(big), big, torch.zeros_like(big)))
    e = torch.where(m > 0.875, ex - 2, ex - 3)
    e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(min=-126)
    y = torch.where(torch.isfinite(big)[..., None], torch.ldexp(f, -e[..., None]), torch.zeros_like(f))
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + (a >= 1.75).to(torch.uint8)
            + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5.0).to(torch.uint8))
    code = (code | (torch.signbit(y).to(torch.uint8) << 3)).flatten(-2)
    scale = torch.where(torch.isfinite(big), e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _values(codes, scales):
    """What codes and scale bytes stand for, in float32."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    v = level[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()].unflatten(-1, (-1, 32))
    s = torch.where(scales == 255, torch.full_like(scales, 0, dtype=torch.float32) + float("nan"),
                    torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.to(torch.int32) - 127))
    return (v * s[..., None]).flatten(-2)


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if case["kind"] == "rope":
        R, Dh, dt = case["R"], case["Dh"], torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s = dict(q=_normal(g, (R, case["Hq"], Dh), dt), k=_normal(g, (R, case["Hkv"], Dh), dt, 2.0),
                 pos=_positions(g, R, case["axes"]), q_norm=None, k_norm=None)
        if case["norm"]:
            s["q_norm"], s["k_norm"] = (1.0 + _normal(g, (2, Dh), scale=0.1)).to(dt).unbind(0)
        return s
    n, past = _lengths(case)
    B, Hkv, Dh, page = case["B"], case["Hkv"], case["Dh"], case["page"]
    lens = [a + b for a, b in zip(n, past)]
    off = [0]
    for r in n:
        off.append(off[-1] + r)
    wide = -(-max(lens) // page)
    n_pages = B * wide + 3
    table = torch.randperm(n_pages, generator=g, device=DEV)[:B * wide].view(B, wide).to(torch.int32).contiguous()
    s = dict(table=table, lens=torch.tensor(lens, dtype=torch.int32, device=DEV), off=off, n_pages=n_pages, longest=max(lens), most=max(n))
    if case["kind"] == "store":
        s["k"] = (_normal(g, (off[-1], Hkv, Dh)) * _spread(g, Dh)).to(torch.bfloat16)
        s["v"] = _normal(g, (off[-1], Hkv, Dh), torch.bfloat16)
        s["slots"] = torch.cat([torch.arange(p, p + r, dtype=torch.int32, device=DEV) for r, p in zip(n, past)])
    else:
        s["q"] = _normal(g, (off[-1], case["Hq"], Dh), torch.bfloat16, 1.5)
    shape = (n_pages, Hkv, page)
    for name in ("k_pool", "v_pool"):
        if case["kind"] == "store":
            pool = torch.zeros(shape + (Dh,), dtype=torch.bfloat16, device=DEV)
        else:
            pool = _normal(g, shape + (Dh,), torch.bfloat16)
            if name == "k_pool":
                pool *= _spread(g, Dh).to(torch.bfloat16)
        if case["cache"] == "mxfp4":
            s[name], s[name[0] + "_scale"] = _quantise(pool)
        else:
            s[name], s[name[0] + "_scale"] = pool, None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if case["kind"] != "rope":
        s["off_dev"] = torch.tensor(s["off"], dtype=torch.int64, device=DEV)
    if own:  # the handles that a program keeps: rotation, page pool, row offsets, scratch memory
        import paper_2608_06411_amd as mp
        if case["kind"] == "rope":
            s["rope"] = mp.RopeParams(head_dim=case["Dh"], rot_dim=case["rot"], sections=_sections(case["rot"], case["axes"]),
                                      interleaved=case["mixed"], theta=10000.0, eps=EPS)
        else:
            s["cache"] = mp.KVCache.from_tensors(s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
            s["rows"] = mp.SeqOffsets(s["off"])
            if case["kind"] == "attend":
                s["ws"] = mp.cache_attention_workspace(s["cache"], s["rows"], case["Hq"], s["table"])
    return s


# ------------------------------------------------------------- plain forms
def _axis_of_pair(rot, axes, mixed):
    """The position axis that turns each pair of a head."""
    sec = _sections(rot, axes)
    if not mixed:
        return torch.repeat_interleave(torch.arange(axes), torch.tensor(sec))
    # pair i belongs to axis i mod A while that axis has pairs left: sort the
    # pairs of all axes by (place within the axis, axis)
    a = torch.repeat_interleave(torch.arange(axes), torch.tensor(sec))
    place = torch.cat(tuple(map(torch.arange, sec)))
    return a[torch.argsort(place * axes + a)]


def _rope_plain(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    axis = _axis_of_pair(rot, c["axes"], c["mixed"]).to(DEV)
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=DEV) * 2 / rot)
    angle = s["pos"].double()[axis].T * freq  # [R, half]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x, g):
        y = x.float()
        if g is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * g.float()
        a, b = y[..., :half], y[..., half:rot]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, y[..., rot:]), -1).to(x.dtype)

    return turn(s["q"], s["q_norm"]), turn(s["k"], s["k_norm"])


def _places(s):
    """Sequence of each new row, and its slot."""
    off = s["off_dev"]
    r = torch.arange(s["off"][-1], device=DEV)
    b = torch.bucketize(r, off[1:], right=True)
    return b, s["lens"].long()[b] - (off[b + 1] - r)


def _store_plain(s):
    page = s["case"]["page"]
    b, slot = _places(s)
    at, place = s["table"].long()[b, slot // page], slot % page
    got = s["slots"].long()
    at_r, place_r = s["table"].long()[b, got // page], got % page

    def one(x, pool, scale):
        if scale is None:
            pool[at, :, place] = x
            return pool[at_r, :, place_r]
        pool[at, :, place], scale[at, :, place] = _quantise(x)
        return _values(pool[at_r, :, place_r], scale[at_r, :, place_r]).to(torch.bfloat16)

    return one(s["k"], s["k_pool"], s["k_scale"]), one(s["v"], s["v_pool"], s["v_scale"])


def _attend_plain(s):
    c = s["case"]
    Hkv, G, Dh, L = c["Hkv"], c["Hq"] // c["Hkv"], c["Dh"], s["longest"]
    B, nm = c["B"], s["most"]
    table = s["table"].long()

    def dense(pool, scale):  # [B, Hkv, L, Dh] in float32
        x = pool[table]
        x = x.float() if scale is None else _values(x, scale[table])
        return x.transpose(1, 2).reshape(B, Hkv, -1, Dh)[:, :, :L].contiguous()

    off, lens = s["off_dev"], s["lens"].long()
    n = off[1:] - off[:-1]
    i = torch.arange(nm, device=DEV)
    row = (off[:-1, None] + i).clamp(max=s["off"][-1] - 1)  # [B, nm], past a sequence's rows: not used
    q = s["q"].float()[row].view(B, nm, Hkv, G, Dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, nm * G, Dh)
    at = (lens - n)[:, None] + i  # each row's index in its sequence
    j = torch.arange(L, device=DEV)
    see = (j <= at[..., None]) & (j < lens[:, None, None])
    if c["window"]:
        see &= (at[..., None] - j < c["window"]) | (j < c["sinks"])
    z = torch.matmul(q, dense(s["k_pool"], s["k_scale"]).transpose(2, 3).contiguous()) / math.sqrt(Dh)
    z = z.view(B, Hkv, nm, G, L).masked_fill(~see[:, None, :, None], -math.inf)
    z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-3e38))
    z = (z / z.sum(-1, keepdim=True).clamp(min=1e-30)).view(B, Hkv, nm * G, L)
    o = torch.matmul(z, dense(s["v_pool"], s["v_scale"]))
    o = o.view(B, Hkv, nm, G, Dh).permute(0, 2, 1, 3, 4).reshape(B, nm, c["Hq"], Dh).to(torch.bfloat16)
    b, slot = _places(s)
    return o[b, slot - (lens - n)[b]]


def run(s):
    c = s["case"]
    if c["kind"] == "rope":
        if own:
            import paper_2608_06411_amd as mp
            q, k = mp.map_qk_norm_rope(s["rope"], s["q"], s["k"], s["pos"], s["q_norm"], s["k_norm"])
        else:
            q, k = _rope_plain(s)
        return {"q": q, "k": k}
    if c["kind"] == "store":
        if own:
            import paper_2608_06411_amd as mp
            mp.map_cache_append(s["cache"], s["table"], s["lens"], s["k"], s["v"], s["rows"])
            k, v = mp.map_cache_read(s["cache"], s["table"], s["lens"], s["rows"], slots=s["slots"])
        else:
            k, v = _store_plain(s)
        return {"k": k, "v": v}
    if own:
        import paper_2608_06411_amd as mp
        return mp.map_cache_attention(s["cache"], s["table"], s["lens"], s["q"], s["rows"], window=c["window"], sinks=c["sinks"],
                                      workspace=s["ws"])
    return _attend_plain(s)


# ----------------------------------------------------------------- 64 bits
def _nearest_double(x):
    """What a 4-bit page holds for values x [..., Dh] (float64): the format's
    definition, by rounding to the spacing of the levels at each value."""
    f = x.unflatten(-1, (-1, 32))
    big = f.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(big > 0, big, torch.ones_like(big)) / 7.0))
    e = torch.where(big > 7.0 * 2.0 ** e, e + 1, torch.where(big <= 3.5 * 2.0 ** e, e - 1, e))
    e = torch.where(big > 0, e, torch.full_like(e, -126.0)).clamp(min=-126.0)
    y = f / 2.0 ** e
    gap = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0)).double()
    return ((torch.round(y / gap) * gap).clamp(-6, 6) * 2.0 ** e).flatten(-2)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rope":
        rot, axes = case["rot"], case["axes"]
        left, order = _sections(rot, axes), []
        if case["mixed"]:
            a = 0
            while len(order) < rot // 2:
                if left[a % axes]:
                    left[a % axes] -= 1
                    order.append(a % axes)
                a += 1
        else:
            for a in range(axes):
                order += [a] * left[a]
        out = {}
        for name in ("q", "k"):
            x = s[name].double()
            if s[name + "_norm"] is not None:
                x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * s[name + "_norm"].double()
            y = x.clone()
            for i in range(rot // 2):
                t = s["pos"][order[i]].double() * math.exp(-2.0 * i / rot * math.log(10000.0))
                z = torch.complex(x[..., i], x[..., i + rot // 2]) * torch.polar(torch.ones_like(t), t)[:, None]
                y[..., i], y[..., i + rot // 2] = z.real, z.imag
            out[name] = y
        return out
    if case["kind"] == "store":
        # the rows come back from the slots they went to
        return {name: s[name].double() if case["cache"] == "bf16" else _nearest_double(s[name].double()) for name in ("k", "v")}
    n, past = _lengths(case)
    G, page, Dh = case["Hq"] // case["Hkv"], case["page"], case["Dh"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        lo, hi, L = s["off"][b], s["off"][b + 1], n[b] + past[b]
        pages = s["table"][b, :-(-L // page)].long()
        at = torch.arange(past[b], L, device=DEV)[:, None]
        j = torch.arange(L, device=DEV)[None]
        hide = j > at
        if case["window"]:
            hide |= (j <= at - case["window"]) & (j >= case["sinks"])
        for h in range(case["Hkv"]):
            kv = []
            for name in ("k", "v"):
                x = s[name + "_pool"][pages, h].flatten(0, 1)[:L]
                if case["cache"] == "mxfp4":
                    two = torch.stack((x % 16, x // 16), -1).flatten(1).long()
                    p = 2.0 ** (s[name + "_scale"][pages, h].flatten(0, 1)[:L].double() - 127.0)
                    x = level[two] * p.repeat_interleave(32, dim=1)
                kv.append(x.double())
            for g in range(G):
                z = s["q"][lo:hi, h * G + g].double() @ kv[0].T.contiguous() / math.sqrt(Dh)
                z[hide] = -math.inf
                out[lo:hi, h * G + g] = torch.softmax(z, dim=1) @ kv[1]
    return out
