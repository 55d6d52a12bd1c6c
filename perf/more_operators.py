"""What the operators of long windows are timed on: models that norm their queries and keys head by head, rotate part of a head or
by scaled frequencies, and read a few blocks of a long cache that a cheap score selects for each query; the work that a
streaming-video serving program has them do, through the public entry points (`binding`).

Kinds of case:
  write    one layer's fresh tokens: queries and keys normed head by head and rotated, keys and values written into the paged cache
  turn     position correction and repacking of cached rows, all layers, by a table of frequencies of part or all of a head
  bounds   what the blocks of a cache hold: each channel's largest and smallest key, in whole numbers with a power of two a block
  select   which blocks every query reads, by a bound on its products with their keys
  attn     attention of every query over the blocks selected for it: single tokens, questions and whole windows

Inputs come from the seed alone and are drawn on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _write(name, n_tok, **kw):
    c = dict(name=name, kind="write", n_tok=n_tok, q_heads=28, kv_heads=4, head_dim=128, rotary=128, dtype="bf16", axes="sections",
             style="half", base=1e6, scaled=False, weights=True, layout="slot")
    c.update(kw)
    return c


def _turn(name, n_rows, layers, **kw):
    c = dict(name=name, kind="turn", n_rows=n_rows, layers=layers, kv_heads=4, head_dim=128, rotary=128, dtype="bf16", axes="none",
             style="half", base=1e6, scaled=True, layout="slot")
    c.update(kw)
    return c


def _long(kind, name, n_streams, q_len, kv_len, **kw):
    c = dict(name=name, kind=kind, n_streams=n_streams, q_len=q_len, kv_len=kv_len, ragged=0.5, q_heads=28, kv_heads=4, head_dim=128,
             dtype="bf16", where="tail", layout="slot", block=64, n_select=16, n_first=1, n_last=2)
    if kind == "bounds":
        c["new"] = 0                # entries at a window's end that are new, 0: all of them
    if kind == "attn":
        c["lse"] = True
    c.update(kw)
    return c


def listed():
    return [
        # one new token of one stream, one layer: nothing but a launch and latency
        _write("write_one_token", 1),
        # the executed tokens of a batch of 64 streams, one layer
        _write("write_window_64", 22804, q_heads=32, kv_heads=8, axes="none", scaled=True),
        # the reused rows of one stream's window, every layer; half of a head is rotated
        _turn("turn_one_stream", 495, 28, rotary=64),
        # the reused rows of the long window, every layer, keys of three-axis rotary embeddings
        _turn("turn_long_window", 15548, 28, axes="interleaved"),
        # 32 streams over long ragged caches have written a token each: the last block of each is made anew
        _long("bounds", "bounds_tokens_32", 32, 1, 17630, new=1),
        # 32 long windows have slid: every block is made anew
        _long("bounds", "bounds_windows_32", 32, 1, 17630),
        # a token of one stream chooses among the blocks of the long window
        _long("select", "select_token", 1, 1, 17630, ragged=0.0),
        # the executed tokens of the long window choose
        _long("select", "select_window", 1, 2082, 17630, ragged=0.0, where="spread"),
        # one stream answers: a single token reads its share of the long window
        _long("attn", "attn_token", 1, 1, 17630, ragged=0.0),
        # 64 streams answer at once, a token each, over long ragged caches
        _long("attn", "attn_tokens_64", 64, 1, 17630, q_heads=32, kv_heads=8),
        # the joint prefill of the long window's refreshed and new tokens
        _long("attn", "attn_window", 1, 2082, 17630, ragged=0.0, where="spread"),
        # single precision, head_dim 64, questions over odd lengths in small blocks
        _long("attn", "attn_f32_d64", 3, 337, 2439, dtype="f32", q_heads=16, head_dim=64, where="spread", layout="head", block=16, n_select=24),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((28, 4), (32, 8), (16, 4), (12, 3), (8, 8), (2, 1), (16, 1), (7, 1))


def draw(rng):
    kind = rng.choice(("write", "turn", "bounds", "select", "select", "attn", "attn", "attn"))
    hq, hkv = rng.choice(HEADS)
    d = rng.choice((64, 128, 128))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    common = dict(kv_heads=hkv, head_dim=d, dtype=dtype, layout=rng.choice(("head", "slot")))
    turned = dict(rotary=rng.choice((d, d, d // 2, d // 4)), axes=rng.choice(("none", "sections", "interleaved")), style=rng.choice(("half", "pairs")),
                  base=rng.choice((1e4, 1e6)), scaled=rng.random() < 0.5)
    if kind == "write":
        return _write(None, _log(rng, 1, 11000), q_heads=hq, weights=rng.random() < 0.8, **turned, **common)
    if kind == "turn":
        layers = rng.randint(1, 28)
        return _turn(None, _log(rng, 1, max(2, 200000 // layers // max(1, hkv // 4))), layers, **turned, **common)
    block = rng.choice((16, 32, 64, 64))
    # (a selection among few blocks is the same for all inputs)
    kv = _log(rng, 12 * block if kind == "select" else 1, 17000)
    n = _log(rng, 1, max(1, min(64, 250000 // kv)))
    n_select = _log(rng, 2, 1024 // block) if kind != "select" else _log(rng, 2, min(1024 // block, kv // block // 3))
    n_first = rng.randint(0, min(2, n_select - 1))
    common.update(q_heads=hq, block=block, n_select=n_select, n_first=n_first, n_last=rng.randint(0, min(4, n_select - 1 - n_first)),
                  ragged=rng.choice((0.0, 0.5, 0.9)), where=rng.choice(("tail", "spread")))
    if kind == "bounds":
        return _long(kind, None, n, 1, kv, new=rng.choice((0, 0, 1, _log(rng, 1, kv))), **common)
    # queries a stream: one token, or as many as keep the whole within the long window's
    if kind == "select":
        most = 2300000 // (n * hkv * -(-kv // block))
    else:
        most = 8500000 // (n * hkv * n_select * block) // (1 if dtype == "bf16" else 4)
    q = 1 if rng.random() < 0.3 else _log(rng, 1, max(1, min(most, kv, 2100)))
    if kind == "attn":
        common["lse"] = rng.random() < 0.5
    return _long(kind, None, n, q, kv, **common)


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed, device=None):
    g = torch.Generator(device=device or DEV)
    g.manual_seed(seed)
    return g


def _lengths(n, longest, ragged):
    """n lengths from longest*(1-ragged) to longest, the longest among them; the same for every seed, as the outputs' shapes follow them."""
    g = _gen(1000 * n + longest, "cpu")
    u = torch.rand((n,), generator=g, dtype=torch.float64)
    length = (longest * (1.0 - ragged * u)).round().clamp(min=1).long()
    length[int(torch.randint(0, n, (1,), generator=g))] = longest
    return length.tolist()


def _axis_of_pair(axes, pairs):
    if axes == "none":
        return None
    if axes == "interleaved":
        return [i % 3 for i in range(pairs)]
    a, b = pairs // 4, pairs // 4 + 3 * pairs // 8
    return [0 if i < a else 1 if i < b else 2 for i in range(pairs)]


def _inv_freq(c):
    """Frequencies of the rotated pairs, 32 bits.  Scaled for a context four times as long: slow pairs turn a quarter as fast, fast ones as
    they were, a ramp between."""
    r = c["rotary"]
    f = torch.tensor([c["base"] ** (-2.0 * i / r) for i in range(r // 2)], dtype=torch.float64)
    if c["scaled"]:
        ramp = ((32768 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f = f * ramp + f / 4 * (1 - ramp)
    return f.float().to(DEV)


def _turned(c):
    """Frequencies, axes, and the factor that goes with scaled frequencies."""
    axis = _axis_of_pair(c["axes"], c["rotary"] // 2)
    return dict(inv_freq=_inv_freq(c), axis=None if axis is None else torch.tensor(axis, dtype=torch.uint8, device=DEV),
                amplitude=0.1 * math.log(4.0) + 1.0 if c["scaled"] else 1.0)


def _positions(n, g, axes):
    """Positions of n tokens of a window: frames far into a stream, patches of a 26 x 46 grid; text has its position on all axes."""
    t = torch.randint(0, 60000, (n,), generator=g, dtype=torch.int32)
    if axes == "none":
        return t
    p = torch.stack([t, torch.randint(0, 26, (n,), generator=g, dtype=torch.int32), torch.randint(0, 46, (n,), generator=g, dtype=torch.int32)], 1)
    text = torch.rand((n,), generator=g) < 0.1
    p[text] = t[text][:, None].expand(-1, 3)
    return p.contiguous()


def _blocks(lengths, g):
    """A shuffled block table for sequences of these lengths, and how many blocks there are."""
    need = [-(-n // 16) for n in lengths]
    ids = torch.randperm(sum(need), generator=g)
    table = torch.zeros((len(need), max(need)), dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n].int()
        at += n
    return table, at


def prepare(case, seed):
    return {"write": _prepare_write, "turn": _prepare_turn}.get(case["kind"], _prepare_long)(case, seed)


def _prepare_write(c, seed):
    g, h = _gen(seed), _gen(seed, "cpu")
    n, hq, hk, d, dt = c["n_tok"], c["q_heads"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    # queries, keys and values as one projection leaves them: tokens of different size, for the norms to level
    qkv = torch.randn((n, (hq + 2 * hk) * d), generator=g, device=DEV) * torch.exp(0.5 * torch.randn((n, 1), generator=g, device=DEV))
    qkv = qkv.to(dt)
    n_slots = 16 * (-(-n // 16) + 7)
    weight = lambda: (1.0 + 0.3 * torch.randn((d,), generator=g, device=DEV)).to(dt) if c["weights"] else None
    shape = (n_slots, hk, d) if c["layout"] == "slot" else (hk, n_slots, d)
    pool = lambda: torch.zeros(shape, dtype=dt, device=DEV) if c["layout"] == "slot" else torch.zeros(shape, dtype=dt, device=DEV).transpose(0, 1)
    return dict(case=c, q=qkv[:, :hq * d], k=qkv[:, hq * d:(hq + hk) * d], v=qkv[:, (hq + hk) * d:], q_weight=weight(), k_weight=weight(),
                k_cache=pool(), v_cache=pool(), slot=torch.randperm(n_slots, generator=h)[:n].int().to(DEV),
                pos=_positions(n, h, c["axes"]).to(DEV), q_out=torch.empty((n, hq, d), dtype=dt, device=DEV), **_turned(c))


def _prepare_turn(c, seed):
    g, h = _gen(seed), _gen(seed, "cpu")
    n, layers, hk, d, dt = c["n_rows"], c["layers"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    # rows of the old window and their places in the new one: slots run on within cache blocks, as a refresh plan's do
    n_blocks = 2 * -(-n // 16)
    ids = torch.randperm(n_blocks, generator=h)
    run = lambda b: (b[:, None] * 16 + torch.arange(16)).flatten()[:n].int()
    shape = (layers, n_blocks * 16, hk, d) if c["layout"] == "slot" else (layers, hk, n_blocks * 16, d)
    pool = lambda: torch.randn(shape, generator=g, device=DEV).to(dt) if c["layout"] == "slot" else torch.randn(shape, generator=g, device=DEV).to(dt).transpose(1, 2)
    shift = torch.full((n,), -256 - 16 * int(torch.randint(0, 140, (1,), generator=h)), dtype=torch.int32)
    if c["axes"] != "none":
        shift = torch.stack([shift, torch.randint(-2, 3, (n,), generator=h, dtype=torch.int32), torch.randint(-2, 3, (n,), generator=h, dtype=torch.int32)], 1)
    return dict(case=c, k_pool=pool(), v_pool=pool(), src=run(ids[:n_blocks // 2]).to(DEV), dst=run(ids[n_blocks // 2:]).to(DEV),
                delta=shift.contiguous().to(DEV), **_turned(c))


def _prepare_long(c, seed):
    g, h = _gen(seed), _gen(seed, "cpu")
    b, hq, hk, d, dt = c["n_streams"], c["q_heads"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    kv = _lengths(b, c["kv_len"], c["ragged"])
    nq = [min(x, n) for x, n in zip(_lengths(b, c["q_len"], c["ragged"]), kv)]
    table, n_blocks = _blocks(kv, h)
    pos = []
    for n, x in zip(kv, nq):
        if c["where"] == "tail":
            pos.append(torch.arange(n - x, n))
        else:       # a block of refreshed rows somewhere in the window, and its end
            head = x // 2
            at = int(torch.randint(0, n - x + 1, (1,), generator=h))
            pos.append(torch.cat([torch.arange(at, at + head), torch.arange(n - (x - head), n)]))
    width = 16 * table.shape[1]
    st = dict(case=c, table=table.to(DEV), n_q=sum(nq), n_sel=-(-width // c["block"]), q_pos=torch.cat(pos).int().to(DEV),
              cu_q=torch.tensor([0] + nq).cumsum(0).int().to(DEV), kv_len=torch.tensor(kv).int().to(DEV),
              stream=torch.repeat_interleave(torch.arange(b), torch.tensor(nq)).to(DEV))
    # stretches of a window look alike (a region over some frames): their keys share a direction; a run of queries looks for three of
    # them, each head with a stress of its own
    shape = (n_blocks * 16, hk, d) if c["layout"] == "slot" else (hk, n_blocks * 16, d)
    view = lambda t: t if c["layout"] == "slot" else t.transpose(0, 1)
    stretch = torch.randn((b, -(-c["kv_len"] // 97), hk, d), generator=g, device=DEV)
    noise = lambda: view(torch.randn(shape, generator=g, device=DEV))
    keys = noise()
    entry = torch.arange(width, device=DEV)
    slot = (st["table"].long()[:, entry // 16] * 16 + entry % 16)
    held = entry[None] < st["kv_len"][:, None]
    of = stretch[:, (entry // 97).clamp(max=stretch.shape[1] - 1)]
    keys[slot[held]] = 0.7 * keys[slot[held]] + 0.7 * of[held]
    del of
    st["k_cache"] = keys.to(dt)
    if c["kind"] == "attn":
        st["v_cache"] = noise().to(dt)
    del keys
    if c["kind"] != "bounds":
        order = torch.arange(st["n_q"], device=DEV)
        pick = torch.randint(0, 1 << 30, (-(-st["n_q"] // 13), 3), generator=g, device=DEV)[order // 13] % (-(-st["kv_len"][st["stream"]] // 97))[:, None]
        wanted = stretch[st["stream"][:, None], pick]                                          # [n_q][3][hk][d]
        stress = torch.rand((st["n_q"], 3, hk, hq // hk, 1), generator=g, device=DEV)
        q = torch.randn((st["n_q"], hk, hq // hk, d), generator=g, device=DEV)
        for i in range(3):
            q += stress[:, i] * wanted[:, i, :, None]
        st["q"] = q.view(st["n_q"], hq, d).to(dt)
    st["bounds"] = torch.zeros((b, hk, st["n_sel"], 2, d), dtype=torch.int8, device=DEV)
    st["scales"] = torch.zeros((b, hk, st["n_sel"]), dtype=torch.uint8, device=DEV)
    st["since"] = None
    if c["kind"] != "bounds" or c["new"]:       # as earlier calls have left them
        _plain_bounds(st)
    if c["kind"] == "bounds" and c["new"]:
        st["since"] = (st["kv_len"] - c["new"]).clamp(min=0)
        first = st["since"] // c["block"]
        gone = torch.arange(st["n_sel"], device=DEV)[None] >= first[:, None]
        st["bounds"].masked_fill_(gone[:, None, :, None, None], 0)
        st["scales"].masked_fill_(gone[:, None], 0)
    if c["kind"] == "select":
        st["selected"] = torch.empty((st["n_q"], hk, c["n_select"]), dtype=torch.int32, device=DEV)
    if c["kind"] == "attn":
        st["selected"] = _plain_select(st)
        st["out"] = torch.empty_like(st["q"])
        st["stat"] = torch.empty((st["n_q"], hq), device=DEV) if c["lse"] else None
        del st["bounds"], st["scales"]
    if own and c["kind"] != "bounds":
        from paper_2604_06036_amd import binding as cs
        if c["kind"] == "select":
            nbytes = cs.cs_select_blocks_workspace(st["n_q"], b, hq, hk, d, table.shape[1], c["block"])
        else:
            nbytes = cs.cs_selected_attn_workspace(st["n_q"], b, hq, hk, d, c["block"], c["n_select"])
        st["ws"] = torch.empty((max(16, nbytes),), dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------------------------- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"write": _own_write, "turn": _own_turn, "bounds": _own_bounds, "select": _own_select, "attn": _own_attn}[kind](state)
    return {"write": _plain_write, "turn": _plain_turn, "bounds": _plain_bounds, "select": _plain_select, "attn": _plain_attn}[kind](state)


def _own_write(s):
    from paper_2604_06036_amd import binding as cs
    c = s["case"]
    cs.cs_norm_rope_refresh_scatter(s["q"], s["q_out"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["slot"], s["pos"], s["axis"], s["inv_freq"],
                                    s["k_cache"], s["v_cache"], c["n_tok"], c["q_heads"], c["kv_heads"], c["head_dim"], c["rotary"], s["q"].stride(0),
                                    s["k"].stride(0), s["v"].stride(0), s["k_cache"].stride(0), s["k_cache"].stride(1), EPS, s["amplitude"],
                                    cs.CS_ROPE_HALF_SPLIT if c["style"] == "half" else cs.CS_ROPE_INTERLEAVED, cs.dtype_code(s["q"]))
    return s["q_out"], s["k_cache"], s["v_cache"]


def _own_turn(s):
    from paper_2604_06036_amd import binding as cs
    c, k = s["case"], s["k_pool"]
    cs.cs_kv_rerotate_freqs(k, s["v_pool"], s["src"], s["dst"], s["delta"], s["axis"], s["inv_freq"], c["n_rows"], c["layers"], c["kv_heads"],
                            c["head_dim"], c["rotary"], k.stride(0), k.stride(1), k.stride(2),
                            cs.CS_ROPE_HALF_SPLIT if c["style"] == "half" else cs.CS_ROPE_INTERLEAVED, cs.dtype_code(k))
    return k, s["v_pool"]


def _own_bounds(s):
    from paper_2604_06036_amd import binding as cs
    c, k = s["case"], s["k_cache"]
    cs.cs_key_bounds(k, s["since"], s["kv_len"], s["table"], s["table"].shape[1], cs.CS_KV_BLOCK, c["block"], s["bounds"], s["scales"], c["n_streams"],
                     c["kv_heads"], c["head_dim"], k.stride(0), k.stride(1), cs.dtype_code(k))
    return s["bounds"], s["scales"]


def _own_select(s):
    from paper_2604_06036_amd import binding as cs
    c = s["case"]
    cs.cs_select_blocks(s["q"], s["bounds"], s["scales"], s["cu_q"], s["q_pos"], s["kv_len"], s["table"].shape[1], c["block"], c["n_select"], c["n_first"],
                        c["n_last"], s["selected"], s["n_q"], c["n_streams"], c["q_heads"], c["kv_heads"], c["head_dim"], cs.dtype_code(s["q"]), s["ws"])
    return s["selected"]


def _own_attn(s):
    from paper_2604_06036_amd import binding as cs
    c, k = s["case"], s["k_cache"]
    cs.cs_selected_attn(s["q"], k, s["v_cache"], s["cu_q"], s["q_pos"], s["kv_len"], s["table"], s["table"].shape[1], cs.CS_KV_BLOCK, s["selected"],
                        c["block"], c["n_select"], s["out"], s["stat"], s["n_q"], c["n_streams"], c["q_heads"], c["kv_heads"], c["head_dim"], k.stride(0),
                        k.stride(1), 1.0 / math.sqrt(c["head_dim"]), cs.dtype_code(k), s["ws"])
    return (s["out"], s["stat"]) if c["lse"] else s["out"]


def _cos_sin(pos, s, amplitude):
    """Cosine and sine of every (row, pair): the angles in 64 bits, since a far position loses them in 32."""
    p = pos.double()[:, None] if s["axis"] is None else pos.double()[:, s["axis"].long()]
    angle = p * s["inv_freq"].double()
    return (angle.cos() * amplitude).float(), (angle.sin() * amplitude).float()


def _rotate(x, cos, sin, style):
    """The first elements of x [..., d], as many as cos and sin [..., r/2] say, turned; the others as they are."""
    r = 2 * cos.shape[-1]
    y, rest = x[..., :r], x[..., r:]
    a, b = (y[..., :r // 2], y[..., r // 2:]) if style == "half" else (y[..., 0::2], y[..., 1::2])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    return torch.cat([ra, rb, rest] if style == "half" else [torch.stack([ra, rb], -1).flatten(-2), rest], -1)


def _plain_write(s):
    c = s["case"]
    n, d = c["n_tok"], c["head_dim"]
    cos, sin = (t[:, None] for t in _cos_sin(s["pos"], s, s["amplitude"]))

    def normed(x, weight):
        x = x.float().view(n, -1, d)
        return x if weight is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()

    slot, dt = s["slot"].long(), s["q"].dtype
    s["k_cache"][slot] = _rotate(normed(s["k"], s["k_weight"]), cos, sin, c["style"]).to(dt)
    s["v_cache"][slot] = s["v"].reshape(n, -1, d)
    return _rotate(normed(s["q"], s["q_weight"]), cos, sin, c["style"]).to(dt), s["k_cache"], s["v_cache"]


def _plain_turn(s):
    c, src, dst = s["case"], s["src"].long(), s["dst"].long()
    cos, sin = (t[None, :, None] for t in _cos_sin(s["delta"], s, 1.0))
    s["k_pool"][:, dst] = _rotate(s["k_pool"][:, src].float(), cos, sin, c["style"]).to(s["k_pool"].dtype)
    s["v_pool"][:, dst] = s["v_pool"][:, src]
    return s["k_pool"], s["v_pool"]


def _exponent(amax):
    """The least k >= -95 with amax <= 127 * 2^k, biased by 127."""
    return (((amax.view(torch.int32) + 0x1FFFF) >> 23) - 6).clamp(min=32)


def _times_power(x, biased):
    """x / 2^(biased - 127) in 64 bits, where no power underflows."""
    return x.double() * ((1150 - biased.long()) << 52).view(torch.float64)


def _plain_bounds(s):
    c, kv = s["case"], s["kv_len"].long()
    size = c["block"]
    first = torch.zeros_like(kv) if s["since"] is None else s["since"].long() // size
    count = s["n_sel"] if s["since"] is None else -(-c["new"] // size) + 1
    block = first[:, None] + torch.arange(count, device=kv.device)                             # [b][count]
    entry = block[..., None] * size + torch.arange(size, device=kv.device)
    held = (entry < kv[:, None, None])[..., None, None]
    table = s["table"].long().gather(1, (entry.flatten(1) // 16).clamp(max=s["table"].shape[1] - 1)).view_as(entry)
    k = s["k_cache"][table * 16 + entry % 16].float()                                          # [b][count][size][hk][d]
    high, low = k.masked_fill(~held, -math.inf).amax(2), k.masked_fill(~held, math.inf).amin(2)
    e = _exponent(torch.maximum(high.abs(), low.abs()).amax(-1))
    codes = torch.stack([torch.ceil(_times_power(high, e[..., None])), torch.floor(_times_power(low, e[..., None]))], -2).clamp(-128, 127)
    b, i = (block * size < kv[:, None]).nonzero(as_tuple=True)
    s["bounds"][b, :, block[b, i]] = codes[b, i].to(torch.int8)
    s["scales"][b, :, block[b, i]] = e[b, i].to(torch.uint8)
    return s["bounds"], s["scales"]


def _plain_select(s):
    c = s["case"]
    size, want, hk = c["block"], c["n_select"], c["kv_heads"]
    q = s["q"].float().unflatten(1, (hk, -1))                                                  # [n_q][hk][group][d]
    e = _exponent(q.abs().amax((-1, -2)))[..., None, None]
    codes = _times_power(q, e).round().float()
    # whole numbers below 2^24 throughout: the product is exact
    both = s["bounds"][s["stream"]].float()                                                    # [n_q][hk][n_sel][2][d]
    signed = torch.stack([codes.clamp(min=0), codes.clamp(max=0)], -2).flatten(-2).transpose(-1, -2).contiguous()
    score = torch.matmul(both.flatten(-2), signed).amax(-1)                                    # [n_q][hk][n_sel]
    score = score * ((s["scales"][s["stream"]].int() - 21).clamp(min=0) << 23).view(torch.float32)       # 2^(k - 21): in range for every k
    last = torch.minimum(s["q_pos"].long(), s["kv_len"].long()[s["stream"]] - 1)
    n = torch.where(last >= 0, last // size + 1, 0)[:, None, None]
    block = torch.arange(score.shape[-1], device=score.device)
    fixed = (block < c["n_first"]) | (block >= n - c["n_last"])
    score = torch.where(fixed, math.inf, score).masked_fill(block >= n, -math.inf)
    order = score.sort(dim=-1, descending=True, stable=True).indices[..., :want]
    kept = torch.where(order < n, order, 1 << 30).sort(-1).values
    kept = torch.where(kept < 1 << 30, kept, -1).int()
    return torch.cat([kept, kept.new_full(kept.shape[:-1] + (want - kept.shape[-1],), -1)], -1)


def _entries(s):
    """The entries that every query and kv head reads, whether they count, and their slots [n_q][hk][n_select * block]."""
    size = s["case"]["block"]
    entry = (s["selected"].long()[..., None] * size + torch.arange(size, device=s["q"].device)).flatten(-2)
    seen = (entry >= 0) & (entry <= torch.minimum(s["q_pos"].long(), s["kv_len"].long()[s["stream"]] - 1)[:, None, None])
    entry = torch.where(seen, entry, 0)
    table = s["table"].long()[s["stream"]].gather(1, (entry // 16).flatten(1)).view_as(entry)
    return seen, table * 16 + entry % 16


def _plain_attn(s):
    c = s["case"]
    seen, slot = _entries(s)
    head = torch.arange(c["kv_heads"], device=slot.device)[:, None]
    q = s["q"].float().unflatten(1, (c["kv_heads"], -1)) * (1.0 / math.sqrt(c["head_dim"]))
    x = torch.matmul(s["k_cache"][slot, head].float(), q.transpose(-1, -2).contiguous())       # [n_q][hk][entries][group]
    x = x.masked_fill(~seen[..., None], -math.inf)
    m = x.amax(-2, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(-2)
    out = torch.matmul(p.transpose(-1, -2).contiguous(), s["v_cache"][slot, head].float()) / total.clamp(min=1e-30)[..., None]
    out = out.flatten(1, 2).to(s["q"].dtype)
    return (out, (m.squeeze(-2) + total.log()).flatten(1)) if c["lse"] else out


# ---------------------------------------------------------------------------------------------- work

def _sizes(case):
    """Entries of all streams, queries, blocks a query selects, blocks of all streams, as the mean lengths give them."""
    mean = 1.0 - 0.5 * case["ragged"] * (1.0 - 1.0 / case["n_streams"])
    kv = max(1.0, case["kv_len"] * mean)
    q = min(max(1.0, min(case["q_len"], case["kv_len"]) * mean), kv)
    seen = (kv - q / 2 if case["where"] == "tail" else 0.75 * kv) / case["block"]
    return case["n_streams"] * kv, case["n_streams"] * q, max(1.0, min(case["n_select"], seen)), case["n_streams"] * max(1.0, kv / case["block"])


def work(case):
    kind, d, hk = case["kind"], case["head_dim"], case["kv_heads"]
    elem = 4 if case["dtype"] == "f32" else 2
    if kind == "write":
        row = (case["q_heads"] + 2 * hk) * d
        return {"bytes": case["n_tok"] * (2 * row * elem + 8), "flops": case["n_tok"] * 7 * row}
    if kind == "turn":
        row = 2 * case["layers"] * hk * d
        return {"bytes": case["n_rows"] * (2 * row * elem + 12), "flops": case["n_rows"] * 1.5 * row}
    entries, queries, kept, blocks = _sizes(case)
    if kind == "bounds":
        if case["new"]:
            entries = min(entries, case["n_streams"] * (case["new"] + case["block"] / 2))
        return {"bytes": entries * hk * (d * elem + 2 * d / case["block"]), "flops": entries * hk * d * 2}
    if kind == "select":
        return {"bytes": blocks * hk * (2 * d + 1) + queries * (case["q_heads"] * d * elem + 4 * hk * case["n_select"]),
                "flops": queries * case["q_heads"] * blocks / case["n_streams"] * 4 * d}
    read = min(entries, queries * kept * case["block"])
    return {"bytes": read * hk * 2 * d * elem + queries * (case["q_heads"] * (2 * d * elem + (4 if case["lse"] else 0)) + 4 * hk * case["n_select"]),
            "flops": queries * kept * case["block"] * case["q_heads"] * 4 * d}


# ---------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    """What a pass returns, from the definitions in 64 bits, on inputs of the same seed."""
    if case["kind"] in ("bounds", "select"):
        return None                                # whole numbers
    s = prepare(case, seed)
    return {"write": _exact_write, "turn": _exact_turn, "attn": _exact_attn}[case["kind"]](case, s)


def _exact_turned(x, pos, c, s, factor):
    """Pairs of x [rows][heads][d] as complex numbers, turned by their angles."""
    r = c["rotary"]
    axis = _axis_of_pair(c["axes"], r // 2)
    p = pos.double()[:, None].expand(-1, r // 2) if axis is None else torch.stack([pos[:, a].double() for a in axis], 1)
    turn = torch.polar(torch.full_like(p, factor), p * s["inv_freq"].double())[:, None]
    x = x.double().clone()
    if c["style"] == "half":
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn
        x[..., :r // 2], x[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :r].unflatten(-1, (-1, 2)).contiguous()) * turn
        x[..., :r] = torch.view_as_real(z).flatten(-2)
    return x


def _exact_write(c, s):
    n, d = c["n_tok"], c["head_dim"]

    def normed(x, weight):
        x = x.reshape(n, -1, d).double()
        if weight is None:
            return x
        return x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + EPS) * weight.double()

    q = _exact_turned(normed(s["q"], s["q_weight"]), s["pos"], c, s, s["amplitude"])
    k, v = s["k_cache"].double(), s["v_cache"].double()
    k[s["slot"].long()] = _exact_turned(normed(s["k"], s["k_weight"]), s["pos"], c, s, s["amplitude"])
    v[s["slot"].long()] = s["v"].reshape(n, -1, d).double()
    return q, k, v


def _exact_turn(c, s):
    k, v = s["k_pool"].double(), s["v_pool"].double()
    src, dst = s["src"].long(), s["dst"].long()
    for layer in range(c["layers"]):
        k[layer, dst] = _exact_turned(s["k_pool"][layer, src], s["delta"], c, s, 1.0)
        v[layer, dst] = s["v_pool"][layer, src].double()
    return k, v


def _exact_attn(c, s):
    """Kv head by kv head, a few queries at a time."""
    size, hk, hq, d, n_q = c["block"], c["kv_heads"], c["q_heads"], c["head_dim"], s["n_q"]
    group = hq // hk
    out = torch.zeros((n_q, hq, d), dtype=torch.float64, device=DEV)
    stat = torch.zeros((n_q, hq), dtype=torch.float64, device=DEV)
    step = max(1, (1 << 22) // (c["n_select"] * size))
    for g in range(hk):
        for t0 in range(0, n_q, step):
            t = slice(t0, min(n_q, t0 + step))
            which = s["stream"][t]
            blocks = s["selected"][t, g].long()
            j = (blocks[:, :, None] * size + torch.arange(size, device=DEV)).reshape(blocks.shape[0], -1)
            off = (blocks < 0).repeat_interleave(size, 1) | (j > s["q_pos"][t].long()[:, None]) | (j >= s["kv_len"][which].long()[:, None])
            j = j.masked_fill(off, 0)
            slot = s["table"][which[:, None], j // 16].long() * 16 + j % 16
            x = torch.einsum("tgd,ted->tge", s["q"][t, g * group:(g + 1) * group].double(), s["k_cache"][slot, g].double()) / math.sqrt(d)
            x = x.masked_fill(off[:, None], -math.inf)
            lse = torch.logsumexp(x, -1)
            weight = torch.where(torch.isinf(lse)[..., None], 0.0, torch.exp(x - lse[..., None]))
            stat[t, g * group:(g + 1) * group] = lse
            out[t, g * group:(g + 1) * group] = torch.einsum("tge,ted->tgd", weight, s["v_cache"][slot, g].double())
    return (out, stat) if c["lse"] else out
