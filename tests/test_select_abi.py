"""Refusals of the operators of long windows: decided on the host, before anything is queued (no device is needed)."""
import pytest
import torch

from paper_2604_06036_amd import binding as cs

A = 1 << 20         # an aligned address that no refused call looks at
WRITE = dict(q=A, q_out=A, k=A, v=A, qw=A, kw=A, slot=A, pos=A, axis=A, freq=A, kc=A, vc=A, n=3, hq=4, hkv=2, d=64, r=32, sq=512, sk=512, sv=512, ss=128, sh=64,
             eps=1e-6, amp=1.0, style=0, dt=cs.CS_BF16, stream=None)
MOVE = dict(kc=A, vc=A, src=A, dst=A, delta=A, axis=None, freq=A, n=3, layers=2, hkv=2, d=64, r=32, sl=4096, ss=128, sh=64, style=0, dt=cs.CS_BF16, stream=None)
BOUNDS = dict(kc=A, since=None, kv=A, bt=A, mb=8, bs=16, sel=64, b=A, sc=A, s=2, hkv=2, d=64, ss=128, sh=64, dt=cs.CS_BF16, stream=None)
SELECT = dict(q=A, b=A, sc=A, cu=A, pos=A, kv=A, mb=8, sel=64, want=4, first=1, last=1, out=A, n=3, s=2, hq=4, hkv=2, d=64, dt=cs.CS_BF16, ws=A, wsb=1 << 40, stream=None)
ATTN = dict(q=A, kc=A, vc=A, cu=A, pos=A, kv=A, bt=A, mb=8, bs=16, listed=A, sel=64, want=4, out=A, lse=None, n=3, s=2, hq=4, hkv=2, d=64, ss=128, sh=64, scale=0.1,
            dt=cs.CS_BF16, ws=A, wsb=1 << 40, stream=None)
I, U, W = cs.CS_EINVAL, cs.CS_EUNSUPPORTED, cs.CS_EWORKSPACE
NAN, INF = float("nan"), float("inf")

REFUSED = [
    ("cs_norm_rope_refresh_scatter", WRITE, I, [
        dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(slot=None), dict(kc=None), dict(vc=None), dict(freq=None), dict(n=-1), dict(hq=-1), dict(hkv=-1),
        dict(hq=0, hkv=0), dict(d=0), dict(r=-16), dict(r=80), dict(sq=-8), dict(sq=248), dict(sk=120), dict(sv=120), dict(ss=-32), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN),
        dict(eps=INF), dict(eps=1e-31), dict(amp=NAN), dict(amp=INF)]),
    ("cs_norm_rope_refresh_scatter", WRITE, U, [
        dict(d=72), dict(d=272, sq=2048, sk=2048, sv=2048), dict(r=24), dict(r=8), dict(dt=cs.CS_KV4), dict(dt=7), dict(style=2), dict(sq=516), dict(sk=516), dict(sv=516), dict(ss=132),
        dict(sh=68), dict(q=A + 8), dict(q_out=A + 2), dict(k=A + 4), dict(v=A + 8), dict(qw=A + 4), dict(kw=A + 8), dict(kc=A + 8), dict(vc=A + 1), dict(hq=70000, sq=70000 * 64),
        dict(hkv=33000, sk=33000 * 64, sv=33000 * 64), dict(n=1 << 40)]),
    ("cs_kv_rerotate_freqs", MOVE, I, [dict(kc=None), dict(vc=None), dict(src=None), dict(delta=None), dict(freq=None), dict(n=-1), dict(layers=-1), dict(hkv=0), dict(d=0), dict(r=0), dict(r=80),
                                       dict(r=-16), dict(sl=-1)]),
    ("cs_kv_rerotate_freqs", MOVE, U, [dict(d=72), dict(d=272), dict(r=24), dict(r=40), dict(style=5), dict(dt=cs.CS_KV4), dict(sl=33), dict(ss=132), dict(sh=4), dict(kc=A + 4), dict(vc=A + 4),
                                       dict(hkv=65536), dict(n=1 << 40)]),
    ("cs_key_bounds", BOUNDS, I, [dict(kc=None), dict(kv=None), dict(bt=None), dict(b=None), dict(sc=None), dict(mb=0), dict(sel=0), dict(s=-1), dict(hkv=0), dict(ss=-8), dict(sh=-8)]),
    ("cs_key_bounds", BOUNDS, U, [dict(sel=8), dict(sel=40), dict(sel=144), dict(bs=32), dict(d=32), dict(d=96), dict(d=256), dict(dt=cs.CS_KV4), dict(ss=132), dict(sh=4), dict(kc=A + 8),
                                  dict(b=A + 8), dict(hkv=65536), dict(mb=1 << 27)]),
    ("cs_select_blocks", SELECT, I, [dict(q=None), dict(b=None), dict(sc=None), dict(cu=None), dict(pos=None), dict(kv=None), dict(out=None), dict(mb=0), dict(sel=0), dict(want=0), dict(first=-1),
                                     dict(last=-1), dict(first=3, last=2), dict(first=1 << 30, last=(1 << 30) + 1), dict(n=-1), dict(s=-1), dict(hq=5), dict(hq=0), dict(hkv=0)]),
    ("cs_select_blocks", SELECT, U, [dict(sel=8), dict(sel=144), dict(want=257), dict(d=32), dict(d=256), dict(hq=34), dict(dt=cs.CS_KV4), dict(q=A + 8), dict(b=A + 8), dict(n=1 << 26),
                                     dict(mb=1 << 27), dict(mb=4 * 32768 + 1), dict(hkv=65536, hq=65536)]),
    ("cs_selected_attn", ATTN, I, [dict(q=None), dict(kc=None), dict(vc=None), dict(cu=None), dict(pos=None), dict(kv=None), dict(bt=None), dict(listed=None), dict(out=None), dict(mb=0),
                                   dict(sel=0), dict(want=0), dict(n=-1), dict(s=-1), dict(hq=5), dict(hq=0), dict(hkv=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF),
                                   dict(ss=-8)]),
    ("cs_selected_attn", ATTN, U, [dict(sel=8), dict(sel=144), dict(want=257), dict(d=32), dict(d=256), dict(bs=32), dict(hq=34), dict(dt=cs.CS_KV4), dict(ss=132), dict(sh=4), dict(q=A + 8),
                                   dict(out=A + 8), dict(kc=A + 8), dict(vc=A + 8), dict(n=1 << 26), dict(mb=1 << 27), dict(hkv=65536, hq=65536)]),
]


@pytest.mark.parametrize("fn,good,code,change", [(fn, good, code, ch) for fn, good, code, changes in REFUSED for ch in changes])
def test_refused_before_anything_is_queued(fn, good, code, change):
    assert set(change) <= set(good)
    args = dict(good, **change)
    assert getattr(cs.lib(), fn)(*args.values()) == code


@pytest.mark.parametrize("fn,good,empty", [("cs_norm_rope_refresh_scatter", WRITE, dict(n=0)), ("cs_kv_rerotate_freqs", MOVE, dict(n=0)), ("cs_kv_rerotate_freqs", MOVE, dict(layers=0)),
                                           ("cs_key_bounds", BOUNDS, dict(s=0)), ("cs_select_blocks", SELECT, dict(n=0)), ("cs_select_blocks", SELECT, dict(s=0)),
                                           ("cs_selected_attn", ATTN, dict(n=0)), ("cs_selected_attn", ATTN, dict(s=0))])
def test_nothing_to_do_is_no_error(fn, good, empty):
    assert getattr(cs.lib(), fn)(*dict(good, **empty).values()) == cs.CS_OK


def z(n, dt=torch.int32):
    return torch.zeros((n,), dtype=dt)


BF, I8, U8, F = torch.bfloat16, torch.int8, torch.uint8, torch.float32
P_WRITE = dict(q=z(768, BF), q_out=z(768, BF), k=z(384, BF), v=z(384, BF), qw=z(64, BF), kw=z(64, BF), slot=z(3), pos=z(3), axis=None, freq=z(16, F), kc=z(4096, BF), vc=z(4096, BF), n=3,
               hq=4, hkv=2, d=64, r=32, sq=256, sk=128, sv=128, ss=128, sh=64, eps=1e-6, amp=1.0, style=0, dt=cs.CS_BF16)
P_MOVE = dict(kc=z(8192, BF), vc=z(8192, BF), src=z(3), dst=z(3), delta=z(3), axis=None, freq=z(16, F), n=3, layers=2, hkv=2, d=64, r=32, sl=4096, ss=128, sh=64, style=0, dt=cs.CS_BF16)
P_BOUNDS = dict(kc=z(8192, BF), since=None, kv=z(2), bt=z(16), mb=8, bs=16, sel=64, b=z(2 * 2 * 2 * 128, I8), sc=z(8, U8), s=2, hkv=2, d=64, ss=128, sh=64, dt=cs.CS_BF16)
P_SELECT = dict(q=z(768, BF), b=z(2 * 2 * 2 * 128, I8), sc=z(8, U8), cu=z(3), pos=z(3), kv=z(2), mb=8, sel=64, want=4, first=1, last=1, out=z(24), n=3, s=2, hq=4, hkv=2, d=64, dt=cs.CS_BF16)
P_ATTN = dict(q=z(768, BF), kc=z(8192, BF), vc=z(8192, BF), cu=z(3), pos=z(3), kv=z(2), bt=z(16), mb=8, bs=16, listed=z(24), sel=64, want=4, out=z(768, BF), lse=z(12, F), n=3, s=2, hq=4, hkv=2,
              d=64, ss=128, sh=64, scale=0.1, dt=cs.CS_BF16)

PYTHON = [
    ("cs_norm_rope_refresh_scatter", P_WRITE, [
        ("slot", z(2)), ("slot", z(3, torch.int64)), ("pos", z(2)), ("pos", z(6)[::2]), ("axis", z(15, U8)), ("axis", z(16)), ("axis", z(32, U8)[::2]), ("freq", z(16, torch.float64)),
        ("freq", z(15, F)), ("freq", z(32, F)[::2]), ("qw", z(64, F)), ("kw", z(63, BF)), ("kw", z(128, BF)[::2]), ("q", z(768, F)), ("q", z(700, BF)), ("k", z(380, BF)), ("v", z(384, F)),
        ("q_out", z(700, BF)), ("q_out", z(1536, BF)[::2]), ("kc", z(4096, F)), ("vc", z(4096, torch.float16))]),
    ("cs_kv_rerotate_freqs", P_MOVE, [("src", z(2)), ("src", z(3, torch.int64)), ("dst", z(2)), ("delta", z(2)), ("delta", z(3, F)), ("axis", z(15, U8)), ("axis", z(16, torch.int64)),
                                      ("freq", z(16, torch.float64)), ("freq", z(8, F))]),
    ("cs_key_bounds", P_BOUNDS, [("since", z(1)), ("since", z(2, torch.int64)), ("kv", z(1)), ("kv", z(2, torch.int64)), ("bt", z(15)), ("bt", z(16, torch.int64)), ("bt", z(32)[::2]),
                                 ("b", z(1023, I8)), ("b", z(1024, U8)), ("sc", z(7, U8)), ("sc", z(8, I8))]),
    ("cs_select_blocks", P_SELECT, [("q", z(700, BF)), ("q", z(768, F)), ("q", z(1536, BF)[::2]), ("b", z(1023, I8)), ("sc", z(7, U8)), ("cu", z(2)), ("cu", z(3, torch.int64)), ("pos", z(2)),
                                    ("pos", z(3, torch.int64)), ("kv", z(1)), ("out", z(23)), ("out", z(24, torch.int64))]),
    ("cs_selected_attn", P_ATTN, [("q", z(700, BF)), ("q", z(768, F)), ("kc", z(8192, F)), ("vc", z(8192, torch.float16)), ("cu", z(2)), ("pos", z(2)), ("kv", z(1)), ("bt", z(15)),
                                  ("bt", z(16, torch.int64)), ("listed", z(23)), ("listed", z(24, torch.int64)), ("out", z(700, BF)), ("out", z(768, F)), ("lse", z(11, F)), ("lse", z(12, BF))]),
]


@pytest.mark.parametrize("fn,good,name,value", [(fn, good, name, value) for fn, good, changes in PYTHON for name, value in changes])
def test_tensors_that_do_not_hold_what_the_call_reads_are_refused(fn, good, name, value):
    with pytest.raises(ValueError, match=fn):
        getattr(cs, fn)(*dict(good, **{name: value}).values())


@pytest.mark.parametrize("fn,good", [(fn, good) for fn, good, _ in PYTHON])
def test_tensors_on_the_host_are_refused(fn, good):
    with pytest.raises(ValueError, match="device tensor"):
        getattr(cs, fn)(*good.values())


def test_workspaces_that_are_smaller_than_said():
    for fn, good in (("cs_select_blocks", P_SELECT), ("cs_selected_attn", P_ATTN)):
        with pytest.raises(ValueError, match="workspace"):
            getattr(cs, fn)(*good.values(), z(8, U8), 16)
