"""Refusals of the 4-bit cache calls: decided on the host, before anything is queued (no device is needed)."""
import ctypes

import pytest

from paper_2604_06036_amd import binding as cs

A = 1 << 20         # an aligned address that no refused call looks at
ROPE = dict(q=A, q_out=A, k=A, v=A, slot=A, pos=A, axis=A, kc=A, vc=A, ks=A, vs=A, n=3, hq=4, hkv=2, d=64, sq=512, sk=512, sv=512, ss=128, sh=64,
            base=1e6, style=0, dt=cs.CS_BF16, cdt=cs.CS_KV4, stream=None)
GATHER = dict(kc=A, ks=A, vc=A, vs=A, slot=A, n=3, layers=2, hkv=2, d=64, sl=4096, ss=128, sh=64, ko=A, vo=A, dt=cs.CS_BF16, stream=None)
MOVE = dict(kc=A, ks=A, vc=A, vs=A, src=A, dst=A, delta=A, axis=None, n=3, layers=2, hkv=2, d=64, sl=4096, ss=128, sh=64, base=1e6, style=0, stream=None)
ATTN = dict(q=A, kc=A, ks=A, vc=A, vs=A, cu=A, pos=A, kv=A, bt=A, mb=4, bs=16, out=A, lse=None, n=3, s=1, hq=4, hkv=2, d=64, ss=128, sh=64, scale=0.1,
            dt=cs.CS_BF16, ws=A, wsb=1 << 40, stream=None)
WEIGHTS = dict(q=A, lse=None, kc=A, ks=A, cu=A, pos=A, kv=A, bt=A, mb=4, bs=16, wi=A, wo=A, decay=1.0, n=3, s=1, hq=4, hkv=2, d=64, ss=128, sh=64, scale=0.1,
               dt=cs.CS_BF16, cdt=cs.CS_KV4, ws=A, wsb=1 << 40, stream=None)
EVICT = dict(w=A, kv=A, bo=A, mbo=8, bn=A, mbn=4, s=2, budget=64, first=1, last=1, ren=1, kept=A, src=A, dst=A, delta=A, kvn=A + 4096, wn=None, stream=None)
I, U, W = cs.CS_EINVAL, cs.CS_EUNSUPPORTED, cs.CS_EWORKSPACE
NAN, INF = float("nan"), float("inf")

REFUSED = [
    ("cs_rope_refresh_scatter", ROPE, I, [dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(slot=None), dict(kc=None), dict(vc=None), dict(ks=None),
                                          dict(vs=None), dict(pos=None), dict(n=-1), dict(hq=-1), dict(hkv=-1), dict(hq=0, hkv=0), dict(d=0), dict(sq=-8),
                                          dict(sq=248), dict(sk=120), dict(sv=120), dict(ss=-32), dict(base=0.0), dict(base=-1.0), dict(base=NAN), dict(base=INF)]),
    ("cs_rope_refresh_scatter", ROPE, U, [dict(d=80), dict(d=96), dict(d=320), dict(d=72, cdt=cs.CS_BF16), dict(dt=3), dict(cdt=cs.CS_F32), dict(cdt=7), dict(style=2),
                                          dict(sq=516), dict(sk=516), dict(ss=136), dict(sh=48), dict(q=A + 8), dict(q_out=A + 2), dict(k=A + 4), dict(kc=A + 8), dict(vc=A + 1),
                                          dict(hq=70000, sq=70000 * 64)]),
    ("cs_kv4_gather", GATHER, I, [dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None), dict(slot=None), dict(ko=None, vo=None), dict(n=-1), dict(layers=-1), dict(hkv=0),
                                  dict(d=0), dict(sl=-32)]),
    ("cs_kv4_gather", GATHER, U, [dict(d=96), dict(d=320), dict(dt=cs.CS_KV4), dict(sl=16), dict(ss=100), dict(sh=16), dict(ko=A + 8), dict(vo=A + 4), dict(kc=A + 8)]),
    ("cs_kv4_rerotate", MOVE, I, [dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None), dict(src=None), dict(delta=None), dict(n=-1), dict(layers=-1), dict(hkv=0), dict(base=0.0),
                                  dict(base=NAN), dict(sl=-1)]),
    ("cs_kv4_rerotate", MOVE, U, [dict(d=32), dict(d=288), dict(style=5), dict(sl=33), dict(ss=48), dict(sh=8), dict(kc=A + 4), dict(vc=A + 4)]),
    ("cs_kv4_window_attn", ATTN, I, [dict(q=None), dict(kc=None), dict(ks=None), dict(vc=None), dict(vs=None), dict(cu=None), dict(pos=None), dict(kv=None), dict(bt=None),
                                     dict(out=None), dict(mb=0), dict(mb=-1), dict(n=-1), dict(s=-1), dict(hq=5), dict(hkv=0), dict(hq=0), dict(scale=0.0), dict(scale=-1.0),
                                     dict(scale=NAN), dict(scale=INF), dict(ss=-32)]),
    ("cs_kv4_window_attn", ATTN, U, [dict(d=32), dict(d=96), dict(d=256), dict(bs=32), dict(hq=34), dict(dt=cs.CS_KV4), dict(ss=40), dict(sh=8), dict(q=A + 8), dict(out=A + 8),
                                     dict(kc=A + 8), dict(vc=A + 8), dict(n=1 << 26), dict(ss=1 << 26), dict(hkv=70000, hq=70000), dict(mb=1 << 27)]),
    ("cs_attn_weights", WEIGHTS, I, [dict(q=None), dict(kc=None), dict(ks=None), dict(cu=None), dict(pos=None), dict(kv=None), dict(bt=None), dict(wo=None), dict(mb=0), dict(n=-1),
                                     dict(s=-1), dict(hq=5), dict(scale=0.0), dict(scale=NAN), dict(decay=-0.1), dict(decay=1.1), dict(decay=NAN)]),
    ("cs_attn_weights", WEIGHTS, U, [dict(d=32), dict(bs=8), dict(hq=34), dict(dt=cs.CS_KV4), dict(cdt=cs.CS_F32), dict(cdt=5), dict(ss=40), dict(ss=132, cdt=cs.CS_BF16), dict(q=A + 8),
                                     dict(kc=A + 8), dict(mb=1 << 27), dict(n=1 << 31), dict(n=1 << 28, hq=2)]),
    ("cs_attn_weights", WEIGHTS, W, [dict(ws=None), dict(ws=A + 8), dict(wsb=16)]),
    ("cs_plan_evict", EVICT, I, [dict(w=None), dict(kv=None), dict(bo=None), dict(bn=None), dict(kept=None), dict(src=None), dict(dst=None), dict(delta=None), dict(kvn=None), dict(s=-1),
                                 dict(budget=0), dict(first=-1), dict(last=-1), dict(mbo=0), dict(mbn=0), dict(budget=65), dict(mbn=3)]),
    ("cs_plan_evict", EVICT, U, [dict(mbo=1 << 27), dict(mbn=1 << 27), dict(budget=(1 << 30) + 1, mbn=8)]),
]


@pytest.mark.parametrize("fn,good,code,change", [(fn, good, code, ch) for fn, good, code, changes in REFUSED for ch in changes])
def test_refused_before_anything_is_queued(fn, good, code, change):
    assert set(change) <= set(good)
    args = dict(good, **change)
    assert getattr(cs.lib(), fn)(*args.values()) == code


@pytest.mark.parametrize("fn,good,empty", [("cs_rope_refresh_scatter", ROPE, dict(n=0)), ("cs_kv4_gather", GATHER, dict(n=0)), ("cs_kv4_gather", GATHER, dict(layers=0)),
                                           ("cs_kv4_rerotate", MOVE, dict(n=0)), ("cs_kv4_rerotate", MOVE, dict(layers=0)), ("cs_kv4_window_attn", ATTN, dict(n=0)),
                                           ("cs_kv4_window_attn", ATTN, dict(s=0)), ("cs_attn_weights", WEIGHTS, dict(s=0)), ("cs_plan_evict", EVICT, dict(s=0))])
def test_nothing_to_do_is_no_error(fn, good, empty):
    args = dict(good, **empty)
    assert getattr(cs.lib(), fn)(*(None if v == A else v for v in args.values())) == cs.CS_OK


def test_attention_workspace_too_small_is_refused():
    need = cs.cs_kv4_window_attn_workspace(1, 1, 28, 4, 128, 2048)
    if need == 0:
        pytest.skip("no shape of one token takes a workspace")
    args = dict(ATTN, n=1, hq=28, hkv=4, d=128, mb=2048, ss=128, sh=1 << 22)
    for change in (dict(ws=None), dict(wsb=need - 1), dict(ws=A + 8)):
        assert cs.lib().cs_kv4_window_attn(*dict(args, **change).values()) == cs.CS_EWORKSPACE


def test_workspaces_of_empty_calls_are_empty():
    assert cs.cs_attn_weights_workspace(0, 4, 8, 2, 64, 8) == 0 == cs.cs_attn_weights_workspace(4, 0, 8, 2, 64, 8)
    assert cs.cs_kv4_window_attn_workspace(0, 4, 8, 2, 64, 8) == 0
    assert cs.cs_attn_weights_workspace(4, 2, 8, 2, 64, 8) >= 2 * 2 * 128 * 4


def test_binding_refuses_tensors_that_are_too_short():
    torch = pytest.importorskip("torch")
    z = lambda n, dt=torch.int32: torch.zeros((n,), dtype=dt)
    with pytest.raises(ValueError, match="slot"):
        cs.cs_kv4_gather(z(64, torch.uint8), z(4, torch.uint8), None, None, z(2), 3, 1, 1, 64, 0, 64, 64, z(192, torch.bfloat16), None, cs.CS_BF16)
    with pytest.raises(ValueError, match="k_out"):
        cs.cs_kv4_gather(z(64, torch.uint8), z(4, torch.uint8), None, None, z(3), 3, 1, 1, 64, 0, 64, 64, z(191, torch.bfloat16), None, cs.CS_BF16)
    with pytest.raises(ValueError, match="delta"):
        cs.cs_kv4_rerotate(None, None, None, None, z(3), z(3), z(8), z(32, torch.uint8), 3, 1, 1, 64, 0, 64, 64, 1e6, 0)
    with pytest.raises(ValueError, match="q holds fewer"):
        cs.cs_rope_refresh_scatter(z(2 * 128 + 63, torch.bfloat16), None, None, None, None, z(3), None, None, None, None, None, 3, 1, 0, 64, 128, 0, 0, 0, 0, 1e6, 0,
                                   cs.CS_BF16, cs.CS_KV4)
    with pytest.raises(ValueError, match="lse"):
        cs.cs_kv4_window_attn(z(256), None, None, None, None, z(2), z(2), z(1), z(4), 4, 16, z(256), z(1), 2, 1, 2, 1, 64, 64, 64, 0.1, cs.CS_F32)
    with pytest.raises(ValueError, match="weight_out"):
        cs.cs_attn_weights(z(256), None, None, None, z(2), z(2), z(1), z(4), 4, 16, None, z(63), 1.0, 2, 1, 2, 1, 64, 64, 64, 0.1, cs.CS_F32, cs.CS_F32)
    with pytest.raises(ValueError, match="kept"):
        cs.cs_plan_evict(z(64), z(1), z(4), 4, z(4), 4, 1, 8, 0, 0, True, z(7), z(8), z(8), z(8), z(1), None)
    with pytest.raises(ValueError, match="device tensor"):
        cs.cs_plan_evict(z(64), z(1), z(4), 4, z(4), 4, 1, 8, 0, 0, True, z(8), z(8), z(8), z(8), z(1), None)


@pytest.mark.parametrize("fn,good,code,change", [
    ("cs_rope_refresh_scatter", ROPE, U, dict(n=1 << 30)), ("cs_rope_refresh_scatter", ROPE, U, dict(n=1 << 62)),
    ("cs_kv4_gather", GATHER, U, dict(n=1 << 27)), ("cs_kv4_gather", GATHER, U, dict(n=1 << 62)), ("cs_kv4_gather", GATHER, U, dict(n=1 << 16, layers=1 << 16)),
    ("cs_kv4_rerotate", MOVE, U, dict(n=1 << 31)), ("cs_kv4_rerotate", MOVE, U, dict(n=1 << 62)),
    ("cs_attn_weights", WEIGHTS, U, dict(n=1 << 24)), ("cs_attn_weights", WEIGHTS, U, dict(mb=1 << 24, s=32)), ("cs_attn_weights", WEIGHTS, U, dict(mb=(1 << 27) - 1)),
    ("cs_plan_evict", EVICT, U, dict(s=1 << 22)), ("cs_plan_evict", EVICT, I, dict(kvn=A, kv=A)), ("cs_plan_evict", EVICT, I, dict(w=A, wn=A))])
def test_more_than_a_launch_holds_and_outputs_over_inputs(fn, good, code, change):
    assert getattr(cs.lib(), fn)(*dict(good, **change).values()) == code


@pytest.mark.parametrize("fn,good,code,change", [
    ("cs_rope_refresh_scatter", ROPE, U, dict(hq=65536, sq=65536 * 64)), ("cs_rope_refresh_scatter", ROPE, U, dict(n=100000, hq=65536, sq=65536 * 64)),
    ("cs_rope_refresh_scatter", ROPE, U, dict(hkv=32768, sk=32768 * 64, sv=32768 * 64)),
    ("cs_kv4_rerotate", MOVE, U, dict(n=(1 << 31) + 1, hkv=2)), ("cs_kv4_rerotate", MOVE, U, dict(n=1 << 24, hkv=256)),
    ("cs_kv4_window_attn", ATTN, U, dict(n=(1 << 26) - 1, hq=64, hkv=64)),                 # 2^25 workgroups: row tiles of 128 rows
    ("cs_kv4_window_attn", ATTN, U, dict(n=(1 << 26) - 1, s=1 << 26, hq=16, hkv=2)),       # row tiles of 16 rows
    ("cs_attn_weights", WEIGHTS, U, dict(n=1, s=1 << 20, hq=32, hkv=32, mb=16)),           # 2^25 workgroups
    ("cs_attn_weights", WEIGHTS, U, dict(n=1 << 26, hq=32, hkv=2, lse=A)), ("cs_attn_weights", WEIGHTS, U, dict(mb=(1 << 27) - 256, lse=A)),
    ("cs_attn_weights", WEIGHTS, U, dict(d=96)), ("cs_attn_weights", WEIGHTS, U, dict(sh=40)), ("cs_attn_weights", WEIGHTS, U, dict(ss=66, sh=2, dt=cs.CS_F32, cdt=cs.CS_F32)),
    ("cs_kv4_window_attn", ATTN, U, dict(mb=(1 << 27) - 64)), ("cs_plan_evict", EVICT, U, dict(mbo=(1 << 27) - 1024)), ("cs_plan_evict", EVICT, U, dict(mbn=(1 << 27) - 1024)),
    ("cs_attn_weights", WEIGHTS, I, dict(hkv=0)), ("cs_attn_weights", WEIGHTS, I, dict(scale=INF)), ("cs_attn_weights", WEIGHTS, I, dict(ss=-32))])
def test_limits_are_those_of_the_header(fn, good, code, change):
    assert getattr(cs.lib(), fn)(*dict(good, **change).values()) == code
