"""Decode attention over a shared prefix without a device: what the call refuses before anything is
launched, and the workspace it asks for."""
import ctypes

import pytest

import paper_2604_21335_amd as stc

FAKE = ctypes.c_void_p(0x1000)      # aligned, never dereferenced: calls must fail earlier
ODD = ctypes.c_void_p(0x1004)
SHAPE = dict(B=5, Hq=8, Hkv=2, D=128, N=100, G=8, v_cap_groups=800, N_cap=0)


def _call(shape=None, **kw):
    a = dict(q=FAKE, K=FAKE, v=FAKE, mask=FAKE, off=FAKE, idx=None, k=7, Kt=FAKE, Vt=FAKE, n=FAKE,
             cap=16, type=0, out=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    s = stc.make_shape(**dict(SHAPE, **(shape or {})))
    return stc.load_library().stc_decode_attention_shared(
        ctypes.byref(s), a["q"], a["K"], a["v"], a["mask"], a["off"], a["idx"], a["k"], a["Kt"], a["Vt"],
        a["n"], a["cap"], a["type"], a["out"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    *[({p: None}, "NULL") for p in ("q", "K", "v", "mask", "off", "out", "Kt", "Vt", "n")],
    *[({p: ODD}, "ALIGN") for p in ("q", "K", "v", "mask", "off", "idx", "out", "Kt", "Vt")],
    (dict(n=ctypes.c_void_p(0x1002)), "ALIGN"),
    (dict(k=0), "SHAPE"), (dict(k=8), "SHAPE"), (dict(cap=-1), "SHAPE"), (dict(cap=(1 << 30) + 1), "SHAPE"),
    (dict(type=2), "SHAPE"), (dict(type=-1), "SHAPE"), (dict(shape=dict(D=96)), "SHAPE"),
    (dict(shape=dict(Hq=34)), "SHAPE"), (dict(shape=dict(G=3)), "SHAPE"), (dict(shape=dict(B=0)), "SHAPE"),
    (dict(shape=dict(N=0)), "SHAPE"), (dict(shape=dict(v_cap_groups=0)), "SHAPE"),
    (dict(ws=None), "WORKSPACE"), (dict(wsb=16), "WORKSPACE"), (dict(ws=ODD), "WORKSPACE")])
def test_refuses(kw, status):
    assert _call(**kw) == getattr(stc, "STC_ERR_" + status)


def test_null_shape():
    assert stc.load_library().stc_decode_attention_shared(
        None, FAKE, FAKE, FAKE, FAKE, FAKE, None, 1, None, None, None, 0, 0, FAKE, FAKE, 1 << 30,
        None) == stc.STC_ERR_NULL


def test_workspace():
    s = stc.make_shape(**SHAPE)
    assert stc.stc_shared_workspace_bytes(s, 0, 16) == stc.stc_shared_workspace_bytes(s, 8, 16) == 0
    assert stc.stc_shared_workspace_bytes(s, 7, -1) == 0
    assert stc.stc_shared_workspace_bytes(stc.make_shape(**dict(SHAPE, D=80)), 7, 16) == 0
    need = stc.stc_shared_workspace_bytes(s, 7, 16)
    assert need > 0 and _call(wsb=need - 1) == stc.STC_ERR_WORKSPACE
    # every call's numbers of partial results fit what a size_t and a launch can count
    big = stc.make_shape(2047, 512, 32, 128, 1 << 20, 8, 1 << 23)
    assert 0 < stc.stc_shared_workspace_bytes(big, 1 << 16, 1 << 20) < 1 << 40


def test_a_prefix_is_one_element():
    cache = stc.RoutedCache.__new__(stc.RoutedCache)
    cache.B = 2
    with pytest.raises(ValueError):
        stc.SharedPrefix(cache, 4, 16)


def test_a_prefix_is_whole():
    """One with a tail of its own, or that grows while sequences continue it, is refused: its tail would
    not be attended, and new tokens' positions would move."""
    cache = stc.RoutedCache.__new__(stc.RoutedCache)
    cache.B, cache.N, cache.n_tail = 1, 64, 3
    with pytest.raises(ValueError):
        stc.SharedPrefix(cache, 4, 16)
    b = stc.SharedPrefix.__new__(stc.SharedPrefix)
    b.prefix, b.N = cache, 64
    for tail, n in ((3, 64), (0, 67)):
        cache.n_tail, cache.N = tail, n
        with pytest.raises(ValueError):
            b.append(None, None, None)
        with pytest.raises(ValueError):
            b.attend(None)


def test_positions_behind_given_ones_have_to_be_said():
    cache = stc.RoutedCache.__new__(stc.RoutedCache)
    cache.B, cache.N, cache.n_tail, cache.next_pos = 1, 64, 0, None
    b = stc.SharedPrefix.__new__(stc.SharedPrefix)
    b.prefix, b.N, b.pos0, b.rotary = cache, 64, None, stc.Rotary.__new__(stc.Rotary)
    with pytest.raises(ValueError, match="pos0"):
        b.append(None, None, None)
