"""Rotary positions without a device: frequencies against the oracle and closed forms, and what the
calls refuse before anything is launched."""
import ctypes
import math

import numpy as np
import pytest

import paper_2604_21335_amd as stc
from oracle import stc_oracle as O

KINDS = dict(none=stc.STC_ROTARY_SCALE_NONE, linear=stc.STC_ROTARY_SCALE_LINEAR,
             base=stc.STC_ROTARY_SCALE_BASE, channels=stc.STC_ROTARY_SCALE_CHANNELS,
             wavelengths=stc.STC_ROTARY_SCALE_WAVELENGTHS)
FAKE = ctypes.c_void_p(0x1000)      # aligned, never dereferenced: calls must fail earlier
ODD = ctypes.c_void_p(0x1004)


# pow and log are within a few units of 2^-53 of the true value; the exponents are at most 2.
@pytest.mark.parametrize("rot", [16, 48, 64, 128])
@pytest.mark.parametrize("base", [1e4, 1e6])
@pytest.mark.parametrize("kind", list(KINDS))
def test_turns_are_the_formulas(rot, base, kind):
    extra = {} if kind == "none" else dict(factor=4.0)
    if kind in ("channels", "wavelengths"):
        extra.update(original_len=8192, slow=1.0, fast=32.0)
    got = stc.stc_rotary_turns(rot, base=base, kind=KINDS[kind], **extra).numpy()
    np.testing.assert_allclose(got, O.rotary_turns(rot, base, kind, **extra), rtol=1e-14, atol=0)


def test_turns_at_the_ends():
    plain = stc.stc_rotary_turns(64).numpy()
    assert plain[0] == 1 / (2 * math.pi)
    slow = stc.stc_rotary_turns(64, kind=stc.STC_ROTARY_SCALE_BASE, factor=8.0).numpy()
    assert slow[0] == plain[0]                        # the fastest pair stays
    np.testing.assert_allclose(slow[-1], plain[-1] / 8, rtol=1e-14)   # the slowest slows by factor
    for kind in (stc.STC_ROTARY_SCALE_CHANNELS, stc.STC_ROTARY_SCALE_WAVELENGTHS):
        t = stc.stc_rotary_turns(128, base=5e5, kind=kind, factor=8.0, original_len=8192, slow=1.0,
                                 fast=4.0).numpy()
        p = stc.stc_rotary_turns(128, base=5e5).numpy()
        np.testing.assert_allclose(t[0], p[0], rtol=1e-15)
        np.testing.assert_allclose(t[-1], p[-1] / 8, rtol=1e-15)
        r = t / p
        assert ((r[1:] <= r[:-1] + 1e-15).all() and ((r > 0.126) & (r < 0.999)).any())


@pytest.mark.parametrize("kw", [
    dict(rot_dim=0), dict(rot_dim=8), dict(rot_dim=24), dict(rot_dim=144), dict(base=1.0),
    dict(base=math.nan), dict(base=math.inf), dict(kind=5), dict(kind=-1),
    dict(kind=1, factor=0.0), dict(kind=2, factor=-1.0), dict(kind=1, factor=math.nan),
    dict(kind=3, factor=2.0, original_len=0, slow=1.0, fast=2.0),
    dict(kind=3, factor=2.0, original_len=64, slow=0.0, fast=2.0),
    dict(kind=4, factor=2.0, original_len=64, slow=2.0, fast=2.0),
    dict(kind=4, factor=2.0, original_len=64, slow=2.0, fast=math.inf)])
def test_turns_refuse(kw):
    kw = dict(dict(rot_dim=64), **kw)
    with pytest.raises(stc.StcError) as e:
        stc.stc_rotary_turns(kw.pop("rot_dim"), **kw)
    assert e.value.status == stc.STC_ERR_SHAPE


@pytest.mark.parametrize("kw", [dict(kind=1, factor=5e-324), dict(kind=2, factor=5e-324),
                                dict(base=1.5, kind=2, factor=1e-302),
                                dict(kind=4, factor=1e-310, original_len=64, slow=1.0, fast=2.0)])
def test_turns_refuse_frequencies_that_are_not_finite(kw):
    s = stc.stc_rotary_scaling_t(kw["kind"], kw.get("original_len", 0), kw.get("base", 1e4), kw["factor"],
                                 kw.get("slow", 0.0), kw.get("fast", 0.0))
    out = (ctypes.c_double * 32)(*[7.0] * 32)
    assert stc.load_library().stc_rotary_turns(64, ctypes.byref(s), out) == stc.STC_ERR_SHAPE
    assert list(out) == [7.0] * 32


def test_turns_refuse_null():
    lib = stc.load_library()
    s = stc.stc_rotary_scaling_t(0, 0, 1e4, 1.0, 0.0, 0.0)
    assert lib.stc_rotary_turns(64, None, (ctypes.c_double * 32)()) == stc.STC_ERR_NULL
    assert lib.stc_rotary_turns(64, ctypes.byref(s), None) == stc.STC_ERR_NULL


def _call(**kw):
    a = dict(B=2, H=3, N=5, D=128, rot=64, layout=0, turns=FAKE, amp=1.0, pos=None, pos0=0, x=FAKE,
             xs=(1920, 128, 384), y=FAKE, ys=(1920, 640, 128))
    a.update(kw)
    s3 = lambda v: None if v is None else (ctypes.c_int64 * 3)(*v)  # noqa: E731
    return stc.load_library().stc_rotary(
        a["B"], a["H"], a["N"], a["D"], a["rot"], a["layout"], a["turns"], a["amp"], a["pos"],
        a["pos0"], a["x"], s3(a["xs"]), a["y"], s3(a["ys"]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(turns=None), "NULL"), (dict(x=None), "NULL"), (dict(y=None), "NULL"), (dict(xs=None), "NULL"),
    (dict(ys=None), "NULL"), (dict(B=0), "SHAPE"), (dict(B=65536), "SHAPE"), (dict(H=0), "SHAPE"),
    (dict(N=0), "SHAPE"), (dict(H=1 << 16, N=1 << 15), "SHAPE"), (dict(D=96), "SHAPE"),
    (dict(D=64, rot=128), "SHAPE"), (dict(rot=0), "SHAPE"), (dict(rot=40), "SHAPE"),
    (dict(layout=2), "SHAPE"), (dict(layout=0x102), "SHAPE"), (dict(layout=-1), "SHAPE"),
    (dict(amp=math.nan), "SHAPE"), (dict(amp=math.inf), "SHAPE"), (dict(pos0=2**31 - 4), "SHAPE"),
    (dict(ys=(1920, 0, 128)), "SHAPE"), (dict(ys=(1920, 640, 64)), "SHAPE"),
    (dict(x=ODD), "ALIGN"), (dict(y=ODD), "ALIGN"), (dict(turns=ODD), "ALIGN"),
    (dict(pos=ctypes.c_void_p(0x1002)), "ALIGN"), (dict(xs=(1920, 128, 388)), "ALIGN"),
    (dict(xs=(-1920, 128, 384)), "ALIGN"), (dict(ys=(1924, 640, 128)), "ALIGN")])
def test_rotary_refuses(kw, status):
    assert _call(**kw) == getattr(stc, "STC_ERR_" + status)


@pytest.mark.parametrize("D,H,N", [(64, 1, (1 << 30) - 63), (128, 1, (1 << 29) - 31), (128, 1 << 15, 1 << 14),
                                   (64, 1 << 10, 1 << 20), (64, 1, 2**31 - 1)])
def test_rotary_refuses_more_than_a_launch_counts(D, H, N):
    """2^32 threads and more, a thread for 16 channels, in workgroups of 256."""
    assert -(-H * N * (D // 16) // 256) * 256 >= 1 << 32
    s = (H * N * D, N * D, D)
    assert _call(B=1, D=D, H=H, N=N, xs=s, y=ctypes.c_void_p(0x100000), ys=s) == stc.STC_ERR_SHAPE


# B, H, N, D = 2, 3, 5, 128
@pytest.mark.parametrize("ys", [(1920, 128, 128), (1920, 128, 256), (640, 128, 384), (1920, 640, 120),
                                (1912, 640, 128), (1920, 632, 128), (1 << 62, 128, 1 << 61)])
def test_rotary_refuses_rows_that_overlap(ys):
    assert _call(y=ctypes.c_void_p(0x100000), ys=ys) == stc.STC_ERR_SHAPE


# B, H, N = 2, 3, 5; in a dimension of one element the stride does not count
@pytest.mark.parametrize("ys", [(1920, 640, 128), (1920, 128, 640), (3840, 128, 384)])
def test_rotary_refuses_another_order_in_place(ys):
    other = ctypes.c_void_p(0x100000)
    assert _call(y=other, ys=ys, amp=math.nan) == stc.STC_ERR_SHAPE     # what is refused anyway
    assert _call(ys=ys) == stc.STC_ERR_SHAPE
    assert _call(ys=ys, D=64) == stc.STC_ERR_SHAPE


def _append(shape=None, **kw):
    a = dict(q=FAKE, qs=1024, k=FAKE, ks=256, v=FAKE, vs=256, qo=ctypes.c_void_p(0x2000), Kt=FAKE,
             Vt=FAKE, n=FAKE, n_out=None, cap=16, rot=64, layout=0, turns=FAKE, amp=1.0, pos=None,
             pos0=0, status=None)
    a.update(kw)
    s = stc.make_shape(**dict(dict(B=2, Hq=8, Hkv=2, D=128, N=100, G=8, v_cap_groups=800), **(shape or {})))
    return stc.load_library().stc_rotary_append(
        ctypes.byref(s), a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["qo"], a["Kt"], a["Vt"],
        a["n"], a["n_out"], a["cap"], a["rot"], a["layout"], a["turns"], a["amp"], a["pos"], a["pos0"],
        a["status"], None)


@pytest.mark.parametrize("kw,status", [
    *[({p: None}, "NULL") for p in ("q", "k", "v", "qo", "Kt", "Vt", "n", "turns")],
    *[({p: ODD}, "ALIGN") for p in ("q", "k", "v", "qo", "Kt", "Vt", "turns")],
    *[({p: ctypes.c_void_p(0x1002)}, "ALIGN") for p in ("n", "n_out", "pos")],
    *[({p: 1028}, "ALIGN") for p in ("qs", "ks", "vs")], (dict(qs=-1024), "ALIGN"),
    (dict(cap=0), "SHAPE"), (dict(rot=8), "SHAPE"), (dict(rot=136), "SHAPE"), (dict(rot=-16), "SHAPE"),
    (dict(layout=0x100), "SHAPE"), (dict(layout=3), "SHAPE"), (dict(amp=math.nan), "SHAPE"),
    (dict(pos0=2**31 - 10), "SHAPE"), (dict(shape=dict(D=96)), "SHAPE"), (dict(shape=dict(Hq=7)), "SHAPE"),
    (dict(qo=FAKE, qs=2048), "SHAPE")])
def test_append_refuses(kw, status):
    assert _append(**kw) == getattr(stc, "STC_ERR_" + status)


def test_a_cache_without_its_own_keys_takes_no_rotary():
    cache = stc.RoutedCache.__new__(stc.RoutedCache)
    cache.n_cap = 0
    with pytest.raises(ValueError):
        cache.build(None, None, rotary=object())
