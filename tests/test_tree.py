"""Drafted tokens without a device: what the calls refuse before anything is launched, the workspace they ask
for, and what the classes refuse."""
import ctypes

import pytest

import paper_2604_21335_amd as stc

FAKE = ctypes.c_void_p(0x10000)     # aligned, never dereferenced: calls must fail earlier
ODD, ODD2 = ctypes.c_void_p(0x10004), ctypes.c_void_p(0x10002)
SHAPE = dict(B=5, Hq=8, Hkv=2, D=128, N=100, G=8, v_cap_groups=800, N_cap=0)
I64 = ctypes.c_int64


def _shape(kw):
    return stc.make_shape(**dict(SHAPE, **(kw or {})))


def _append(shape=None, **kw):
    a = dict(T=3, q=FAKE, qs=(3 * 1024, 1024), k=FAKE, ks=(3 * 256, 256), v=FAKE, vs=(3 * 256, 256),
             qo=ctypes.c_void_p(0x90000), Kt=FAKE, Vt=FAKE, n=FAKE, nd=None, cap=16, tree=None, per=0, rot=64,
             layout=0, turns=FAKE, amp=1.0, pos=None, pos0=0, status=None)
    a.update(kw)
    s = _shape(shape)
    strides = [None if a[x] is None else (I64 * 2)(*a[x]) for x in ("qs", "ks", "vs")]
    return stc.load_library().stc_rotary_append_tree(
        ctypes.byref(s), a["T"], a["q"], strides[0], a["k"], strides[1], a["v"], strides[2], a["qo"], a["Kt"],
        a["Vt"], a["n"], a["nd"], a["cap"], a["tree"], a["per"], a["rot"], a["layout"], a["turns"], a["amp"],
        a["pos"], a["pos0"], a["status"], None)


@pytest.mark.parametrize("kw,status", [
    *[({p: None}, "NULL") for p in ("q", "qs", "k", "ks", "v", "vs", "qo", "Kt", "Vt", "n", "turns")],
    *[({p: ODD}, "ALIGN") for p in ("q", "k", "v", "qo", "Kt", "Vt", "turns", "tree")],
    *[({p: ODD2}, "ALIGN") for p in ("n", "nd", "pos", "status")],
    (dict(qs=(3 * 1024, 1020)), "ALIGN"), (dict(ks=(-8, 256)), "ALIGN"), (dict(vs=(4, 256)), "ALIGN"),
    (dict(T=0), "SHAPE"), (dict(T=65), "SHAPE"), (dict(cap=0), "SHAPE"), (dict(cap=(1 << 30) + 1), "SHAPE"),
    (dict(per=2), "SHAPE"), (dict(per=-1), "SHAPE"), (dict(rot=24), "SHAPE"), (dict(rot=144), "SHAPE"),
    (dict(layout=2), "SHAPE"), (dict(layout=0x100), "SHAPE"), (dict(amp=float("inf")), "SHAPE"),
    (dict(pos0=2**31 - 15), "SHAPE"), (dict(qo=FAKE, qs=(3 * 1024, 2048)), "SHAPE"),
    (dict(qo=FAKE, qs=(4096, 1024)), "SHAPE"), (dict(shape=dict(D=96)), "SHAPE"), (dict(shape=dict(B=0)), "SHAPE")])
def test_append_refuses(kw, status):
    assert _append(**kw) == getattr(stc, "STC_ERR_" + status)


def _attend(shape=None, **kw):
    a = dict(T=3, P=1, q=FAKE, K=FAKE, v=FAKE, mask=FAKE, off=FAKE, idx=None, k=7, Kt=FAKE, Vt=FAKE, n=FAKE,
             nd=None, cap=16, tree=None, per=0, type=0, out=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    s = _shape(shape)
    return stc.load_library().stc_decode_attention_tree(
        ctypes.byref(s), a["T"], a["P"], a["q"], a["K"], a["v"], a["mask"], a["off"], a["idx"], a["k"], a["Kt"],
        a["Vt"], a["n"], a["nd"], a["cap"], a["tree"], a["per"], a["type"], a["out"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    *[({p: None}, "NULL") for p in ("q", "K", "v", "mask", "off", "out", "Kt", "Vt", "n")],
    *[({p: ODD}, "ALIGN") for p in ("q", "K", "v", "mask", "off", "idx", "out", "Kt", "Vt", "tree")],
    *[({p: ODD2}, "ALIGN") for p in ("n", "nd")],
    (dict(T=0), "SHAPE"), (dict(T=65), "SHAPE"), (dict(P=0), "SHAPE"), (dict(P=2), "SHAPE"), (dict(P=6), "SHAPE"),
    (dict(k=0), "SHAPE"), (dict(k=8), "SHAPE"), (dict(cap=0), "SHAPE"), (dict(cap=-1), "SHAPE"),
    (dict(cap=(1 << 30) + 1), "SHAPE"), (dict(per=2), "SHAPE"), (dict(type=2), "SHAPE"),
    (dict(shape=dict(D=96)), "SHAPE"), (dict(shape=dict(Hq=34)), "SHAPE"), (dict(shape=dict(G=3)), "SHAPE"),
    (dict(shape=dict(N=0)), "SHAPE"), (dict(shape=dict(v_cap_groups=0)), "SHAPE"),
    (dict(ws=None), "WORKSPACE"), (dict(wsb=16), "WORKSPACE"), (dict(ws=ODD), "WORKSPACE")])
def test_attention_refuses(kw, status):
    assert _attend(**kw) == getattr(stc, "STC_ERR_" + status)


def test_workspace():
    s = stc.make_shape(**SHAPE)
    w = stc.stc_tree_workspace_bytes
    for bad in ((s, 0, 7, 16), (s, 65, 7, 16), (s, 3, 0, 16), (s, 3, 8, 16), (s, 3, 7, 0), (s, 3, 7, 16, 2),
                (stc.make_shape(**dict(SHAPE, D=80)), 3, 7, 16)):
        assert w(*bad) == 0
    for P in (1, 5):
        need = w(s, 3, 7, 16, n_prefix=P)
        assert need > 0 and _attend(P=P, wsb=need - 1) == stc.STC_ERR_WORKSPACE
    # far prefixes and tails: numbers of partial results fit what a launch counts
    big = stc.make_shape(2047, 512, 32, 128, 1 << 20, 8, 1 << 23)
    for P in (1, 2047):
        assert 0 < w(big, 16, 1 << 16, 1 << 20, n_prefix=P) < 1 << 42


def _ptrs(at):
    return (ctypes.c_void_p * len(at))(*at)


def _tails(call, shape=None, layers=2, **kw):
    size = 5 * 2 * 16 * 128 * 2
    a = dict(T=8, cap=16, K=[0x100000 + i * size for i in range(layers)],
             V=[0x900000 + i * size for i in range(layers)], n=[0x1000 + 32 * i for i in range(layers)],
             out=[0x1000 + 32 * i for i in range(layers)], keep=FAKE, src=FAKE, n_keep=None, status=None,
             count=layers)
    a.update(kw)
    s = _shape(shape)
    p = [None if a[x] is None else _ptrs(a[x]) for x in ("K", "V", "n", "out")]
    lib = stc.load_library()
    if call == "accept":
        return lib.stc_accept_tail(ctypes.byref(s), a["T"], a["count"], *p, a["cap"], a["keep"], None)
    return lib.stc_fork_tail(ctypes.byref(s), a["count"], *p, a["cap"], a["src"], a["n_keep"], a["status"], None)


@pytest.mark.parametrize("call", ["accept", "fork"])
@pytest.mark.parametrize("kw,status", [
    *[({p: None}, "NULL") for p in ("K", "V", "n", "out")],
    (dict(K=[0x100000, 0]), "NULL"), (dict(out=[0, 0x1000]), "NULL"),
    (dict(V=[0x900000, 0xa00008]), "ALIGN"), (dict(n=[0x1002, 0x1020]), "ALIGN"),
    (dict(count=0), "SHAPE"), (dict(count=1025), "SHAPE"), (dict(cap=0), "SHAPE"), (dict(shape=dict(D=96)), "SHAPE"),
    # the same tail twice, as two layers' or as keys and values; tails that overlap
    (dict(K=[0x100000, 0x100000]), "SHAPE"), (dict(V=[0x100000, 0x900000]), "SHAPE"),
    (dict(K=[0x100000, 0x100000 + 16]), "SHAPE"),
    # lengths that another layer's launch writes
    (dict(n=[0x1000, 0x1000], out=[0x1000, 0x1000]), "SHAPE"), (dict(n=[0x1000, 0x1000], out=[0x1000, 0x1020]), "SHAPE"),
    (dict(n=[0x1000, 0x1020], out=[0x1010, 0x1040]), "SHAPE"), (dict(n=[0x1000, 0x1020], out=[0x1020, 0x1040]), "SHAPE"),
    (dict(n=[0x1000, 0x1020], out=[0x1040, 0x1050]), "SHAPE")])
def test_tails_refuse(call, kw, status):
    assert _tails(call, **kw) == getattr(stc, "STC_ERR_" + status)


@pytest.mark.parametrize("call,kw,status", [
    ("accept", dict(keep=None), "NULL"), ("accept", dict(keep=ODD), "ALIGN"), ("accept", dict(T=0), "SHAPE"),
    ("accept", dict(T=65), "SHAPE"), ("fork", dict(src=None), "NULL"), ("fork", dict(src=ODD2), "ALIGN"),
    ("fork", dict(n_keep=ODD2), "ALIGN"), ("fork", dict(status=ODD2), "ALIGN"),
    ("fork", dict(shape=dict(B=4097)), "SHAPE"),
    # the map, or the lengths to keep, where lengths are written
    ("fork", dict(src=ctypes.c_void_p(0x1010)), "SHAPE"), ("fork", dict(n_keep=ctypes.c_void_p(0x1020)), "SHAPE")])
def test_accept_and_fork_refuse(call, kw, status):
    assert _tails(call, **kw) == getattr(stc, "STC_ERR_" + status)


# the sets of kept nodes are read, of all sequences by every layer, while lengths are written
@pytest.mark.parametrize("keep", [0x1000, 0x1010, 0x1020, 0x1030, 0xfe0, 0x1000 - 8])
def test_accept_refuses_kept_sets_where_lengths_are_written(keep):
    assert _tails("accept", keep=ctypes.c_void_p(keep)) == stc.STC_ERR_SHAPE


def test_accept_refuses_kept_sets_where_lengths_of_a_far_layer_are_written():
    n = [0x1000 + 32 * i for i in range(100)]
    at = [0x100000 + 0x10000 * i for i in range(200)]
    for keep in (0x1000 + 32 * 99 + 16, 0x1000 + 32 * 40 - 16):
        assert _tails("accept", layers=100, K=at[:100], V=at[100:], n=[0x10000] * 100, out=n,
                      keep=ctypes.c_void_p(keep)) == stc.STC_ERR_SHAPE


# counts of nodes: written by the one call, where others are read; read by the other, where lengths are written
@pytest.mark.parametrize("have,kw,status", [
    (0x20002, {}, "ALIGN"), (0x30000, dict(n=ctypes.c_void_p(0x30000)), "SHAPE"), (0x30010, dict(n=ctypes.c_void_p(0x30000)), "SHAPE"),
    (0x2fff0, dict(n=ctypes.c_void_p(0x30000)), "SHAPE"), (0x40000, dict(nd=ctypes.c_void_p(0x40000)), "SHAPE"),
    (0x40004, dict(nd=ctypes.c_void_p(0x40000)), "SHAPE"), (0x3fffc, dict(nd=ctypes.c_void_p(0x40000)), "SHAPE"),
    (0x50000, dict(T=65), "SHAPE"), (0x50000, dict(q=None), "NULL")])
def test_append_with_counts_refuses(have, kw, status):
    a = dict(T=3, q=FAKE, n=FAKE, nd=None)
    a.update(kw)
    row = (I64 * 2)(3 * 1024, 1024)
    assert stc.load_library().stc_rotary_append_drafts(
        ctypes.byref(_shape(None)), a["T"], a["q"], row, FAKE, row, FAKE, row, ctypes.c_void_p(0x90000), FAKE, FAKE,
        a["n"], a["nd"], 16, None, 0, 64, 0, FAKE, 1.0, None, 0, ctypes.c_void_p(have), None,
        None) == getattr(stc, "STC_ERR_" + status)


@pytest.mark.parametrize("counts,status", [(0x20002, "ALIGN"), (0x1000, "SHAPE"), (0x1010, "SHAPE"), (0x1030, "SHAPE"),
                                           (0xff0, "SHAPE")])
def test_accept_with_counts_refuses(counts, status):
    size = 5 * 2 * 16 * 128 * 2
    n = _ptrs([0x1000, 0x1020])
    assert stc.load_library().stc_accept_drafts(
        ctypes.byref(_shape(None)), 8, 2, _ptrs([0x100000, 0x100000 + size]), _ptrs([0x900000, 0x900000 + size]), n, n, 16,
        FAKE, ctypes.c_void_p(counts), None) == getattr(stc, "STC_ERR_" + status)


def test_null_shape():
    lib = stc.load_library()
    assert lib.stc_accept_tail(None, 1, 1, None, None, None, None, 1, None, None) == stc.STC_ERR_NULL
    assert lib.stc_fork_tail(None, 1, None, None, None, None, 1, None, None, None, None) == stc.STC_ERR_NULL
    assert stc.load_library().stc_tree_workspace_bytes(None, 1, 1, 1, 1) == 0


def test_a_tree_from_parents():
    bits = stc.tree_from_parents([-1, 0, 0, 2, -1], device="cpu")
    assert bits.tolist() == [0b1, 0b11, 0b101, 0b1101, 0b10000]
    chain = stc.tree_from_parents(list(range(-1, 63)), device="cpu")
    assert chain[:63].tolist() == [(2 << t) - 1 for t in range(63)] and chain[63] == -1
    two = stc.tree_from_parents([[-1, 0], [-1, -1]], device="cpu")
    assert two.tolist() == [[1, 3], [1, 2]]
    for bad in ([], [0], [-1, 1], [-2], list(range(-1, 64)), [[-1], []]):
        with pytest.raises(ValueError):
            stc.tree_from_parents(bad, device="cpu")


def test_drafts_have_the_nodes_that_were_said():
    cache = stc.RoutedCache.__new__(stc.RoutedCache)
    cache.B, cache.N, cache.n_tail, cache.next_pos = 1, 64, 0, 64
    b = stc.SharedPrefix.__new__(stc.SharedPrefix)
    b.prefix, b.N, b.pos0, b.rotary, b.nodes, b._q_tree = cache, 64, None, None, (4, 9), None

    class Rows:
        shape = (1, 5, 8, 64)
    with pytest.raises(ValueError, match="nodes"):
        b.draft(Rows, None, None)
    cache.n_tail = 2                                           # not whole any more
    with pytest.raises(ValueError, match="tail of its own"):
        b.draft(Rows, None, None)
    with pytest.raises(ValueError, match="tail of its own"):
        b._attend_tree(Rows, None, None, None, None)


def test_prefixes_of_their_own_do_not_exchange_tails():
    b = stc.OwnPrefixes.__new__(stc.OwnPrefixes)
    with pytest.raises(ValueError):
        b.fork(src=[0])


@pytest.mark.parametrize("bad", [None, 3, "tails", {}])
def test_layers_are_lists(bad):
    with pytest.raises(TypeError):
        stc.stc_accept_tail(stc.make_shape(**SHAPE), 3, bad, [], [], 16, None)
    with pytest.raises(TypeError):
        stc.stc_fork_tail(stc.make_shape(**SHAPE), bad, [], [], 16, None)


def test_layers_are_some():
    for n in (0, 1025):
        with pytest.raises(ValueError):
            stc.stc_accept_tail(stc.make_shape(**SHAPE), 3, [None] * n, [None], [None], 16, None)
