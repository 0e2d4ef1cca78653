"""Drafted tokens from positions to accepted rows, tails that sequences take over, and rounds of all of them."""
import numpy as np
import pytest
import torch

import paper_2604_21335_amd as stc
from oracle import stc_oracle as O
from tests import parity as PT
from tests.helpers import bits_to_f64, randn_bf16
from tests.test_tree_gpu import BF16, DEV, F32, dev_bits, limits, random_tree

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------
def append(B, T, Hq, Hkv, D, rot, cap, n, nd=None, tree=None, interleaved=False, pos=None, pos0=0, fused=False,
           amplitude=1.0, seed=0, base=1e4):
    """Runs the call and compares every element of what it may write with the rotation in 64 bits."""
    rng = np.random.default_rng(seed)
    rows = randn_bf16(rng, (B, T, Hq + 2 * Hkv, D))
    n = np.resize(n, B).astype(np.int32)
    nd = None if nd is None else np.resize(nd, B).astype(np.int32)
    Kt, Vt, q0 = randn_bf16(rng, (B, Hkv, cap, D)), randn_bf16(rng, (B, Hkv, cap, D)), randn_bf16(rng, (B, T, Hq, D))
    turns = O.rotary_turns(rot, base) if rot else None
    x = PT.to_dev_bf16(rows)
    parts = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    if not fused:
        parts = [p.contiguous() for p in parts]
    dq, dK, dV = PT.to_dev_bf16(q0), PT.to_dev_bf16(Kt), PT.to_dev_bf16(Vt)
    dn = torch.from_numpy(n).to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    shape = stc.make_shape(B, Hq, Hkv, D, 16, 1, 16)
    stc.stc_rotary_append_tree(
        shape, *parts, dq, dK, dV, dn, cap, torch.from_numpy(turns).to(DEV) if rot else None, rot,
        stc.STC_ROTARY_INTERLEAVED if interleaved else stc.STC_ROTARY_HALVES,
        tree=None if tree is None else dev_bits(tree), n_draft=None if nd is None else torch.from_numpy(nd).to(DEV),
        amplitude=amplitude, pos=None if pos is None else torch.from_numpy(pos.astype(np.int32)).to(DEV), pos0=pos0,
        dev_status=status)
    torch.cuda.synchronize()
    assert np.array_equal(dn.cpu().numpy(), n)
    got = [PT.host_bf16(t) for t in (dq, dK, dV)]
    want = [q0.copy(), Kt.copy(), Vt.copy()]
    full = False
    for b in range(B):
        nodes = T if nd is None else min(max(nd[b], 0), T)
        if n[b] >= 0 and nodes > max(cap - int(n[b]), 0):       # (no nodes need no room)
            full = True
        if n[b] < 0 or nodes > cap - n[b]:
            continue
        for t in range(nodes):
            if pos is not None:
                at = pos[b, t]
            else:
                bits = (1 << t) - 1 if tree is None else int((tree if tree.ndim == 1 else tree[b])[t])
                at = pos0 + n[b] + sum(bits >> u & 1 for u in range(t))
            y = bits_to_f64(rows[b, t, :Hq + Hkv])
            if rot:
                y = O.rotary(y, np.float64(at), turns, rot, interleaved, amplitude)
            exact = bits_to_f64(rows[b, t, :Hq + Hkv])
            copied = [np.array_equal(got[0][b, t, :, rot:], rows[b, t, :Hq, rot:]),
                      np.array_equal(got[1][b, :, n[b] + t, rot:], rows[b, t, Hq:Hq + Hkv, rot:]),
                      np.array_equal(got[2][b, :, n[b] + t], rows[b, t, Hq + Hkv:])]
            assert all(copied), (b, t, copied)
            g = bits_to_f64(np.concatenate([got[0][b, t], got[1][b, :, n[b] + t]]))
            # one rounding to bf16, 2^-8 of the value; before it cosine and sine are off by 2^-19 (the instructions'
            # error, and half a step of the reduced angle in 32 bits, 2^-25 turns), products and sum by 2^-22
            size = np.abs(exact).max(-1, keepdims=True) * 2 * amplitude
            assert (np.abs(g - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -17 * size + 1e-38).all(), (b, t)
            for w, gg, i in ((want[0], got[0], (b, t)), (want[1], got[1], (b, slice(None), n[b] + t)),
                             (want[2], got[2], (b, slice(None), n[b] + t))):
                w[i] = gg[i]
    for w, g in zip(want, got):
        assert np.array_equal(w, g)                            # nothing else was written
    assert int(status.item()) == int(full)
    return got


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,rot", [(1, 1, 1, 1, 64, 64), (3, 5, 8, 2, 128, 128), (4, 64, 7, 1, 128, 64),
                                              (2, 63, 32, 32, 64, 16), (5, 17, 28, 4, 128, 48), (2, 3, 4, 2, 64, 0)])
def test_append(B, T, Hq, Hkv, D, rot, interleaved, fused):
    rng = np.random.default_rng(T)
    append(B, T, Hq, Hkv, D, rot, T + 20, [0, 20, -1, 7, 13], nd=[T, T - 1, T, 1, 0], tree=random_tree(rng, B, T),
           interleaved=interleaved, fused=fused, pos0=100, seed=T)


def test_append_chain_one_tree_and_given_positions():
    rng = np.random.default_rng(0)
    append(3, 9, 4, 2, 128, 128, 30, [0, 5, 21], pos0=32768)
    append(3, 9, 4, 2, 128, 128, 30, [0, 5, 21], tree=random_tree(rng, 1, 9)[0], pos0=32768)
    append(3, 9, 4, 2, 128, 128, 30, [0, 5, 21], pos=rng.integers(-5, 2**31, size=(3, 9)), amplitude=1.3)
    # bits of nodes behind a node do not count for its position
    append(2, 4, 4, 2, 128, 128, 30, [3, 8], tree=np.array([15, 14, 13, 15], dtype=np.uint64))


def test_append_far_positions():
    append(2, 64, 4, 2, 64, 64, 100, [0, 36], pos0=2**31 - 100, base=5e5)


@pytest.mark.parametrize("T", [1, 4, 64])
def test_append_where_there_is_no_room(T):
    cap = 64
    append(7, T, 4, 2, 64, 32, cap, [cap - T, cap - T + 1, cap, cap + 5, 2**31 - 1, -1, -2**31])
    append(3, T, 4, 2, 64, 32, cap, [cap - 1, cap, cap + 1], nd=[1, 0, -3])


def test_append_in_place_of_the_queries():
    rng = np.random.default_rng(1)
    q = PT.to_dev_bf16(randn_bf16(rng, (3, 5, 4, 64)))
    k, v = (PT.to_dev_bf16(randn_bf16(rng, (3, 5, 2, 64))) for _ in range(2))
    shape = stc.make_shape(3, 4, 2, 64, 16, 1, 16)
    r = stc.Rotary(64)
    Kt = torch.zeros(2, 3, 2, 20, 64, dtype=BF16, device=DEV)
    n = torch.tensor([0, 3, 9], dtype=torch.int32, device=DEV)
    out = torch.zeros_like(q)
    stc.stc_rotary_append_tree(shape, q, k, v, out, Kt[0], Kt[1], n, 20, r.turns, 64, r.layout)
    stc.stc_rotary_append_tree(shape, q, k, v, q, Kt[0], Kt[1], n, 20, r.turns, 64, r.layout)
    assert torch.equal(q, out)
    with pytest.raises(stc.StcError):                          # a slice of a projection's output has other strides
        x = torch.zeros(3, 5, 8, 64, dtype=BF16, device=DEV)
        stc.stc_rotary_append_tree(shape, x[:, :, :4], k, v, x.view(-1)[:q.numel()].view(q.shape), Kt[0], Kt[1], n,
                                   20, r.turns, 64, r.layout)
    with pytest.raises(ValueError):
        stc.stc_rotary_append_tree(shape, q.transpose(1, 2), k, v, q, Kt[0], Kt[1], n, 20, r.turns, 64, r.layout)


def test_one_node_is_an_appended_token():
    rng = np.random.default_rng(2)
    q = PT.to_dev_bf16(randn_bf16(rng, (4, 8, 128)))
    k, v = (PT.to_dev_bf16(randn_bf16(rng, (4, 2, 128))) for _ in range(2))
    shape, r = stc.make_shape(4, 8, 2, 128, 16, 1, 16), stc.Rotary(128, base=1e6)
    n = torch.tensor([0, 3, -1, 7], dtype=torch.int32, device=DEV)
    got = []
    for tree in (False, True):
        Kt, Vt = (torch.zeros(4, 2, 8, 128, dtype=BF16, device=DEV) for _ in range(2))
        out = torch.zeros_like(q)
        if tree:
            stc.stc_rotary_append_tree(shape, q[:, None], k[:, None], v[:, None], out, Kt, Vt, n, 8, r.turns, 128,
                                       r.layout, pos0=50)
        else:
            stc.stc_rotary_append(shape, q, k, v, out, Kt, Vt, n, 8, r.turns, 128, r.layout, pos0=50)
        got.append((out, Kt, Vt))
    assert all(torch.equal(a, b) for a, b in zip(*got))


# ------------------------------------------------------------------------------------------
# accept and fork
# ------------------------------------------------------------------------------------------
class Tails:
    def __init__(self, L, B, Hkv, cap, D, n, seed=0):
        rng = np.random.default_rng(seed)
        self.L, self.B, self.cap = L, B, cap
        self.K, self.V = (rng.integers(0, 1 << 16, size=(L, B, Hkv, cap, D)).astype(np.uint16) for _ in range(2))
        self.n = np.stack([np.resize(np.roll(n, i), B) for i in range(L)]).astype(np.int32)
        self.shape = stc.make_shape(B, Hkv, Hkv, D, 16, 1, 16)
        self.reset()

    def reset(self):
        self.dK, self.dV = ([PT.to_dev_bf16(x) for x in y] for y in (self.K, self.V))
        self.dn = [torch.from_numpy(x).to(DEV) for x in self.n]

    def check(self, want, outs=None):
        torch.cuda.synchronize()
        for i in range(self.L):
            K, V, n = want(i)
            assert np.array_equal(PT.host_bf16(self.dK[i]), K) and np.array_equal(PT.host_bf16(self.dV[i]), V)
            assert np.array_equal((outs or self.dn)[i].cpu().numpy(), n)


def check_accept(L, B, Hkv, cap, D, T, n, keep, apart=False, seed=0):
    t = Tails(L, B, Hkv, cap, D, n, seed)
    keep = np.resize(np.array(keep, dtype=np.uint64), B)
    outs = [torch.full((B,), 77, dtype=torch.int32, device=DEV) for _ in range(L)] if apart else None
    stc.stc_accept_tail(t.shape, T, t.dK, t.dV, t.dn, cap, dev_bits(keep), n_outs=outs)

    def want(i):
        K, V, m = t.K[i].copy(), t.V[i].copy(), t.n[i].copy()
        for b in range(B):
            K[b], m[b] = O.accept(t.K[i, b], t.n[i, b], T, keep[b])
            V[b], _ = O.accept(t.V[i, b], t.n[i, b], T, keep[b])
        return K, V, m
    t.check(want, outs)


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("L,B,Hkv,D", [(1, 1, 1, 64), (3, 5, 2, 128), (1, 4, 40, 128), (130, 3, 1, 64)])
@pytest.mark.parametrize("T", [1, 2, 9, 33, 64])
def test_accept(T, L, B, Hkv, D, apart):
    rng = np.random.default_rng(T + B)
    full = 2**64 - 1
    keep = [0, full, 1 << (T - 1), int(rng.integers(0, 2**63)) * 2 + 1, int(rng.integers(0, 2**63)), full ^ 1, full >> 1,
            0xAAAAAAAAAAAAAAAA, 0x5555555555555555, 1]
    cap = T + 30
    for i in range(0, 10, max(B, 2)):
        check_accept(L, B, Hkv, cap, D, T, [0, 30, 7, -1, 13], keep[i:] + keep[:i], apart, seed=i)


def test_accept_where_rows_end():
    for T in (3, 64):
        cap = 70
        check_accept(2, 7, 2, cap, 64, T, [cap - 2, cap - 1, cap, cap + 4, 2**31 - 1, -1, -2**31],
                     [2**64 - 1, 0b110, 0b11, 0b10], apart=False)


def check_fork(L, B, Hkv, cap, D, n, src, n_keep=None, apart=False, seed=0):
    t = Tails(L, B, Hkv, cap, D, n, seed)
    src = np.resize(np.array(src, dtype=np.int32), B)
    keep = None if n_keep is None else np.resize(np.array(n_keep, dtype=np.int32), B)
    outs = [torch.full((B,), 77, dtype=torch.int32, device=DEV) for _ in range(L)] if apart else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    stc.stc_fork_tail(t.shape, t.dK, t.dV, t.dn, cap, torch.from_numpy(src).to(DEV),
                      n_keep=None if keep is None else torch.from_numpy(keep).to(DEV), n_outs=outs, dev_status=status)

    def want(i):
        K, m = O.fork(t.K[i], t.n[i], src, keep)
        return K, O.fork(t.V[i], t.n[i], src, keep)[0], m
    t.check(want, outs)
    assert int(status.item()) == int(((src < -2) | (src >= B)).any())


@pytest.mark.parametrize("apart", [False, True])
@pytest.mark.parametrize("L,B,Hkv,cap,D", [(1, 1, 1, 5, 64), (2, 6, 2, 100, 128), (1, 33, 3, 130, 64), (70, 4, 1, 9, 128),
                                           (1, 200, 1, 40, 128), (1, 5, 2, 3000, 128)])
def test_fork(L, B, Hkv, cap, D, apart):
    rng = np.random.default_rng(B)
    n = rng.integers(-1, cap + 1, size=B)
    n[0] = cap
    maps = [np.arange(B), np.roll(np.arange(B), 1), rng.permutation(B), rng.integers(0, B, size=B), np.zeros(B),
            rng.integers(-2, B, size=B), np.arange(B)[::-1]]
    for i, src in enumerate(maps):
        check_fork(L, B, Hkv, cap, D, n, src, apart=apart, seed=i)
        check_fork(L, B, Hkv, cap, D, n, src, n_keep=rng.integers(-3, cap + 4, size=B), apart=apart, seed=i)


@pytest.mark.parametrize("B", [257, 1000, 2049, 4096])
@pytest.mark.parametrize("D", [64, 128])
def test_fork_of_many(B, D):
    """Columns of a row in turns, where not all sequences' rows fit one workgroup's registers."""
    rng = np.random.default_rng(B)
    check_fork(1, B, 1, 3, D, rng.integers(0, 4, size=B), rng.permutation(B))
    check_fork(2, B, 2, 2, D, rng.integers(0, 3, size=B), rng.integers(-2, B, size=B))


def test_fork_from_what_is_no_sequence():
    check_fork(2, 6, 2, 20, 64, [3, 25, 2**31 - 1, -1, -2**31, 7], [6, -3, 2**31 - 1, -2**31, 2, 1])
    check_fork(1, 6, 2, 20, 64, [3, 25, 2**31 - 1, -1, -2**31, 7], [1, 2, 4, 3, 5, 2], n_keep=[30, 2**31 - 1, 5, 5, -2**31, 1])


def test_layers_that_do_not_fit():
    t = Tails(2, 3, 2, 10, 64, [1, 2, 3])
    keep = torch.zeros(3, dtype=torch.int64, device=DEV)
    src = torch.zeros(3, dtype=torch.int32, device=DEV)
    for K, V, n, o, error in (
            (t.dK, t.dV[:1], t.dn, None, ValueError), (t.dK, t.dV, t.dn, t.dn[:1], ValueError),
            ([t.dK[0][:2], t.dK[1]], t.dV, t.dn, None, ValueError), ([t.dK[0].float(), t.dK[1]], t.dV, t.dn, None, TypeError),
            ([t.dK[0], t.dK[0]], t.dV, t.dn, None, stc.StcError), (t.dK, t.dK, t.dn, None, stc.StcError),
            (t.dK, t.dV, [t.dn[0], t.dn[0]], None, stc.StcError), (t.dK, t.dV, [t.dn[0].long(), t.dn[1]], None, TypeError),
            ([t.dK[0].cpu(), t.dK[1]], t.dV, t.dn, None, TypeError), ([None, t.dK[1]], t.dV, t.dn, None, stc.StcError),
            ([t.dK[0].transpose(1, 2), t.dK[1]], t.dV, t.dn, None, ValueError)):
        with pytest.raises(error):
            stc.stc_accept_tail(t.shape, 3, K, V, n, 10, keep, n_outs=o)
        with pytest.raises(error):
            stc.stc_fork_tail(t.shape, K, V, n, 10, src, n_outs=o)
    with pytest.raises(ValueError):
        stc.stc_accept_tail(t.shape, 3, t.dK, t.dV, t.dn, 10, keep[:2])
    with pytest.raises(stc.StcError):                          # the map is one of the lengths that are written
        stc.stc_fork_tail(t.shape, t.dK, t.dV, t.dn, 10, t.dn[0])
    # layers may share lengths that are written elsewhere
    outs = [torch.zeros(3, dtype=torch.int32, device=DEV) for _ in range(2)]
    stc.stc_accept_tail(t.shape, 3, t.dK, t.dV, [t.dn[0]] * 2, 10, keep + 1, n_outs=outs)
    assert outs[0].tolist() == outs[1].tolist() == [2, 3, 4]


def test_accept_and_fork_in_a_graph():
    """Replayed as lengths, kept sets and maps change, between eager work."""
    L, B, Hkv, cap, D, T = 3, 6, 2, 200, 128, 8
    t = Tails(L, B, Hkv, cap, D, [20] * 6)
    keep = torch.zeros(B, dtype=torch.int64, device=DEV)
    src = torch.arange(B, dtype=torch.int32, device=DEV)

    def call():
        stc.stc_accept_tail(t.shape, T, t.dK, t.dV, t.dn, cap, keep)
        stc.stc_fork_tail(t.shape, t.dK, t.dV, t.dn, cap, src)
    call()
    torch.cuda.synchronize()
    t.reset()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    K, V, n = t.K.copy(), t.V.copy(), t.n.copy()
    rng = np.random.default_rng(0)
    for turn in range(5):
        k, s = rng.integers(0, 256, size=B), rng.integers(0, B, size=B)
        for x, y in ((keep, k.astype(np.int64)), (src, s.astype(np.int32))):
            x.copy_(torch.from_numpy(y))
        g.replay()
        torch.cuda.synchronize()
        for i in range(L):
            for b in range(B):
                K[i, b], m = O.accept(K[i, b], n[i, b], T, k[b])
                V[i, b], n[i, b] = O.accept(V[i, b], n[i, b], T, k[b])
            V[i] = O.fork(V[i], n[i], s)[0]
            K[i], n[i] = O.fork(K[i], n[i], s)
        t.check(lambda i: (K[i], V[i], n[i]))


# ------------------------------------------------------------------------------------------
# all of them together
# ------------------------------------------------------------------------------------------
def make_layers(L, B, own, D=64, Hq=6, Hkv=2, N=100, cap=120, nodes=(1, 7), dtype=F32, seed=0, N_cap=128):
    rng = np.random.default_rng(seed)
    r = stc.Rotary(D, device=DEV)
    layers, host = [], []
    P = B if own else 1
    for _ in range(L):
        K, V = randn_bf16(rng, (P, Hkv, N, D)), randn_bf16(rng, (P, Hkv, N, D))
        mask = rng.integers(0, 256, size=(P, Hkv, N)).astype(np.uint16)
        c = stc.RoutedCache(P, Hq, Hkv, D, N, 8, 4, device=DEV, n_cap=N_cap)
        c.build(PT.to_dev_bf16(K), PT.to_dev_bf16(V), mask_in=PT.to_dev_u16(mask))
        layers.append(stc.OwnPrefixes(c, cap, r, dtype, nodes=nodes) if own else
                      stc.SharedPrefix(c, B, cap, r, dtype, nodes=nodes))
        host.append((K, V, mask))
    return rng, layers, host


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rounds_of_drafts_equal_token_by_token(own, dtype):
    """Two layers, rounds in which trees are drafted and a path of each is accepted; beside them the accepted tokens
    one by one.  Tails and lengths are equal bit by bit, and the nodes' outputs those of the single steps within
    what each may be off."""
    B, D, Hq, Hkv, T = 3, 64, 6, 2, 7
    rng, layers, host = make_layers(2, B, own, dtype=dtype)
    _, single, _ = make_layers(2, B, own, dtype=dtype)
    for turn in range(6):
        bits = random_tree(rng, B, T, back=3)
        tree = dev_bits(bits)
        nd = rng.integers(1, T + 1, size=B).astype(np.int32)
        last = np.array([rng.integers(0, x) for x in nd])
        keep = bits[np.arange(B), last]
        new = [PT.to_dev_bf16(randn_bf16(rng, (B, T, Hq + 2 * Hkv, D))) for _ in layers]
        d_nd = torch.from_numpy(nd).to(DEV)
        outs = []
        for x, rows in zip(layers, new):
            got = x.step_tree(rows[:, :, :Hq], rows[:, :, Hq:Hq + Hkv], rows[:, :, Hq + Hkv:], tree, d_nd)
            n0 = x.n_tail.cpu().numpy()
            K, V, mask = host[len(outs)]
            want, size, top, on = O.tree_attention_all(
                PT.host_bf16(x._q_tree[:B * T * Hq * D].view(B, T, Hq, D)), K, V, mask, None, 8, PT.host_bf16(x.K_tail),
                PT.host_bf16(x.V_tail), n0, bits, nd)
            lim = limits(want, size, top, 220, D, dtype)
            assert (np.abs(got.double().cpu().numpy() - want) <= lim)[on].all()
            outs.append((got.clone(), want, lim))
        layers[0].accept(dev_bits(keep), T, layers[1:])
        # the same tokens one by one; sequences whose path has ended are padding meanwhile
        path = [[u for u in range(T) if int(k) >> u & 1] for k in keep]
        for i in range(max(len(p) for p in path)):
            at = [p[i] if i < len(p) else -1 for p in path]
            for j, (x, rows) in enumerate(zip(single, new)):
                n = x.n_tail.clone()
                gone = torch.tensor([a < 0 for a in at], device=DEV)
                x.n_tail[gone] = -1
                pick = rows[torch.arange(B), torch.tensor([max(a, 0) for a in at])]
                got = x.step(pick[:, :Hq], pick[:, Hq:Hq + Hkv], pick[:, Hq + Hkv:]).double().cpu().numpy()
                for b, a in enumerate(at):
                    if a >= 0:
                        want, lim = outs[j][1][b, a], outs[j][2][b, a]
                        assert (np.abs(got[b] - want) <= lim).all(), (turn, i, j, b)
                x.n_tail[gone] = n[gone]
        for x, y in zip(layers, single):
            assert torch.equal(x.n_tail, y.n_tail)
            for b in range(B):
                n = int(x.n_tail[b])
                assert torch.equal(x.K_tail[b, :, :n], y.K_tail[b, :, :n])
                assert torch.equal(x.V_tail[b, :, :n], y.V_tail[b, :, :n])
    assert int(layers[0].n_tail.min()) >= 6 and int(layers[0].dev_status) == 0


def test_beams():
    """Sequences fork, go on differently, are freed and start anew; each then equals one that was built alone."""
    B, D, Hq, Hkv = 4, 64, 6, 2
    rng, (a,), host = make_layers(1, B, False, seed=3)
    tokens = {b: [] for b in range(B)}

    def go(alive):
        rows = PT.to_dev_bf16(randn_bf16(rng, (B, Hq + 2 * Hkv, D)))
        out = a.step(rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:])
        for b in alive:
            tokens[b] = tokens[b] + [rows[b]]
        return out
    for _ in range(5):
        go(range(B))
    a.fork(torch.tensor([1, 0, 1, 3], dtype=torch.int32, device=DEV))
    tokens = {0: tokens[1], 1: tokens[0], 2: tokens[1], 3: tokens[3]}
    for _ in range(3):
        go(range(B))
    a.fork(torch.tensor([2, -1, 2, -2], dtype=torch.int32, device=DEV),
           n_keep=torch.tensor([6, 9, 99, 9], dtype=torch.int32, device=DEV))
    tokens = {0: tokens[2][:6], 1: [], 2: tokens[2], 3: []}
    assert a.n_tail.tolist() == [6, -1, 8, 0]
    for _ in range(2):
        out = go([0, 2, 3]).clone()
    assert a.n_tail.tolist() == [8, -1, 10, 2] and int(a.dev_status) == 0
    _, (alone,), _ = make_layers(1, B, False, seed=3)
    for b in (0, 2, 3):
        alone.n_tail.fill_(-1)
        alone.n_tail[b] = 0
        for row in tokens[b]:
            got = alone.step(*(row[None].expand(B, -1, -1)[:, s].contiguous()
                               for s in (slice(0, Hq), slice(Hq, Hq + Hkv), slice(Hq + Hkv, None))))
        n = len(tokens[b])
        assert torch.equal(a.K_tail[b, :, :n], alone.K_tail[b, :, :n])
        assert torch.equal(a.V_tail[b, :, :n], alone.V_tail[b, :, :n])
        assert torch.equal(got[b], out[b])
    a.fork(n_keep=torch.tensor([3, 3, 3, 3], dtype=torch.int32, device=DEV))
    assert a.n_tail.tolist() == [3, -1, 3, 2]


def test_a_question_as_a_chain_that_is_accepted_whole():
    """A prompt's tokens, 7 at a time, into the tails: rows and lengths of token by token."""
    B, D, Hq, Hkv, T = 3, 64, 6, 2, 7
    rng, (a,), _ = make_layers(1, B, False)
    _, (b,), _ = make_layers(1, B, False)
    lens = [7, 20, 12]
    rows = PT.to_dev_bf16(randn_bf16(rng, (B, 21, Hq + 2 * Hkv, D)))
    for i in range(0, 21, T):
        nd = torch.tensor([min(max(x - i, 0), T) for x in lens], dtype=torch.int32, device=DEV)
        part = rows[:, i:i + T]
        out = a.step_tree(part[:, :, :Hq], part[:, :, Hq:Hq + Hkv], part[:, :, Hq + Hkv:], None, nd)
        a.accept((torch.ones(B, dtype=torch.int64, device=DEV) << nd.long()) - 1, T)
    assert a.n_tail.tolist() == lens
    for i in range(20):
        b.n_tail[torch.tensor([i >= x for x in lens], device=DEV)] = -1
        got = b.step(rows[:, i, :Hq], rows[:, i, Hq:Hq + Hkv], rows[:, i, Hq + Hkv:])
    for s, n in enumerate(lens):
        assert torch.equal(a.K_tail[s, :, :n], b.K_tail[s, :, :n]) and torch.equal(a.V_tail[s, :, :n], b.V_tail[s, :, :n])
    # the second sequence's last token: both within 2^-13 (weights' parts, sums of 120 tokens) of its exact output
    assert (out[1, 5] - got[1]).abs().max() <= 2.0 ** -12


def test_pages_of_prefixes_of_their_own():
    """The pages that each sequence's root selects, attended by its nodes."""
    B, D, Hq, Hkv, T = 3, 64, 6, 2, 7
    rng, (a,), ((K, V, mask),) = make_layers(1, B, True)
    rows = PT.to_dev_bf16(randn_bf16(rng, (B, T, Hq + 2 * Hkv, D)))
    bits = random_tree(rng, B, T)
    q = a.draft(rows[:, :, :Hq], rows[:, :, Hq:Hq + Hkv], rows[:, :, Hq + Hkv:], dev_bits(bits))
    a.prefix.select(q[:, 0].contiguous())
    out = a.attend_tree(q, dev_bits(bits), page_idx=a.prefix.page_idx)
    want, size, top, on = O.tree_attention_all(PT.host_bf16(q), K, V, mask, a.prefix.page_idx.cpu().numpy(), 8,
                                               PT.host_bf16(a.K_tail), PT.host_bf16(a.V_tail), np.zeros(B, int), bits)
    assert on.all() and (np.abs(out.double().cpu().numpy() - want) <= limits(want, size, top, 100, D, F32)).all()


def test_a_round_in_a_graph():
    """Draft, attend and accept, captured once and replayed as the tails grow; each replay against an eager twin."""
    B, D, Hq, Hkv, T = 3, 64, 6, 2, 7
    rng, (a,), _ = make_layers(1, B, False)
    _, (b,), _ = make_layers(1, B, False)
    x = torch.zeros(B, T, Hq + 2 * Hkv, D, dtype=BF16, device=DEV)
    tree, keep = torch.zeros(B, T, dtype=torch.int64, device=DEV), torch.zeros(B, dtype=torch.int64, device=DEV)
    nd = torch.zeros(B, dtype=torch.int32, device=DEV)

    def call(s):
        s.step_tree(x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], tree, nd)
        s.accept(keep, T)
    call(a)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(a)
    for turn in range(5):
        bits = random_tree(rng, B, T)
        tree.copy_(dev_bits(bits))
        nd.copy_(torch.from_numpy(rng.integers(1, T + 1, size=B).astype(np.int32)))
        keep.copy_(tree[torch.arange(B), (nd - 1).long()])
        x.copy_(PT.to_dev_bf16(randn_bf16(rng, (B, T, Hq + 2 * Hkv, D))))
        g.replay()
        torch.cuda.synchronize()
        call(b)
        torch.cuda.synchronize()
        assert torch.equal(a.n_tail, b.n_tail) and torch.equal(a._out_tree, b._out_tree), turn
        for s in range(B):
            n = int(a.n_tail[s])
            assert torch.equal(a.K_tail[s, :, :n], b.K_tail[s, :, :n]) and torch.equal(a.V_tail[s, :, :n], b.V_tail[s, :, :n])
