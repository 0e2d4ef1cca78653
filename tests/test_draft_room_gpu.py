"""Drafts that a sequence has no room for: nothing of them is written, and the calls behind leave its tail, its length
and its rows of the outputs as they are."""
import numpy as np
import pytest
import torch

import paper_2604_21335_amd as stc
from oracle import stc_oracle as O
from tests import parity as PT
from tests.helpers import randn_bf16
from tests.test_drafts_gpu import make_layers
from tests.test_tree_gpu import BF16, DEV, F32, dev_bits, limits, random_tree

pytestmark = pytest.mark.gpu
B, D, Hq, Hkv, T, CAP = 6, 64, 6, 2, 7, 40
# room for all nodes, for one, for just all, for none; padding; for all but one
FIRST = np.array([0, CAP - 1, CAP - T, CAP, -1, CAP - T + 1], dtype=np.int32)


def make(own, L=2, seed=5):
    rng, layers, host = make_layers(L, B, own, cap=CAP, seed=seed)
    for x in layers:
        x.n_tail.copy_(torch.from_numpy(FIRST))
        for t in (x.K_tail, x.V_tail, x._q_tree, x._out_tree):
            t.copy_(PT.to_dev_bf16(randn_bf16(rng, tuple(t.shape))))
    return rng, layers, host


def inputs(rng, turn, layers):
    """Trees, counts and kept sets of a turn; in the first, kept nodes that are not there."""
    bits = random_tree(rng, B, T)
    counts = np.array([T, 2, T, 1, T, T]) if turn == 0 else rng.integers(0, T + 1, size=B)
    kept = np.array([2**T - 1, 2**T - 1, 1, 1, 1, 0b111], dtype=np.uint64) if turn == 0 else bits[:, -1]
    rows = [PT.to_dev_bf16(randn_bf16(rng, (B, T, Hq + 2 * Hkv, D))) for _ in layers]
    return bits, counts.astype(np.int32), kept, rows


def parts(rows):
    return rows[:, :, :Hq], rows[:, :, Hq:Hq + Hkv], rows[:, :, Hq + Hkv:]


def view(t):
    return t[:B * T * Hq * D].view(B, T, Hq, D)


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("counted", [False, True])
@pytest.mark.parametrize("again", [False, True])
def test_a_round_leaves_a_sequence_without_room_as_it_is(own, counted, again):
    """Two layers, each call against the oracle.  again: the counts are given to the attention as well."""
    rng, layers, host = make(own)
    for turn in range(5):
        bits, counts, kept, rows = inputs(rng, turn, layers)
        nd = torch.from_numpy(counts).to(DEV) if counted else None
        now = layers[0].n_tail.cpu().numpy()
        nodes = counts if counted else np.full(B, T, dtype=np.int32)
        has = np.where((now >= 0) & (now.astype(np.int64) + nodes <= CAP), nodes, 0)
        tails = []
        for x, r, (K, V, mask) in zip(layers, rows, host):
            x.dev_status.zero_()
            old = [PT.host_bf16(t) for t in (x.K_tail, x.V_tail, view(x._q_tree))]
            old_out = view(x._out_tree).clone()
            q = x.draft(*parts(r), dev_bits(bits), nd)
            assert int(x.dev_status) == int(((now >= 0) & (nodes > has)).any())
            new = [PT.host_bf16(t) for t in (x.K_tail, x.V_tail, q)]
            for b in range(B):
                m, n = int(has[b]), max(int(now[b]), 0)
                for o, w in zip(old[:2], new[:2]):
                    assert np.array_equal(w[b, :, :n], o[b, :, :n]) and np.array_equal(w[b, :, n + m:], o[b, :, n + m:])
                assert np.array_equal(new[1][b, :, n:n + m], PT.host_bf16(r[b, :m, Hq + Hkv:].transpose(0, 1)))
                assert np.array_equal(new[2][b, m:], old[2][b, m:])
            out = x.attend_tree(q, dev_bits(bits), nd if again else None)
            want, size, top, on = O.tree_attention_all(new[2], K, V, mask, None, 8, new[0], new[1], now, bits, has)
            lim = limits(want, size, top, 100 + CAP, D, F32)
            assert (np.abs(out.double().cpu().numpy() - want) <= lim)[on].all(), turn
            off = torch.from_numpy(~on).to(DEV)
            assert torch.equal(out[off], old_out[off]), turn
            tails.append(new[:2])
        layers[0].accept(dev_bits(kept), T, layers[1:])
        for x, y in zip(layers, tails):
            for t, rows0 in zip((x.K_tail, x.V_tail), y):
                for b in range(B):
                    want, n = O.accept(rows0[b], now[b], T, int(kept[b]) & (1 << int(has[b])) - 1)
                    assert np.array_equal(PT.host_bf16(t[b]), want) and int(x.n_tail[b]) == n, (turn, b)


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("counted", [False, True])
def test_captured_rounds_leave_a_sequence_without_room_as_it_is(own, counted):
    """A captured round, replayed until sequences are full and beyond, against an eager twin."""
    rng, layers, _ = make(own)
    _, twins, _ = make(own)
    tree, keep = torch.zeros(B, T, dtype=torch.int64, device=DEV), torch.zeros(B, dtype=torch.int64, device=DEV)
    nd = torch.zeros(B, dtype=torch.int32, device=DEV) if counted else None
    rows = [torch.zeros(B, T, Hq + 2 * Hkv, D, dtype=BF16, device=DEV) for _ in layers]

    def go(some):
        for x, r in zip(some, rows):
            x.step_tree(*parts(r), tree, nd)
        some[0].accept(keep, T, some[1:])
    go(layers), go(twins)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go(layers)
    for turn in range(12):
        bits, counts, kept, new = inputs(rng, turn, layers)
        tree.copy_(dev_bits(bits)), keep.copy_(dev_bits(kept))
        if counted:
            nd.copy_(torch.from_numpy(counts))
        for r, n in zip(rows, new):
            r.copy_(n)
        before = [(x.n_tail.clone(), x.K_tail.clone(), x.V_tail.clone()) for x in layers]
        g.replay()
        torch.cuda.synchronize()
        go(twins)
        torch.cuda.synchronize()
        nodes = torch.from_numpy(counts).to(DEV) if counted else torch.full((B,), T, device=DEV)
        for x, y, (n, K, V) in zip(layers, twins, before):
            for a in ("n_tail", "K_tail", "V_tail", "_q_tree", "_out_tree"):
                assert torch.equal(getattr(x, a), getattr(y, a)), (turn, a)
            full = (n + nodes > CAP) | (n < 0)
            assert torch.equal(x.n_tail[full], n[full])
            assert torch.equal(x.K_tail[full], K[full]) and torch.equal(x.V_tail[full], V[full])
            assert int(x.n_tail.max()) <= CAP


@pytest.mark.parametrize("T", [1, 5, 64])
@pytest.mark.parametrize("counted", [False, True])
def test_counts_of_what_was_written(T, counted):
    """Both sides of the end of the tail, lengths and counts that are none."""
    cap, n = 70, [0, 70 - T, 71 - T, 69, 70, 75, 2**31 - 1, -1, -2**31, 3, 4, 5]
    B, Hkv, D = len(n), 2, 64
    nd = [T, T, T, 1, 1, 1, T, T, T, 0, -5, T + 9]
    q = torch.zeros(B, T, 4, D, dtype=BF16, device=DEV)
    kv = torch.ones(B, T, Hkv, D, dtype=BF16, device=DEV)
    Kt, Vt = (torch.zeros(B, Hkv, cap, D, dtype=BF16, device=DEV) for _ in range(2))
    have = torch.full((B + 2,), 77, dtype=torch.int32, device=DEV)
    dn = torch.tensor(n, dtype=torch.int32, device=DEV)
    shape = stc.make_shape(B, 4, Hkv, D, 16, 1, 16)
    stc.stc_rotary_append_tree(shape, q, kv, kv, q, Kt, Vt, dn, cap, None, 0, 0, n_have=have[1:-1],
                               n_draft=torch.tensor(nd, dtype=torch.int32, device=DEV) if counted else None)
    nodes = [min(max(x, 0), T) if counted else T for x in nd]
    want = [x if m >= 0 and m + x <= cap else 0 for x, m in zip(nodes, n)]
    assert have.tolist() == [77] + want + [77]
    written = Kt[:, 0, :, 0].sum(1).int()
    assert written.tolist() == want


@pytest.mark.parametrize("L", [1, 3, 70])
def test_accepted_nodes_are_those_that_are_there(L):
    """Counts of none, some, all and more than all nodes, bits of others set."""
    T, cap, B, Hkv, D = 9, 30, 6, 1, 64
    rng = np.random.default_rng(L)
    K, V = (randn_bf16(rng, (L, B, Hkv, cap, D)) for _ in range(2))
    n = np.array([0, 5, 21, 25, -1, 7], dtype=np.int32)
    nd = np.array([0, 4, 9, 9, 3, 70], dtype=np.int32)
    keep = rng.integers(0, 2**63, size=B).astype(np.uint64) * np.uint64(2) + np.uint64(1)
    dK, dV = ([PT.to_dev_bf16(x) for x in y] for y in (K, V))
    dn = [torch.from_numpy(n).to(DEV) for _ in range(L)]
    stc.stc_accept_tail(stc.make_shape(B, Hkv, Hkv, D, 16, 1, 16), T, dK, dV, dn, cap, dev_bits(keep),
                        n_draft=torch.from_numpy(nd).to(DEV))
    for i in range(L):
        for b in range(B):
            there = int(keep[b]) & (1 << min(int(nd[b]), T)) - 1
            for t, x in ((dK, K), (dV, V)):
                want, m = O.accept(x[i, b], n[b], T, there)
                assert np.array_equal(PT.host_bf16(t[i][b]), want) and int(dn[i][b]) == m


def test_counts_that_do_not_fit():
    _, (x,), _ = make(False, L=1)
    q = torch.zeros(B, T, Hq, D, dtype=BF16, device=DEV)
    for bad, error in ((torch.zeros(1, dtype=torch.int32, device=DEV), ValueError),
                       (torch.zeros(B, dtype=torch.int64, device=DEV), TypeError)):
        with pytest.raises(error):
            x.attend_tree(q, None, bad)
    with pytest.raises(stc.StcError):
        stc.stc_accept_tail(x.shape, T, [x.K_tail], [x.V_tail], [x.n_tail], CAP, torch.zeros(B, dtype=torch.int64, device=DEV),
                            n_draft=x.n_tail)
