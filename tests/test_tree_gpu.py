"""Attention of drafted tokens over compressed prefixes and tails, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2604_21335_amd as stc
from oracle import stc_oracle as O
from tests import parity as PT
from tests.helpers import randn_bf16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
NAN = 0x7FC0


def limits(want, size, top, tokens, D, dtype):
    """How far an output may be off, from the arithmetic.  e: relative error of a weight.  Two bf16 parts leave
    2^-16 of it; the exponent is a float dot product of D terms, scaled and shifted in base 2, off by at most
    (D + 4) 2^-24 of the sum of magnitudes behind it, which shifts the weight by as much; the exponential itself by
    2^-22.  Weighted sum and sum of weights each carry e and the roundings of at most `tokens` additions.  A bf16
    output is that, rounded: half a step, 2^-8 of the value."""
    e = 2.0 ** -16 + (D + 4) * 2.0 ** -24 * max(top, 1.0) + 2.0 ** -22
    lim = (2 * e + (tokens + 64) * 2.0 ** -24) * size
    return lim + (2.0 ** -8 * (np.abs(want) + lim) if dtype == BF16 else 0) + 1e-30


def random_tree(rng, B, T, back=6):
    """Bits of ancestors and itself; a node's parent is one of the nodes before it."""
    seen = np.zeros((B, T), dtype=np.uint64)
    for t in range(T):
        seen[:, t] = np.uint64(1) << np.uint64(t)
        if t:
            seen[:, t] |= seen[np.arange(B), rng.integers(max(0, t - back), t, size=B)]
    return seen


def dev_bits(x):
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int64)).to(DEV)


class Case:
    """Host arrays of prefixes, tails and nodes, and their device copies; what must not be read holds NaN."""

    def __init__(self, B, T, Hq, Hkv, D, N, G, cap, seed=0, each=False, n_tail=None, n_draft=None, tree="random",
                 n_cap=0, scale=1.0, v_cap=None):
        rng = np.random.default_rng(seed)
        self.B, self.T, self.Hq, self.Hkv, self.D, self.N, self.G, self.cap = B, T, Hq, Hkv, D, N, G, cap
        P = self.P = B if each else 1
        self.q = randn_bf16(rng, (B, T, Hq, D), scale)
        self.K, self.V = randn_bf16(rng, (P, Hkv, N, D)), randn_bf16(rng, (P, Hkv, N, D))
        self.mask = rng.integers(0, 1 << G, size=(P, Hkv, N)).astype(np.uint16)
        self.Kt, self.Vt = (randn_bf16(rng, (B, Hkv, cap, D)) for _ in range(2))
        self.n = rng.integers(0, max(cap - T, 0) + 1, size=B) if n_tail is None else np.resize(n_tail, B)
        self.n = self.n.astype(np.int32)
        self.nd = None if n_draft is None else np.resize(n_draft, B).astype(np.int32)
        self.tree = random_tree(rng, B, T) if isinstance(tree, str) else tree
        Nc = n_cap or N
        off = np.zeros((P, Hkv, Nc + 1), dtype=np.uint32)
        kept = ((self.mask[..., None].astype(np.int64) >> np.arange(G)) & 1).sum(-1)
        off[..., 1:N + 1] = kept.cumsum(2)
        off[..., N + 1:] = 0xFFFFFFF0
        self.v_cap = v_cap or max(int(off[..., N].max()), 1) + 3
        v = np.full((P, Hkv, self.v_cap, D // G), NAN, dtype=np.uint16)
        for p in range(P):
            for h in range(Hkv):
                packed = O.pack_values(self.V[p, h], self.mask[p, h], off[p, h, :N + 1], G)[:self.v_cap]
                v[p, h, :len(packed)] = packed
        K = np.full((P, Hkv, Nc, D), NAN, dtype=np.uint16)
        K[:, :, :N] = self.K
        m = np.full((P, Hkv, Nc), 0xFFFF, dtype=np.uint16)
        m[..., :N] = self.mask
        Kt, Vt, q = self.Kt.copy(), self.Vt.copy(), self.q.copy()
        for b in range(B):
            nodes = T if self.nd is None else min(max(self.nd[b], 0), T)
            if self.n[b] < 0:
                nodes = 0
            first = max(self.n[b], 0)
            Kt[b, :, first + nodes:] = NAN
            Vt[b, :, first + nodes:] = NAN
            q[b, nodes:] = NAN
        self.d = dict(q=PT.to_dev_bf16(q), K=PT.to_dev_bf16(K), v=PT.to_dev_bf16(v), mask=PT.to_dev_u16(m),
                      off=torch.from_numpy(off.view(np.int32)).to(DEV), Kt=PT.to_dev_bf16(Kt),
                      Vt=PT.to_dev_bf16(Vt), n=torch.from_numpy(self.n).to(DEV),
                      nd=None if self.nd is None else torch.from_numpy(self.nd).to(DEV),
                      tree=None if self.tree is None else dev_bits(self.tree))
        self.shape = stc.make_shape(B, Hq, Hkv, D, N, G, self.v_cap, N_cap=n_cap)

    def run(self, dtype=F32, pages=None, k=None, out=None, ws=None, **other):
        d = dict(self.d, **other)
        k = k or ((self.N + 15) // 16 if pages is None else pages.shape[-1])
        need = stc.stc_tree_workspace_bytes(self.shape, self.T, k, self.cap, n_prefix=self.P)
        ws = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device=DEV) if ws is None else ws
        if out is None:
            out = torch.full((self.B, self.T, self.Hq, self.D), float("nan"), dtype=dtype, device=DEV)
        p = None if pages is None else torch.from_numpy(pages.astype(np.int32)).to(DEV)
        stc.stc_decode_attention_tree(self.shape, d["q"], d["K"], d["v"], d["mask"], d["off"], p, k, d["Kt"],
                                      d["Vt"], d["n"], self.cap, out, ws[:need], tree=d["tree"], n_draft=d["nd"],
                                      n_prefix=self.P)
        torch.cuda.synchronize()
        assert (ws[need:] == 0xFF).all()
        return out

    def want(self, pages=None, k=None):
        NP = (self.N + 15) // 16
        listed = np.tile(np.arange(k or NP), (self.P, self.Hkv, 1)) if pages is None else pages
        tree = self.tree
        if tree is not None and tree.ndim == 1:
            tree = np.tile(tree, (self.B, 1))
        return O.tree_attention_all(self.q, self.K, self.V, self.mask, listed, self.G, self.Kt, self.Vt, self.n,
                                    tree, self.nd)

    def check(self, dtype=F32, pages=None, k=None):
        got = self.run(dtype, pages, k).double().cpu().numpy()
        want, size, top, on = self.want(pages, k)
        lim = limits(want, size, top, self.N + self.cap, self.D, dtype)
        bad = ~(np.abs(got - want) <= lim) & on[:, :, None, None]
        assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], lim[bad][:4])
        assert np.isnan(got[~on]).all()                        # left as it was
        if on.any():
            off = np.linalg.norm((got - want)[on]) / max(np.linalg.norm(want[on]), 1e-30)
            assert off <= (1e-5 if dtype == F32 else 2.0 ** -8) * max(1.0, top / 50), off
        return got


# rows of a KV head on both sides of 32, 64, 128, 256, partly filled; one prefix and prefixes of their own
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("D,G", [(128, 8), (64, 4)])
@pytest.mark.parametrize("B,T,R,Hkv", [(1, 1, 1, 1), (3, 5, 2, 2), (2, 2, 16, 1), (1, 33, 1, 2), (4, 4, 4, 2),
                                       (2, 64, 1, 1), (1, 64, 2, 1), (3, 13, 7, 1), (2, 9, 16, 1), (5, 8, 7, 2)])
def test_rows(B, T, R, Hkv, D, G, each, dtype):
    Case(B, T, R * Hkv, Hkv, D, 200, G, T + 40, seed=B + T + R, each=each).check(dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,R,Hkv,N", [(9, 30, 1, 2, 700), (6, 11, 16, 1, 20001), (1, 64, 16, 1, 9000),
                                         (20, 64, 1, 4, 63)])
def test_many_rows(B, T, R, Hkv, N, D):
    Case(B, T, R * Hkv, Hkv, D, N, 8, T + 70, seed=N, n_draft=[T, 1, T - 1, 0, T + 9]).check(BF16)


def test_many_prefixes():
    """More streams than the chip has compute units in several rounds, and in one."""
    for B, T in ((40, 3), (150, 2)):
        Case(B, T, 16, 8, 64, 40, 4, 30, seed=B, each=True, n_tail=[0, 3, -1, 28, 9]).check()


# more sequences than a wavefront has lanes, some of them padding or without nodes; tails that are more than the prefix,
# so that workgroups with and without a share of the prefix take different shares of them
@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,N,cap", [(70, 5, 4, 2, 64, 90, 40), (130, 3, 6, 1, 128, 33, 70), (300, 2, 8, 8, 64, 40, 120),
                                                (65, 17, 3, 3, 64, 300, 200), (200, 1, 16, 1, 128, 600, 9)])
def test_many_sequences(B, T, Hq, Hkv, D, N, cap, each):
    n = [cap - T, 0, 5, -1, cap // 2, 31, 1, 33]
    Case(B, T, Hq, Hkv, D, N, 8, cap, seed=B, each=each, n_tail=np.minimum(n, cap - T),
         n_draft=[T, 0, max(T - 1, 1), 1, T]).check(BF16 if each else F32)
    Case(B, T, Hq, Hkv, D, N, 8, cap, seed=B + 1, each=each).check()


# up to 32 rows of 64 and more streams: their tiles in one row, cut anywhere
@pytest.mark.parametrize("D,G", [(128, 8), (64, 4)])
@pytest.mark.parametrize("N", [1, 17, 31, 33, 100, 500, 1300])
def test_few_rows_of_many_prefixes(N, D, G):
    c = Case(16, 4, 32, 4, D, N, G, 90, seed=N, each=True, n_cap=N + 7)
    c.check()
    NP = (N + 15) // 16
    rng = np.random.default_rng(N)
    for k in {1, min(2, NP), min(5, NP), NP}:
        pages = np.stack([[rng.permutation(NP)[:k] for _ in range(4)] for _ in range(16)])
        pages[3, 1, -1], pages[7, 0, 0] = NP, -1
        c.check(BF16, pages=pages)
    c.check(k=(NP + 1) // 2)


@pytest.mark.parametrize("N,T,R,Hkv,D", [(9000, 64, 16, 8, 64), (17000, 40, 4, 1, 64), (17000, 64, 16, 4, 64)])
def test_float_outputs_of_many_rows(N, T, R, Hkv, D):
    """Two and three parts of a weight, 4 and 8 wavefronts to a tile."""
    Case(1, T, R * Hkv, Hkv, D, N, 8, T + 9, seed=N + R).check()


@pytest.mark.parametrize("Hkv,T,R", [(64, 2, 4), (70, 5, 1)])
def test_few_rows_of_one_prefix_with_many_heads(Hkv, T, R):
    Case(3, T, R * Hkv, Hkv, 64, 400, 4, 50, seed=Hkv, n_draft=[T, 1, T]).check()


# lengths of the prefix that end inside a page, a tile, a group's turn, a split
@pytest.mark.parametrize("B,T,Hq,Hkv,D,each", [(2, 3, 4, 2, 128, True), (3, 6, 10, 2, 64, False), (4, 20, 5, 1, 128, False)])
@pytest.mark.parametrize("N", [1, 15, 16, 17, 31, 32, 33, 63, 65, 127, 129, 255, 257, 1000, 4001])
def test_lengths_of_the_prefix(N, B, T, Hq, Hkv, D, each):
    Case(B, T, Hq, Hkv, D, N, 8, T + 5, seed=N, each=each).check()


# tails whose nodes begin and end on both sides of tiles and pieces; no room for some nodes, or for all
@pytest.mark.parametrize("D,Hkv,R", [(128, 2, 4), (64, 1, 16), (128, 3, 1)])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64])
@pytest.mark.parametrize("cap", [64, 65, 128, 300])
def test_lengths_of_the_tails(cap, T, D, Hkv, R):
    n = [0, 1, cap - T, -1, 31, 32, 33, 63, 30, 29, cap - T + 1, cap - 1, cap, cap + 9, 96, 127]
    Case(len(n), T, R * Hkv, Hkv, D, 50, 4, cap, seed=cap + T, n_tail=n, n_draft=[T, max(T - 1, 0), T + 3]).check()


@pytest.mark.parametrize("each", [False, True])
def test_long_tails(each):
    Case(3, 7, 8, 2, 128, 33, 8, 5000, seed=1, each=each, n_tail=[4990, 17, 2304]).check()
    Case(1, 64, 16, 1, 64, 33, 8, 9000, seed=2, each=each, n_tail=[8930]).check()


# tails in hundreds of pieces, of which few or none hold tokens in some of the calls
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,Hq,Hkv,n", [(1, 1, 1, 1, [39000]), (2, 3, 4, 2, [39990, 33]), (3, 2, 5, 1, [-1, 0, 20001]),
                                          (1, 9, 16, 2, [64]), (4, 1, 2, 1, [39999, 39998, 40000, 7])])
def test_tails_in_hundreds_of_pieces(B, T, Hq, Hkv, n, D):
    cap = 40000
    Case(B, T, Hq, Hkv, D, 33, 8, cap, seed=B + T, n_tail=n, n_draft=[T, max(T - 1, 0), 1, T]).check()
    Case(B, T, Hq, Hkv, D, 70, 4, cap, seed=B + T + 1, each=True, n_tail=n).check(BF16)


@pytest.mark.parametrize("T", [1, 5, 64])
def test_a_chain_and_one_tree_for_all(T):
    c = Case(4, T, 6, 2, 128, 90, 8, 150, tree=None, seed=T)
    chain = c.check()
    ones = np.array([(2 << t) - 1 for t in range(T)], dtype=np.uint64)
    same = c.run(tree=dev_bits(ones))
    assert np.array_equal(same.cpu().numpy(), chain)
    assert np.array_equal(c.run(tree=dev_bits(np.tile(ones, (4, 1)))).cpu().numpy(), chain)
    one = random_tree(np.random.default_rng(T), 1, T)[0]
    Case(4, T, 6, 2, 128, 90, 8, 150, tree=one, seed=T).check()


@pytest.mark.parametrize("B", [1, 3])
def test_any_bits(B):
    """Sets that are no trees: nodes that see nothing (not themselves either), later nodes, nodes that are not there."""
    T = 40
    rng = np.random.default_rng(B)
    bits = rng.integers(0, 2**63, size=(B, T), dtype=np.uint64) << np.uint64(1) | rng.integers(0, 2, size=(B, T)).astype(np.uint64)
    bits[:, 3] = 0
    Case(B, T, 4, 2, 64, 70, 4, 100, tree=bits, n_draft=[T, 7, 33], seed=B).check()


def test_nothing_to_attend_gives_zeros():
    bits = np.zeros((4, 3), dtype=np.uint64)
    bits[:, 1] = 2
    c = Case(4, 3, 4, 2, 64, 40, 4, 9, n_tail=[0, 2, 0, -1], tree=bits, n_draft=[3, 3, 1, 3])
    out = torch.full((4, 3, 4, 64), 3.0, device=DEV)
    pages = np.full((1, 2, 2), -1)
    c.run(pages=pages, out=out)
    assert (out[0, [0, 2]] == 0).all() and out[0, 1].any() and out[1].ne(0).any(-1).all()
    assert (out[2, 0] == 0).all() and (out[2, 1:] == 3).all() and (out[3] == 3).all()
    c.check(pages=pages)


@pytest.mark.parametrize("each", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_page_lists(D, each):
    rng = np.random.default_rng(D)
    c = Case(3, 9, 6, 2, D, 1000 - 5, 4, 30, n_cap=1040, each=each, seed=D)
    for k in (1, 2, 5, 63):
        pages = np.stack([[rng.permutation(63)[:k] for _ in range(2)] for _ in range(c.P)])
        c.check(pages=pages)
        pages[0, 0, 0], pages[-1, 1, -1] = -1, 63
        if k > 2:
            pages[0, 1, 1], pages[-1, 0, 2] = 2**31 - 1, -2**31
        c.check(pages=pages)
    c.check(k=7)


@pytest.mark.parametrize("G,D", [(1, 64), (2, 64), (16, 128), (4, 128)])
def test_value_groups(G, D):
    Case(2, 6, 4, 2, D, 150, G, 15, seed=G, each=True).check()


def test_values_behind_the_capacity_count_as_dropped():
    c = Case(2, 6, 4, 2, 128, 90, 8, 15, v_cap=100)
    kept = ((c.mask[..., None].astype(np.int64) >> np.arange(8)) & 1).reshape(1, 2, -1)
    kept *= kept.cumsum(-1) <= 100
    c.mask = (kept.reshape(1, 2, 90, 8) << np.arange(8)).sum(-1).astype(np.uint16)
    c.check()


def test_infinities_and_nan_of_nodes_reach_those_that_see_them():
    """In keys and values, of nodes that other nodes of the sequence do not see, next to what all see."""
    for D, n in ((128, [5, 30, 64]), (64, [0, 33, 90])):
        T, B = 20, 3
        c = Case(B, T, 6, 2, D, 70, 4, 120, n_tail=n, seed=D)
        clean = c.run()
        want, size, top, on = c.want()
        Kt, Vt = c.Kt.copy(), c.Vt.copy()
        hit = np.zeros((B, T), dtype=bool)                     # nodes that see a node with bad values
        for b in range(B):
            for t, val in ((4, 0x7F80), (9, 0xFF80), (13, NAN)):
                Vt[b, :, n[b] + t, 7:D - 3] = val
                hit[b] |= (c.tree[b] >> np.uint64(t) & np.uint64(1)).astype(bool)
            Kt[b, :, n[b] + 17, 5] = NAN
            hit_k = (c.tree[b] >> np.uint64(17) & np.uint64(1)).astype(bool)
            got = c.run(Kt=PT.to_dev_bf16(Kt), Vt=PT.to_dev_bf16(Vt))
            other = torch.from_numpy(~(hit[b] | hit_k)).to(DEV)
            assert other.any() and torch.equal(got[b][other], clean[b][other])
            seen = torch.from_numpy(hit[b] & ~hit_k).to(DEV)
            assert seen.any() and not torch.isfinite(got[b][seen][..., 7:D - 3]).any()
            assert torch.equal(got[b][seen][..., :7], clean[b][seen][..., :7])
            assert torch.equal(got[b][seen][..., D - 3:], clean[b][seen][..., D - 3:])
            assert got[b][torch.from_numpy(hit_k).to(DEV)].isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_and_ordered_scores(dtype):
    for scale in (0.01, 8.0, 60.0):
        Case(3, 9, 8, 2, 128, 700, 8, 90, scale=scale, seed=int(scale)).check(dtype)


def test_a_node_alone_is_a_step():
    """T = 1 over a prefix for all, the token's row appended: the shared step's results."""
    c = Case(7, 1, 8, 2, 128, 500, 8, 60, tree=None, n_tail=[0, 59, 3, -1, 32, 31, 7])
    c.check()
    n1 = torch.where(c.d["n"] >= 0, c.d["n"] + 1, -1)
    out = torch.zeros(7, 8, 128, device=DEV)
    NP = 32
    ws = torch.empty(stc.stc_shared_workspace_bytes(c.shape, NP, 60), dtype=torch.uint8, device=DEV)
    stc.stc_decode_attention_shared(c.shape, c.d["q"], c.d["K"][0], c.d["v"][0], c.d["mask"][0], c.d["off"][0], None,
                                    NP, c.d["Kt"], c.d["Vt"], n1, 60, out, ws)
    want, size, top, on = c.want()
    lim = limits(want, size, top, 560, 128, F32)
    assert (np.abs(out.double().cpu().numpy() - want[:, 0]) <= lim[:, 0])[on[:, 0]].all()


@pytest.mark.parametrize("each", [False, True])
def test_a_sequence_depends_on_itself_alone(each):
    """Other sequences' lengths, trees and counts change where sums are cut, so roundings, and nothing else."""
    c = Case(6, 12, 8, 2, 128, 300, 8, 200, each=each, n_tail=[50, 0, 150, 7, 188, 30])
    a = c.run()
    n = torch.tensor([50, 188, -1, 0, 3, 30], dtype=torch.int32, device=DEV)
    nd = torch.tensor([12, 1, 5, 0, 12, 12], dtype=torch.int32, device=DEV)
    Kt, Vt = (torch.nan_to_num(c.d[x], nan=1.0) for x in ("Kt", "Vt"))
    tree = c.d["tree"].clone()
    tree[1] = 0
    b = c.run(n=n, nd=nd, tree=tree, Kt=Kt, Vt=Vt, q=torch.nan_to_num(c.d["q"], nan=1.0))
    want, size, top, on = c.want()
    lim = limits(want, size, top, 500, 128, F32)
    for x in (a, b):
        assert (np.abs(x.double().cpu().numpy() - want) <= lim)[[0, 5]].all()


def test_graph_with_lengths_that_change():
    """Two captured graphs with a workspace each, replayed in turn with other lengths, trees and eager work."""
    cs = [Case(4, 6, 8, 2, 128, 400, 8, 100, seed=s, n_tail=[0, 50, 94, 31]) for s in (1, 2)]
    runs = []
    for c in cs:
        need = stc.stc_tree_workspace_bytes(c.shape, 6, 25, 100)
        out = torch.zeros(4, 6, 8, 128, device=DEV)
        ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        d = {k: torch.nan_to_num(x, nan=0.5) if x is not None and x.dtype == BF16 else x for k, x in c.d.items()}
        nd = torch.full((4,), 6, dtype=torch.int32, device=DEV)

        def call(out=out, ws=ws, d=d, nd=nd, c=c):
            stc.stc_decode_attention_tree(c.shape, d["q"], d["K"], d["v"], d["mask"], d["off"], None, 25, d["Kt"],
                                          d["Vt"], d["n"], 100, out, ws, tree=d["tree"], n_draft=nd)
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        runs.append((g, call, out, d, nd))
    rng = np.random.default_rng(0)
    for turn in range(4):
        for g, call, out, d, nd in runs:
            d["n"].copy_(torch.from_numpy(rng.integers(-1, 95, size=4).astype(np.int32)))
            nd.copy_(torch.from_numpy(rng.integers(0, 7, size=4).astype(np.int32)))
            d["tree"].copy_(dev_bits(random_tree(rng, 4, 6)))
            out.fill_(7)
            g.replay()
            torch.cuda.synchronize()
            got = out.clone()
            out.fill_(7)
            call()
            torch.cuda.synchronize()
            assert torch.equal(got, out), turn


def test_on_a_stream_of_its_own():
    c = Case(3, 5, 8, 2, 128, 300, 8, 60)
    want = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = c.run()
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("change,error", [
    (dict(q=lambda d: d["q"][:, :2]), ValueError), (dict(K=lambda d: d["K"].expand(3, -1, -1, -1).contiguous()), ValueError),
    (dict(mask=lambda d: d["mask"][..., :-1].contiguous()), ValueError), (dict(Kt=lambda d: d["Kt"][:, :, 1:].contiguous()), ValueError),
    (dict(Vt=lambda d: d["Vt"][:2]), ValueError), (dict(n=lambda d: d["n"][:2]), ValueError),
    (dict(n=lambda d: d["n"].long()), TypeError), (dict(tree=lambda d: d["tree"][:, :4].contiguous()), ValueError),
    (dict(tree=lambda d: d["tree"].int()), TypeError), (dict(nd=lambda d: d["n"][:1]), ValueError),
    (dict(q=lambda d: d["q"].float()), TypeError), (dict(Kt=lambda d: d["Kt"].transpose(1, 2)), ValueError),
    (dict(n=lambda d: d["n"].cpu()), TypeError), (dict(Kt=lambda d: None), ValueError)])
def test_tensors_that_do_not_fit(change, error):
    c = Case(3, 5, 8, 2, 128, 40, 8, 60)
    if "q" in change and error is ValueError:        # (as if the call had 5 nodes: out and tree say so)
        with pytest.raises(ValueError):
            c.run(q=change["q"](c.d).contiguous())
        return
    with pytest.raises(error):
        c.run(**{k: f(c.d) for k, f in change.items()})
