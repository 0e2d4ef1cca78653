"""Decode attention of a batch over one shared prefix, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2604_21335_amd as stc
from oracle import stc_oracle as O
from tests import parity as PT
from tests.helpers import bits_to_f64, randn_bf16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def limits(want, size, top, tokens, D, dtype):
    """How far an output may be off, from the arithmetic.  e: relative error of a weight.  Two bf16
    parts leave 2^-16 of it, one leaves 2^-8 (half a step of the last part, relative); the exponent is
    a float dot product of D terms, scaled and shifted in base 2, off by at most (D + 4) 2^-24 of the
    sum of magnitudes behind it, which shifts the weight by as much; the exponential itself by 2^-22.
    Weighted sum and sum of weights each carry e and the roundings of at most `tokens` additions."""
    e = (2.0 ** -16 if dtype == F32 else 2.0 ** -8) + (D + 4) * 2.0 ** -24 * max(top, 1.0) + 2.0 ** -22
    lim = (2 * e + (tokens + 64) * 2.0 ** -24) * size
    return lim + (2.0 ** -8 * (np.abs(want) + lim) if dtype == BF16 else 0) + 1e-30


class Case:
    """Host arrays of a prefix and B tails, and their device copies; everything that must not be read
    holds NaN."""

    def __init__(self, B, Hq, Hkv, D, N, G, cap, seed=0, n_tail=None, n_cap=0, scale=1.0, keep=None,
                 v_cap=None):
        rng = np.random.default_rng(seed)
        self.B, self.Hq, self.Hkv, self.D, self.N, self.G, self.cap = B, Hq, Hkv, D, N, G, cap
        self.q = randn_bf16(rng, (B, Hq, D), scale)
        self.K, self.V = randn_bf16(rng, (Hkv, N, D)), randn_bf16(rng, (Hkv, N, D))
        self.mask = rng.integers(0, 1 << G, size=(Hkv, N)).astype(np.uint16)
        if keep is not None:
            self.mask[:] = keep
        self.Kt, self.Vt = (randn_bf16(rng, (B, Hkv, max(cap, 1), D)) for _ in range(2))
        self.n = rng.integers(0, cap + 1, size=B) if n_tail is None else np.resize(n_tail, B)
        self.n = self.n.astype(np.int32)
        Nc = n_cap or N
        off = np.zeros((Hkv, Nc + 1), dtype=np.uint32)
        kept = ((self.mask[..., None].astype(np.int64) >> np.arange(G)) & 1).sum(-1)
        off[:, 1:N + 1] = kept.cumsum(1)
        off[:, N + 1:] = 0xFFFFFFF0                  # past the end: never used
        self.v_cap = v_cap or max(int(off[:, N].max()), 1) + 3
        v = np.full((Hkv, self.v_cap, D // G), 0x7FC0, dtype=np.uint16)
        for h in range(Hkv):
            packed = O.pack_values(self.V[h], self.mask[h], off[h, :N + 1], G)[:self.v_cap]
            v[h, :len(packed)] = packed
        K = np.full((Hkv, Nc, D), 0x7FC0, dtype=np.uint16)
        K[:, :N] = self.K
        m = np.full((Hkv, Nc), 0xFFFF, dtype=np.uint16)
        m[:, :N] = self.mask
        Kt, Vt = self.Kt.copy(), self.Vt.copy()
        for b in range(B):
            Kt[b, :, max(self.n[b], 0):] = 0x7FC0
            Vt[b, :, max(self.n[b], 0):] = 0x7FC0
        self.d = dict(q=PT.to_dev_bf16(self.q), K=PT.to_dev_bf16(K), v=PT.to_dev_bf16(v),
                      mask=PT.to_dev_u16(m), off=torch.from_numpy(off.view(np.int32)).to(DEV),
                      Kt=PT.to_dev_bf16(Kt) if cap else None, Vt=PT.to_dev_bf16(Vt) if cap else None,
                      n=torch.from_numpy(self.n).to(DEV))
        self.shape = stc.make_shape(B, Hq, Hkv, D, N, G, self.v_cap, N_cap=n_cap)

    def run(self, dtype=F32, pages=None, out=None, k=None, **other):
        d = dict(self.d, **other)
        k = k or ((self.N + 15) // 16 if pages is None else pages.shape[1])
        need = stc.stc_shared_workspace_bytes(self.shape, k, self.cap)
        ws = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device=DEV)       # NaN
        if out is None:
            out = torch.full((self.B, self.Hq, self.D), float("nan"), dtype=dtype, device=DEV)
        p = None if pages is None else torch.from_numpy(pages.astype(np.int32)).to(DEV)
        stc.stc_decode_attention_shared(self.shape, d["q"], d["K"], d["v"], d["mask"], d["off"], p, k,
                                        d["Kt"], d["Vt"], d["n"], self.cap, out, ws[:need])
        torch.cuda.synchronize()
        assert (ws[need:] == 0xFF).all()
        return out

    def check(self, dtype=F32, pages=None, k=None):
        got = self.run(dtype, pages, k=k).double().cpu().numpy()
        listed = pages if pages is not None or k is None else np.tile(np.arange(k), (self.Hkv, 1))
        want, size, top = O.shared_attention_all(self.q, self.K, self.V, self.mask, listed, self.G,
                                                 self.Kt if self.cap else None, self.Vt, self.n)
        on = self.n >= 0
        lim = limits(want, size, top, self.N + self.cap, self.D, dtype)
        bad = ~(np.abs(got - want) <= lim) & on[:, None, None]
        assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], lim[bad][:4])
        # errors of different weights are independent, so the whole is far closer than the worst case
        off = np.linalg.norm((got - want)[on]) / max(np.linalg.norm(want[on]), 1e-30)
        assert off <= (1e-5 if dtype == F32 else 2.0 ** -8) * max(1.0, top / 50), off
        return got


# rows of a KV head on both sides of 32, 64 (other forms) and 128 (more blocks of rows), partly filled
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,G", [(128, 8), (64, 4)])
@pytest.mark.parametrize("B,R,Hkv", [(1, 1, 1), (3, 5, 2), (2, 16, 1), (33, 1, 2), (4, 16, 2), (13, 5, 1),
                                     (16, 7, 2), (128, 1, 1), (43, 3, 2), (19, 16, 1)])
def test_rows(B, R, Hkv, D, G, dtype):
    Case(B, R * Hkv, Hkv, D, 200, G, 40, seed=B + R).check(dtype)


# many rows beside tails that are long together: 8 wavefronts to a tile
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,R,Hkv,cap,N", [(129, 1, 4, 210, 63), (300, 1, 4, 90, 700), (33, 16, 4, 800, 129),
                                           (90, 5, 8, 150, 1), (150, 2, 4, 180, 2001)])
def test_wide_tiles(B, R, Hkv, cap, N, D, dtype):
    Case(B, R * Hkv, Hkv, D, N, 8, cap, seed=N, n_tail=[0, 3, cap, -1, 40]).check(dtype)
    c = Case(B, R * Hkv, Hkv, D, N, 4, cap, seed=N + 1, n_tail=[0, 1, -1, 9], n_cap=N + 20)
    NP = (N + 15) // 16
    pages = np.stack([np.random.default_rng(h).permutation(NP) for h in range(Hkv)])
    pages[0, -1] = NP
    c.check(dtype, pages=pages)


# tokens that end inside a page, a tile, a group's turn, a split
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,Hq,Hkv,D", [(2, 4, 2, 128), (9, 10, 2, 64), (40, 5, 1, 128)])
@pytest.mark.parametrize("N", [1, 15, 16, 17, 31, 32, 33, 63, 65, 127, 128, 129, 255, 257, 1000, 4001])
def test_lengths_of_the_prefix(N, B, Hq, Hkv, D, dtype):
    Case(B, Hq, Hkv, D, N, 8, 5, seed=N).check(dtype)


@pytest.mark.parametrize("D,Hkv,R,B", [(128, 2, 4, 8), (64, 1, 16, 11), (128, 3, 1, 70)])
@pytest.mark.parametrize("cap", [0, 1, 2, 31, 33, 128, 129, 700])
def test_lengths_of_the_tails(cap, D, Hkv, R, B):
    n = [0, cap, 1, cap // 2, cap - 1, 2 * cap + 5, -1, 31, 32, 33, 127, 128, 129]
    Case(B, R * Hkv, Hkv, D, 50, 4, cap, seed=cap, n_tail=np.minimum(n, cap + 7)).check()


@pytest.mark.parametrize("G,D", [(1, 64), (1, 128), (2, 64), (8, 64), (16, 128), (4, 128)])
@pytest.mark.parametrize("B", [2, 50])
def test_value_groups(G, D, B):
    Case(B, 4, 2, D, 150, G, 9, seed=G).check()


@pytest.mark.parametrize("keep", [0, 0xFF, 1, 0x80])
def test_tokens_that_keep_nothing_or_all(keep):
    got = Case(5, 4, 2, 128, 90, 8, 0, keep=keep).check()
    if keep == 0:
        assert (got == 0).all()


def test_values_behind_the_capacity_count_as_dropped():
    c = Case(6, 4, 2, 128, 90, 8, 4, keep=0xFF, v_cap=300)
    c.mask[:, 37] = 0x0F                                       # 300 slots: tokens 0 .. 36, half of 37
    c.mask[:, 38:] = 0
    c.check()


@pytest.mark.parametrize("B", [2, 30, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_page_lists(B, D):
    """Pages in any order, the ragged last one among them, entries outside the prefix skipped."""
    rng = np.random.default_rng(B)
    c = Case(B, 6, 2, D, 1000 - 5, 4, 20, n_cap=1040, seed=B)
    for k in (1, 2, 5, 63):
        pages = np.stack([rng.permutation(63)[:k] for _ in range(2)])
        c.check(pages=pages)
        pages[0, 0], pages[1, -1] = -1, 63
        if k > 2:
            pages[1, 1] = 2**31 - 1
            pages[0, 2] = -2**31
        c.check(pages=pages)
    c.check(k=7)                                               # no list: the first pages


def test_nothing_to_attend_gives_zeros():
    c = Case(4, 4, 2, 64, 40, 4, 6, n_tail=[0, 2, 0, -1])
    out = torch.full((4, 4, 64), 3.0, device=DEV)
    pages = np.full((2, 2), -1)
    c.run(pages=pages, out=out)
    assert (out[0] == 0).all() and (out[2] == 0).all() and (out[3] == 3).all()
    assert c.check(pages=pages)[1].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_padding_is_left_as_it_was(dtype):
    c = Case(70, 4, 2, 128, 100, 8, 12, n_tail=[3, -1, 0, -2**31, 12])
    out = torch.full((70, 4, 128), 3.0, dtype=dtype, device=DEV)
    c.run(dtype, out=out)
    on = torch.from_numpy(c.n >= 0)
    assert (out[~on] == 3).all() and not (out[on] == 3).all(-1).any()
    # lengths may be given without tails, to mark padding
    c = Case(5, 4, 2, 128, 100, 8, 0, n_tail=[0, -1, 0, -1, 0])
    out = torch.full((5, 4, 128), 3.0, device=DEV)
    c.run(out=out)
    assert (out[[1, 3]] == 3).all() and not (out[[0, 2, 4]] == 3).all(-1).any()
    every = c.run(n=None)
    assert torch.equal(every[[0, 2, 4]], out[[0, 2, 4]]) and not every.isnan().any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B", [3, 40])
def test_large_and_ordered_scores(B, dtype):
    """Weights on one token, maxima that grow from tile to tile or fall, and by less than what moves
    the running maximum."""
    Case(B, 4, 2, 128, 300, 8, 30, scale=60.0).check(dtype)
    for slope in (-1.0, -0.01, 0.01, 1.0):
        c = Case(B, 4, 2, 128, 300, 8, 30)
        ramp = np.linspace(-150 * slope, 150 * slope, 300)
        K = bits_to_f64(c.K)
        K[..., 0] = ramp
        q = bits_to_f64(c.q)
        q[..., 0] = 11.0
        from tests.helpers import f32_to_bf16_bits
        c.K, c.q = f32_to_bf16_bits(K), f32_to_bf16_bits(q)
        c.d["K"], c.d["q"] = PT.to_dev_bf16(c.K), PT.to_dev_bf16(c.q)
        c.check(dtype)


def test_a_sequence_does_not_depend_on_the_others():
    c = Case(40, 7, 1, 128, 500, 8, 50, seed=3)
    a = c.run()
    order = torch.from_numpy(np.random.default_rng(0).permutation(40)).to(DEV)
    q, Kt, Vt, n = (c.d[x][order].contiguous() for x in ("q", "Kt", "Vt", "n"))
    b = c.run(q=q, Kt=Kt, Vt=Vt, n=n)
    assert torch.equal(a[order], b)
    q[1:] *= 30
    n[1:] = 0
    assert torch.equal(c.run(q=q, Kt=Kt, Vt=Vt, n=n)[0], b[0])
    assert torch.equal(c.run(), a)


def test_agrees_with_a_cache_for_every_sequence():
    """stc_decode_attention_tail over copies of the prefix, tails of one length."""
    B, Hq, Hkv, D, N, G, n = 6, 8, 2, 128, 333, 8, 21
    c = Case(B, Hq, Hkv, D, N, G, n, n_tail=[n])
    s = stc.make_shape(B, Hq, Hkv, D, N, G, c.v_cap)
    rep = lambda t: t[None].expand(B, *t.shape).contiguous()  # noqa: E731
    NP = (N + 15) // 16
    ws = torch.empty(max(16, stc.stc_workspace_bytes(s, stc.STC_WS_ATTENTION_TAIL, NP + 2)),
                     dtype=torch.uint8, device=DEV)
    out = torch.empty(B, Hq, D, device=DEV)
    stc.stc_decode_attention_tail(s, c.d["q"], rep(c.d["K"]), rep(c.d["v"]), rep(c.d["mask"]),
                                  rep(c.d["off"]), None, NP, c.d["Kt"], c.d["Vt"], n, n, out, ws)
    # either is within 2e-5 of the sums on such data
    assert (c.run() - out).abs().max() <= 4e-5


def test_offsets_that_pass_32_bits():
    """A prefix whose keys and values pass 4 GiB, attended at both ends; tails too."""
    N, D = (1 << 32) // 256 + 4096, 128
    K = torch.zeros(1, N, D, dtype=BF16, device=DEV)
    v = torch.zeros(1, N, D, dtype=BF16, device=DEV)
    mask = torch.ones(1, N, dtype=torch.int16, device=DEV)
    off = torch.arange(N + 1, dtype=torch.int32, device=DEV)[None]
    NP = N // 16
    pages = [0, 1, NP - 3, NP - 1, NP // 2]
    rng = np.random.default_rng(4)
    small = Case(40, 2, 1, D, 80, 1, 0, keep=1, n_tail=[0])
    for i, p in enumerate(pages):
        K[0, p * 16:p * 16 + 16] = small.d["K"][0, i * 16:i * 16 + 16]
        v[0, p * 16:p * 16 + 16] = small.d["v"][0, i * 16:i * 16 + 16]
    s = stc.make_shape(40, 2, 1, D, N, 1, N)
    idx = torch.tensor([pages], dtype=torch.int32, device=DEV)
    want, size, top = O.shared_attention_all(small.q, small.K, small.V, small.mask, None, 1, None, None,
                                             small.n)
    for B in (40, 3):                                   # both forms
        s.B = B
        ws = torch.empty(stc.stc_shared_workspace_bytes(s, 5, 0) + 16, dtype=torch.uint8, device=DEV)
        out = torch.empty(B, 2, D, device=DEV)
        stc.stc_decode_attention_shared(s, small.d["q"][:B].contiguous(), K, v, mask, off, idx, 5, None, None,
                                        None, 0, out, ws)
        got = out.double().cpu().numpy()
        assert (np.abs(got - want[:B]) <= limits(want, size, top, 80, D, F32)[:B]).all()
    # the last tail of a batch starts behind 4 GiB of others
    cap = 1 << 19
    Kt = torch.zeros(34, 1, cap, D, dtype=BF16, device=DEV)
    Vt = torch.zeros(34, 1, cap, D, dtype=BF16, device=DEV)
    n = torch.zeros(34, dtype=torch.int32, device=DEV)
    tail = randn_bf16(rng, (1, 1, 50, D))
    Kt[33, 0, :50] = Vt[33, 0, :50] = PT.to_dev_bf16(tail)[0, 0]
    n[33] = 50
    c = Case(34, 2, 1, D, 20, 1, 0, keep=1)
    s = stc.make_shape(34, 2, 1, D, 20, 1, c.v_cap)
    ws = torch.empty(stc.stc_shared_workspace_bytes(s, 2, cap) + 16, dtype=torch.uint8, device=DEV)
    out = torch.empty(34, 2, D, device=DEV)
    stc.stc_decode_attention_shared(s, c.d["q"], c.d["K"], c.d["v"], c.d["mask"], c.d["off"], None, 2, Kt, Vt,
                                    n, cap, out, ws)
    tails = np.repeat(tail, 34, axis=0)
    want, size, top = O.shared_attention_all(c.q, c.K, c.V, c.mask, None, 1, tails, tails, [0] * 33 + [50])
    assert (np.abs(out.double().cpu().numpy() - want) <= limits(want, size, top, 70, D, F32)).all()


def _prefix(N=200, k_pages=16, Hq=8, Hkv=2, D=128, G=8, rotary=None, n_cap=0):
    g = torch.Generator(device=DEV).manual_seed(11)
    c = stc.RoutedCache(1, Hq, Hkv, D, N, G, k_pages, device=DEV, n_cap=n_cap)
    K = torch.randn(1, Hkv, N, D, device=DEV, generator=g).bfloat16()
    V = torch.randn(1, Hkv, N, D, device=DEV, generator=g).bfloat16()
    m = torch.randint(0, 1 << G, (1, Hkv, N), device=DEV, generator=g).to(torch.int16)
    c.build(K, V, mask_in=m, rotary=rotary)
    return c, K, V, m


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B", [3, 20])
def test_a_run_of_steps(B, dtype):
    """Construction with rotary keys, then tokens appended and attended, against the oracle on the
    positions, keys and values themselves; a padded element; tails that differ and fill up."""
    N, Hq, Hkv, D, G, cap, steps = 200, 8, 2, 128, 8, 12, 9
    rot = stc.Rotary(64, stc.STC_ROTARY_INTERLEAVED, base=1e5, device=DEV)
    c, K, V, m = _prefix(N, rotary=rot, n_cap=208)
    b = stc.SharedPrefix(c, B, cap, rotary=rot, out_dtype=dtype)
    start = np.arange(B) % 5
    start[-1] = -1
    b.n_tail.copy_(torch.from_numpy(start.astype(np.int32)))
    b.K_tail.zero_(), b.V_tail.zero_()
    g = torch.Generator(device=DEV).manual_seed(2)
    turns = rot.turns.cpu().numpy()
    host = lambda t: bits_to_f64(PT.host_bf16(t))  # noqa: E731
    Kt, Vt = np.zeros((2, B, Hkv, cap, D), dtype=np.uint16)
    for i in range(steps):
        x = torch.randn(B, Hq + 2 * Hkv, D, device=DEV, generator=g).bfloat16()
        out = b.step(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
        n = start + i
        on = (start >= 0) & (n < cap)
        e = np.nonzero(on)[0]
        want_k = O.rotary(host(x[:, Hq:Hq + Hkv]), N + n[:, None], turns, 64, True)
        got_k = host(b.K_tail)
        assert np.abs(got_k[e, :, n[e]] - want_k[e]).max() <= 2.0 ** -8 * 6      # |k| < 6
        Kt[e, :, n[e]] = PT.host_bf16(b.K_tail)[e, :, n[e]]
        Vt[e, :, n[e]] = PT.host_bf16(x[:, Hq + Hkv:])[e]
        assert np.array_equal(PT.host_bf16(b.V_tail), Vt) and np.array_equal(PT.host_bf16(b.K_tail), Kt)
        want, size, top = O.shared_attention_all(
            PT.host_bf16(b.q), PT.host_bf16(c.K)[0, :, :N], PT.host_bf16(V)[0], PT.host_u16(m)[0], None, G,
            Kt, Vt, n + 1)
        lim = limits(want, size, top, N + cap, D, dtype)
        ok = np.abs(out.double().cpu().numpy() - want) <= lim
        assert ok[start >= 0].all()
    assert b.dev_status.item() == int((start + steps - 1 >= cap).any())
    assert (out[-1] == 0).all()                                 # padding: as allocated


def test_tails_go_on_where_the_prefix_ends():
    """Positions behind a prefix that starts somewhere else, has grown, or whose positions were given."""
    N, B, Hq, Hkv, D, cap = 200, 3, 8, 2, 128, 6
    rot = stc.Rotary(128, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(5)
    K = torch.randn(1, Hkv, N, D, device=DEV, generator=g).bfloat16()
    m = torch.full((1, Hkv, N), 0xFF, dtype=torch.int16, device=DEV)
    x = torch.randn(B, Hq + 2 * Hkv, D, device=DEV, generator=g).bfloat16()
    parts = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    c = stc.RoutedCache(1, Hq, Hkv, D, N, 8, 16, device=DEV, n_cap=224, tail_cap=8)

    def first(pos, given=None, **kw):
        """Queries and tails' first keys, which have to stand at positions pos."""
        b = stc.SharedPrefix(c, B, cap, rotary=rot, **kw)
        b.append(*parts, pos=given)
        want = torch.empty(B, Hq + Hkv, 1, D, dtype=torch.bfloat16, device=DEV)
        rot.apply(x[:, :Hq + Hkv, None], want, pos=torch.tensor(pos, dtype=torch.int32, device=DEV)[:, None])
        assert torch.equal(b.q, want[:, :Hq, 0]) and torch.equal(b.K_tail[:, :, 0], want[:, Hq:, 0])
    c.build(K, K, mask_in=m, rotary=rot)
    first([N] * B)
    c.build(K, K, mask_in=m, rotary=rot, pos0=1000)
    first([1000 + N] * B)
    first([7] * B, pos0=7)
    first([3, 900, -2], given=torch.tensor([3, 900, -2], dtype=torch.int32, device=DEV))
    c.append(K[:, :, 0].contiguous(), K[:, :, 0].contiguous())
    c.flush(1, mask_in=m[:, :, :1].contiguous())
    first([1000 + N + 1] * B)
    c = stc.RoutedCache(1, Hq, Hkv, D, N, 8, 16, device=DEV, n_cap=224)
    c.build(K, K, mask_in=m, rotary=rot, pos=torch.arange(N, dtype=torch.int32, device=DEV)[None] * 2)
    with pytest.raises(ValueError):
        first([N] * B)
    first([2 * N] * B, pos0=2 * N)
    first([3, 900, -2], given=torch.tensor([3, 900, -2], dtype=torch.int32, device=DEV))
    stc.SharedPrefix(c, B, cap).append(*parts)                 # keys that have their positions
    c.build(K, K, mask_in=m, pos0=50)
    first([50 + N] * B)


def test_a_full_tail_repeats_its_last_answer_and_says_so():
    c, *_ = _prefix()
    b = stc.SharedPrefix(c, 3, 2, rotary=stc.Rotary(128, device=DEV))
    b.n_tail.copy_(torch.tensor([0, 1, -1], dtype=torch.int32))
    b.K_tail.zero_(), b.V_tail.zero_()
    g = torch.Generator(device=DEV).manual_seed(8)
    before = None
    for full in (0, 1, 1):
        x = torch.randn(3, 12, 128, device=DEV, generator=g).bfloat16()
        out = b.step(x[:, :8], x[:, 8:10], x[:, 10:]).clone()
        assert b.dev_status.item() == full
        if full:
            assert torch.equal(out[1], before[1]) and torch.equal(b.K_tail[1], keys[1])
        before, keys = out, b.K_tail.clone()
    assert b.n_tail.tolist() == [2, 2, -1]
    b.dev_status.zero_()
    b.n_tail[:2] = 0
    out = b.step(x[:, :8], x[:, 8:10], x[:, 10:])
    assert b.dev_status.item() == 0 and not torch.equal(out[1], before[1])


def test_steps_captured_and_replayed():
    """One graph of a step, replayed as the tails grow, with eager work between the replays."""
    B, cap = 5, 40
    c, *_ = _prefix()
    rot = stc.Rotary(128, device=DEV)
    a, b = (stc.SharedPrefix(c, B, cap, rotary=rot) for _ in range(2))
    for s in (a, b):
        s.K_tail.zero_(), s.V_tail.zero_()
        s.n_tail.copy_(torch.tensor([0, 3, 7, -1, 30], dtype=torch.int32))
    x = torch.randn(B, 12, 128, device=DEV).bfloat16()
    warm = stc.SharedPrefix(c, B, cap, rotary=rot)
    warm.step(x[:, :8], x[:, 8:10], x[:, 10:])                  # LDS limits are raised by a first call
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(x[:, :8], x[:, 8:10], x[:, 10:])
    for i in range(14):
        x.copy_(torch.randn(B, 12, 128, device=DEV))
        graph.replay()
        b.step(x[:, :8], x[:, 8:10], x[:, 10:])
        torch.cuda.synchronize()
        assert torch.equal(a.out, b.out) and torch.equal(a.K_tail, b.K_tail) and torch.equal(a.n_tail, b.n_tail)
    assert a.n_tail.tolist() == [14, 17, 21, -1, 40] and a.dev_status.item() == 1


def test_two_calls_at_once():
    c = Case(40, 7, 1, 128, 700, 8, 30)
    d = Case(3, 8, 2, 64, 900, 4, 60)
    want = c.run(), d.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [None, None]
    outs = [torch.empty(40, 7, 128, device=DEV), torch.empty(3, 8, 64, device=DEV)]
    wss = [torch.empty(stc.stc_shared_workspace_bytes(x.shape, (x.N + 15) // 16, x.cap) + 16, dtype=torch.uint8,
                       device=DEV) for x in (c, d)]
    for _ in range(5):
        for i, (x, st) in enumerate(((c, torch.cuda.current_stream()), (d, side))):
            with torch.cuda.stream(st):
                e = x.d
                stc.stc_decode_attention_shared(x.shape, e["q"], e["K"], e["v"], e["mask"], e["off"], None,
                                                (x.N + 15) // 16, e["Kt"], e["Vt"], e["n"], x.cap, outs[i], wss[i])
    torch.cuda.synchronize()
    got = outs
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_selected_pages_of_the_prefix():
    """Pages from stc_select_pages for one query, attended by a batch."""
    c, *_ = _prefix(N=1500, k_pages=20)
    q = torch.randn(6, 8, 128, device=DEV).bfloat16()
    c.select(q[:1])
    b = stc.SharedPrefix(c, 6, 4)
    out = b.attend(q, c.page_idx[0].contiguous())
    c.attend(q[:1].contiguous())
    assert (out[:1] - c.out).abs().max() <= 4e-5


def test_pages_that_any_of_some_queries_selected():
    """The lists of several sequences' queries, merged by stc_union_pages as if they were heads of one
    sequence, attended by all of them: the pages of the union and no others."""
    n, k, Hkv = 6, 20, 2
    c, *_ = _prefix(N=1500, k_pages=k)
    q = torch.randn(n, 8, 128, device=DEV).bfloat16()
    lists = []
    for i in range(n):
        c.select(q[i:i + 1].contiguous())
        lists.append(c.page_idx[0].clone())
    lists = torch.stack(lists, 1).reshape(1, Hkv * n, k).contiguous()
    cap = min(c.NP, n * k)
    pages = torch.empty(1, Hkv, cap, dtype=torch.int32, device=DEV)
    heads = torch.empty(1, Hkv, cap, dtype=torch.int16, device=DEV)
    stc.stc_union_pages(stc.make_shape(1, Hkv * n, Hkv, 128, 1500, 8, 1), lists, k, pages, heads)
    b = stc.SharedPrefix(c, n, 4)
    got = b.attend(q, pages[0]).clone()
    for h in range(Hkv):
        union = torch.unique(lists[0, h * n:(h + 1) * n])
        assert k < len(union) < cap and pages[0, h, :len(union)].tolist() == union.tolist()
        assert (pages[0, h, len(union):] == -1).all()
        alone = torch.full((Hkv, cap), -1, dtype=torch.int32, device=DEV)
        alone[h, :len(union)] = union.flip(0)                  # another order, the other KV head without pages
        want = b.attend(q, alone)
        assert (got[:, h * 4:h * 4 + 4] - want[:, h * 4:h * 4 + 4]).abs().max() <= 4e-5


def test_tensors_of_another_shape_or_type_are_refused():
    c = Case(2, 4, 2, 64, 40, 4, 6)
    d = c.d
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    out = torch.empty(2, 4, 64, device=DEV)
    ok = [c.shape, d["q"], d["K"], d["v"], d["mask"], d["off"], None, 3, d["Kt"], d["Vt"], d["n"], 6, out, ws]
    stc.stc_decode_attention_shared(*ok)
    short = lambda t: t[..., :-1].contiguous()  # noqa: E731
    for i in (1, 2, 3, 4, 5, 8, 9, 10, 12):
        with pytest.raises(ValueError):
            stc.stc_decode_attention_shared(*ok[:i], short(ok[i]), *ok[i + 1:])
    for i in (1, 2, 3, 4, 5, 8, 9, 10, 12):
        with pytest.raises(TypeError):
            stc.stc_decode_attention_shared(*ok[:i], ok[i].double(), *ok[i + 1:])
    with pytest.raises(TypeError):
        stc.stc_decode_attention_shared(*ok[:1], ok[1].cpu(), *ok[2:])
    for i, v in ((6, torch.zeros(2, 2, dtype=torch.int32, device=DEV)), (11, 5), (1, d["q"].transpose(1, 2))):
        with pytest.raises(ValueError):
            stc.stc_decode_attention_shared(*ok[:i], v, *ok[i + 1:])
    for i, v in ((7, 4), (11, -1), (13, ws[:16]), (10, None)):
        with pytest.raises(stc.StcError):
            stc.stc_decode_attention_shared(*ok[:i], v, *ok[i + 1:])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D,Hkv,N", [(128, 8, 15000), (64, 16, 15003)])
@pytest.mark.parametrize("B", [7, 20])
def test_past_the_caches(B, D, Hkv, N, dtype):
    """Enough of the prefix in one call for loads past the caches; and with the last pages first."""
    c = Case(B, 2 * Hkv, Hkv, D, N, 8, 12, seed=B)
    c.check(dtype)
    NP = (N + 15) // 16
    c.check(dtype, pages=np.tile(np.arange(NP)[::-1], (Hkv, 1)))


@pytest.mark.parametrize("B,R,Hkv,cap", [(6, 4, 2, 40), (40, 5, 1, 40), (300, 1, 4, 90)])
def test_what_is_not_finite_stays_in_its_row(B, R, Hkv, cap):
    """NaN and infinities in one sequence's query, tails or padding do not reach the others."""
    c = Case(B, R * Hkv, Hkv, 128, 300, 8, cap, n_tail=[3, cap, -1, 7, 0])
    want = c.run()
    q, Kt, Vt = (c.d[x].clone() for x in ("q", "Kt", "Vt"))
    q[0, 0], q[2] = float("nan"), float("inf")
    q[1, 1] = float("inf")
    Kt[3, :, 2], Vt[3, :, 1] = float("inf"), float("nan")
    got = c.run(q=q, Kt=Kt, Vt=Vt)
    on = torch.from_numpy(c.n >= 0).to(DEV)[:, None].repeat(1, R * Hkv)
    assert got[0, 0].isnan().all() and got[3].isnan().all()
    on[0, 0] = on[1, 1] = False
    on[3] = False
    assert torch.equal(got[on], want[on]) and got[on].isfinite().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,R,Hkv,cap", [(6, 4, 2, 40), (30, 2, 1, 0), (40, 5, 1, 40), (300, 1, 4, 90)])
def test_large_values_and_what_is_not_finite_in_them(B, R, Hkv, cap, dtype):
    """Values scaled by a power of two, up to the end of what counts, scale the output exactly: |v| < 8, at
    most 390 tokens, weights of up to 2^8, and 2^3 2^107 <= 2^119 / 390.  NaN and infinities stay in their
    channel, those of the prefix in all queries of the KV head, those of a tail in its sequence's."""
    c = Case(B, R * Hkv, Hkv, 128, 300, 8, cap, keep=0xFF, n_tail=[3, cap, 7, 0])
    ramp(c, "K", 32, 7.5, 300)
    want = c.run(dtype)
    far = 2.0 ** 107
    assert np.abs(bits_to_f64(c.V)).max() < 8 and (not cap or np.abs(bits_to_f64(c.Vt)).max() < 8)
    big = lambda t: None if t is None else t * far  # noqa: E731
    assert torch.equal(c.run(dtype, v=big(c.d["v"]), Vt=big(c.d["Vt"])), want * far)
    h = Hkv - 1
    v = c.d["v"].clone()                                       # [Hkv, token * 8 + group, 16 channels]
    v[h, 5 * 8 + 2, 3], v[h, 290 * 8, 0], v[h, 100 * 8 + 7, 15] = float("inf"), float("nan"), float("-inf")
    Vt = None if not cap else c.d["Vt"].clone()
    on = torch.ones(B, R * Hkv, 128, dtype=torch.bool, device=DEV)
    for channel in (2 * 16 + 3, 0, 7 * 16 + 15):
        on[:, h * R:, channel] = False
    if cap:
        Vt[0, 0, 2, 77], Vt[1, 0, cap - 1, 20] = float("inf"), float("nan")
        on[0, :R, 77] = on[1, :R, 20] = False
    got = c.run(dtype, v=v, Vt=Vt)
    assert torch.equal(got[on], want[on]) and got[on].isfinite().all() and not got[~on].isfinite().any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,cap", [(3, 0), (3, 40), (40, 40), (300, 360)])
def test_logits_far_below_zero(B, cap, dtype):
    """Equal logits near the end of what counts: each of them is the largest."""
    c = Case(B, 1, 1, 128, 300, 8, cap, n_tail=[5, 0, cap])
    c.K[:], c.Kt[:], c.q[:] = 0x4680, 0x4680, 0xC500           # 2^14 and -2^11: logits of -1.4 * 2^28
    c.d["K"], c.d["q"] = PT.to_dev_bf16(c.K), PT.to_dev_bf16(c.q)
    if cap:
        c.d["Kt"] = PT.to_dev_bf16(c.Kt)
    got = c.run(dtype).double().cpu().numpy()
    V = bits_to_f64(c.V[0]) * np.repeat((c.mask[0].astype(int)[:, None] >> np.arange(8)) & 1, 16, axis=1)
    for b in range(B):
        n = max(int(c.n[b]), 0) if cap else 0
        want = (V.sum(0) + (bits_to_f64(c.Vt[b, 0, :n]).sum(0) if n else 0)) / (300 + n)
        # weights of one; sums of at most 660 values below 6 in float, one rounding to the output's type
        lim = 660 * 2.0 ** -24 * 6 + (2.0 ** -8 * np.abs(want) if dtype == BF16 else 0)
        assert (np.abs(got[b, 0] - want) <= lim).all()


def test_no_tails_at_all():
    c, *_ = _prefix()
    q = torch.randn(4, 8, 128, device=DEV).bfloat16()
    none = stc.SharedPrefix(c, 4, 0)
    some = stc.SharedPrefix(c, 4, 20)
    assert (none.attend(q) - some.attend(q)).abs().max() <= 4e-5
    with pytest.raises(stc.StcError):
        none.append(q, q[:, :2], q[:, :2])


@pytest.mark.parametrize("B,R,Hkv", [(2100, 16, 1), (9000, 16, 1), (1500, 5, 3)])
def test_thousands_of_sequences(B, R, Hkv):
    """More rows than some rounds of row blocks hold, and lengths that take many scans to add up."""
    c = Case(B, R * Hkv, Hkv, 64, 40, 4, 3, n_tail=[0, 3, -1, 2, 1, 3, 0])
    c.check(BF16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,R,Hkv,cap,N", [(3, 4, 2, 0, 700), (9, 7, 2, 40, 300), (40, 3, 1, 200, 20),
                                           (150, 2, 4, 180, 500)])
def test_bf16_output_is_the_float_output_rounded(B, R, Hkv, cap, N, D):
    """The output's type chooses the output's rounding and nothing else: the weights behind it are those
    of the float output.  Both runs add the same numbers in the same order, so the one rounding, to the
    nearest, is all that may lie between them."""
    c = Case(B, R * Hkv, Hkv, D, N, 8, cap, seed=N + B, n_tail=[cap, 0, 3, cap // 2])
    assert torch.equal(c.run(BF16), c.run(F32).bfloat16())


def check_some(c, some, dtype, pages=None):
    """Case.check for the sequences `some` and the first and last KV head, where the oracle would take long
    for all of them."""
    heads = sorted({0, c.Hkv - 1})
    rows = [h * (c.Hq // c.Hkv) + r for h in heads for r in range(c.Hq // c.Hkv)]
    got = c.run(dtype, pages).double().cpu().numpy()[some][:, rows]
    tails = (c.Kt[some][:, heads], c.Vt[some][:, heads]) if c.cap else (None, None)
    want, size, top = O.shared_attention_all(c.q[some][:, rows], c.K[heads], c.V[heads], c.mask[heads],
                                             pages if pages is None else pages[heads], c.G, *tails, c.n[some])
    lim = limits(want, size, top, c.N + c.cap, c.D, dtype)
    bad = ~(np.abs(got - want) <= lim)
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], lim[bad][:4])


# (sequences, query heads to a KV head, KV heads, tokens, room of the tails), tokens that a turn of the
# loop takes from a split: all tokens that stand between two of one group of wavefronts' tiles
TURNS = [((2, 16, 8, 20003, 0), 256), ((30, 1, 16, 12003, 9), 256),       # a wavefront to a tile
         ((4, 16, 8, 20003, 0), 128), ((8, 8, 8, 16003, 40), 128),        # 2
         ((64, 16, 1, 9003, 33), 64), ((150, 7, 2, 20011, 0), 64),        # 4
         ((48, 8, 8, 4001, 1000), 64), ((512, 1, 16, 8403, 0), 64)]      # 8: beside tails, a long prefix


def turns_of(c, turn, k):
    """Turns of the splits' loops in the mean, at least (more than 2: some split takes 3): the workspace holds
    a partial result of every query for each split and each piece of the tails."""
    parts = stc.stc_shared_workspace_bytes(c.shape, k, c.cap) // (c.B * c.Hq * (c.D + 2) * 4)
    return k * 16 / parts / turn


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("plan,turn", TURNS)
def test_many_tiles_a_split(plan, turn, D):
    """Loops that run for some turns: what they fetch while they work is attended, with and without a list
    of pages, up to a ragged end."""
    B, R, Hkv, N, cap = plan
    c = Case(B, R * Hkv, Hkv, D, N, 8, cap, seed=N, n_tail=[cap, 0, cap // 2, 3], n_cap=N + 20)
    NP = (N + 15) // 16
    assert turns_of(c, turn, NP) > 2
    some = [0, B // 2, B - 1]
    pages = np.stack([np.random.default_rng(h).permutation(NP)[:NP - 5] for h in range(Hkv)])
    pages[0, 40], pages[-1, -1], pages[0, 3] = -1, NP, 2**31 - 1
    pages[0, -1] = NP - 1 if NP - 1 not in pages[0] else pages[0, -1]
    for dtype in (F32, BF16):
        check_some(c, some, dtype)
        check_some(c, some, dtype, pages)


def ramp(c, which, per, step, tokens):
    """Logits of `which` (K or Kt) that rise by `step` in base 2 over `per` tokens, around zero."""
    from tests.helpers import f32_to_bf16_bits
    q = f32_to_bf16_bits(bits_to_f64(c.q) * 0.25)
    q[..., 0] = 0x4100                                         # 8
    at = np.arange(getattr(c, which).shape[-2]) - tokens / 2
    getattr(c, which)[..., 0] = f32_to_bf16_bits(at * (step / per * np.sqrt(c.D) / 8.0 / np.log2(np.e)))
    c.d["q"], c.q, plain = PT.to_dev_bf16(q), q, c.q
    c.d[which] = PT.to_dev_bf16(getattr(c, which))
    return plain


# Logits that rise from one tile of a group to its next by nearly what moves the running maximum, by a little
# more and by much more, and that fall.  Sums that are not scaled down when the maximum moves are then off by
# factors of 2^8 and more.
STEPS = [7.5, 8.5, 40.0, 1.0, -8.5]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("plan,turn", [t for t in TURNS if t[0] in ((2, 16, 8, 20003, 0), (4, 16, 8, 20003, 0),
                                                                    (64, 16, 1, 9003, 33), (48, 8, 8, 4001, 1000))])
def test_maxima_that_move_inside_a_split(plan, turn, D):
    B, R, Hkv, N, cap = plan
    c = Case(B, R * Hkv, Hkv, D, N, 8, cap, seed=N, n_tail=[5, 0, cap])
    assert turns_of(c, turn, (N + 15) // 16) > 2
    for step in STEPS:
        # (with 8 wavefronts the maximum may move every 32 tokens)
        plain = ramp(c, "K", 32 if cap == 1000 else turn, step, N)
        check_some(c, [0, B - 1], F32)
        check_some(c, [B // 2], BF16)
        c.q = plain


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_maxima_that_move_inside_a_tail(D, dtype):
    """Pieces of 8 tiles of 32 tokens: a call of few long tails with 16 query heads to a KV head."""
    c = Case(11, 16, 1, D, 50, 4, 700, seed=D, n_tail=[700, 257, 0, 480, 33, 699])
    for step in STEPS:
        plain = ramp(c, "Kt", 32, step, 700)
        for b in range(c.B):
            c.d["Kt"][b, :, c.n[b]:] = float("nan")
        check_some(c, list(range(11)), dtype)
        c.q = plain
