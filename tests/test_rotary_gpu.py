"""Rotary positions on the GPU against the oracle in 64 bits: layouts, orders of the dimensions,
partial rotation, far and given positions, the inverse, and the form for generated tokens."""
import numpy as np
import pytest
import torch

import paper_2604_21335_amd as stc
from oracle import stc_oracle as O
from tests import parity as PT
from tests.helpers import bits_to_f64, randn_bf16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALVES, INTER = stc.STC_ROTARY_HALVES, stc.STC_ROTARY_INTERLEAVED


def limit(x, want, rot, inter, amp):
    """One rounding to bf16, at most 2^-8 of the value, of a float result that is off by the sine and
    cosine (the hardware's are given 2^-17 here, a 512th of that step) and three float roundings, all
    in proportion to the pair's members: |amp| (|x0| + |x1|) 2^-16."""
    first = np.arange(rot // 2) * (2 if inter else 1)
    second = first + (1 if inter else rot // 2)
    size = np.zeros_like(x)
    size[..., first] = size[..., second] = np.abs(x[..., first]) + np.abs(x[..., second])
    return 2.0 ** -8 * (np.abs(want) + abs(amp) * size * 2.0 ** -16) + abs(amp) * size * 2.0 ** -16


def check(got, x, pos, turns, rot, layout, amp=1.0, inverse=False):
    want = O.rotary(x, pos, turns, rot, layout == INTER, amp, inverse)
    bad = np.abs(got - want) > limit(x, want, rot, layout == INTER, amp)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


def host(t):
    return bits_to_f64(PT.host_bf16(t))


@pytest.mark.parametrize("layout", [HALVES, INTER])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 64), (128, 112)])
@pytest.mark.parametrize("B,H,N", [(1, 1, 1), (2, 3, 5), (1, 4, 33), (3, 7, 70), (2, 2, 129)])
def test_layouts_and_sizes(layout, D, rot, B, H, N):
    """Every order of heads and tokens on either side, with room behind the tokens left alone."""
    rng = np.random.default_rng(B * 1000 + N + D + rot)
    bits = randn_bf16(rng, (B, H, N, D))
    x = bits_to_f64(bits)
    turns = stc.stc_rotary_turns(rot, base=1e4)
    dt = turns.to(DEV)
    dx = PT.to_dev_bf16(bits)
    for tokens_in in (False, True):
        src = dx.transpose(1, 2).contiguous().transpose(1, 2) if tokens_in else dx
        for tokens_out in (False, True):
            cap = N + 3
            y = torch.full((B, cap, H, D) if tokens_out else (B, H, cap, D), 7.0, dtype=torch.bfloat16,
                           device=DEV)
            v = y.transpose(1, 2) if tokens_out else y
            stc.stc_rotary(src, v[:, :, :N], dt, rot, layout, pos0=11)
            torch.cuda.synchronize()
            check(host(v[:, :, :N]), x, 11 + np.arange(N), turns.numpy(), rot, layout)
            assert (v[:, :, N:] == 7).all()
            if rot < D:   # the rest of a head is copied, bit for bit
                assert torch.equal(v[:, :, :N, rot:], dx[..., rot:])


@pytest.mark.parametrize("layout", [HALVES, INTER])
def test_in_place(layout):
    rng = np.random.default_rng(5)
    bits = randn_bf16(rng, (2, 5, 37, 128))
    turns = stc.stc_rotary_turns(96)
    x = PT.to_dev_bf16(bits)
    out = torch.empty_like(x)
    stc.stc_rotary(x, out, turns.to(DEV), 96, layout)
    stc.stc_rotary(x, x, turns.to(DEV), 96, layout)
    assert torch.equal(x, out)


@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0)])
@pytest.mark.parametrize("step", [1, 3])
def test_every_order_of_the_output(order, step):
    """All orders of sequences, heads and tokens, and every third of them; one row too close is refused."""
    sizes = (2, 3, 5)
    whole = [sizes[d] * step for d in order]
    y = torch.full((*whole, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    back = [order.index(d) for d in range(3)]
    v = y[::step, ::step, ::step].permute(*back, 3)
    x = torch.randn(*sizes, 64, device=DEV).bfloat16()
    t, want = stc.stc_rotary_turns(64).to(DEV), torch.empty_like(x)
    stc.stc_rotary(x, want, t, 64, INTER, pos0=4)
    stc.stc_rotary(x, v, t, 64, INTER, pos0=4)
    assert torch.equal(v, want) and (y == 7).sum() == y.numel() - x.numel()
    close = y.as_strided((*sizes, 64), (15 * 64, 64, 128, 1))
    with pytest.raises(stc.StcError):
        stc.stc_rotary(x, close, t, 64, INTER)
    assert torch.equal(v, want)


def test_in_place_in_another_order_is_refused():
    """Rows would be overwritten before they are read; where a dimension holds one element its stride is no
    order."""
    x = torch.randn(2, 8, 8, 64, device=DEV).bfloat16()
    t = stc.stc_rotary_turns(64).to(DEV)
    before = x.clone()
    with pytest.raises(stc.StcError) as e:
        stc.stc_rotary(x, x.transpose(1, 2), t, 64, HALVES)
    assert e.value.status == stc.STC_ERR_SHAPE and torch.equal(x, before)
    one, want = x[:1, :1], torch.empty_like(x[:1, :1])
    stc.stc_rotary(one, want, t, 64, HALVES)
    stc.stc_rotary(one, one.as_strided(one.shape, (8, 4096, 64, 1)), t, 64, HALVES)
    assert torch.equal(one, want) and torch.equal(x[1], before[1])


@pytest.mark.parametrize("pos", [[0, -1, -5, 1], [2**31 - 1, -2**31, 10**6, 12345678], [3, 3, 3, 3]])
def test_given_and_far_positions(pos):
    rng = np.random.default_rng(9)
    bits = randn_bf16(rng, (3, 6, 4, 128))
    turns = stc.stc_rotary_turns(128, base=5e5)
    p = np.array([pos, pos[::-1], np.roll(pos, 1)], dtype=np.int64)
    y = torch.empty(3, 6, 4, 128, dtype=torch.bfloat16, device=DEV)
    stc.stc_rotary(PT.to_dev_bf16(bits), y, turns.to(DEV), 128, HALVES,
                   pos=torch.from_numpy(p.astype(np.int32)).to(DEV))
    check(host(y), bits_to_f64(bits), p[:, None, :], turns.numpy(), 128, HALVES)


@pytest.mark.parametrize("pos0", [0, 131071, 10**6, 2**31 - 40, -2**31])
def test_first_position_and_amplitude(pos0):
    rng = np.random.default_rng(2)
    bits = randn_bf16(rng, (1, 4, 40, 64))
    turns = stc.stc_rotary_turns(64, base=1e6, kind=stc.STC_ROTARY_SCALE_CHANNELS, factor=8.0,
                                 original_len=4096, slow=1.0, fast=32.0)
    y = torch.empty(1, 4, 40, 64, dtype=torch.bfloat16, device=DEV)
    stc.stc_rotary(PT.to_dev_bf16(bits), y, turns.to(DEV), 64, INTER, pos0=pos0, amplitude=1.2079)
    check(host(y), bits_to_f64(bits), pos0 + np.arange(40), turns.numpy(), 64, INTER, np.float32(1.2079))


@pytest.mark.parametrize("layout", [HALVES, INTER])
def test_the_inverse_is_the_gradient(layout):
    """Against the formula, and against differences: the map is linear, so the difference quotient of
    <g, rotary(x)> is <g, rotary(e)>, which has to be <inverse(g), e>."""
    rng = np.random.default_rng(7)
    B, H, N, D, rot, amp = 2, 3, 19, 128, 64, 1.25
    gb, eb = randn_bf16(rng, (B, H, N, D)), randn_bf16(rng, (B, H, N, D))
    turns = stc.stc_rotary_turns(rot)
    dt = turns.to(DEV)
    back, fwd = (torch.empty(B, H, N, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    stc.stc_rotary(PT.to_dev_bf16(gb), back, dt, rot, layout, pos0=77, amplitude=amp, inverse=True)
    stc.stc_rotary(PT.to_dev_bf16(eb), fwd, dt, rot, layout, pos0=77, amplitude=amp)
    g, e = bits_to_f64(gb), bits_to_f64(eb)
    check(host(back), g, 77 + np.arange(N), turns.numpy(), rot, layout, amp, inverse=True)
    a, b = g * host(fwd), host(back) * e
    # each term of either sum carries a relative error of 2^-8 and the sine's share
    slack = (2.0 ** -8 + 2.0 ** -13) * (np.abs(a).sum(-1) + np.abs(b).sum(-1)) + 1e-6
    assert (np.abs(a.sum(-1) - b.sum(-1)) <= slack).all()


def test_position_zero_and_padding_copy():
    """Position 0 leaves the values as they are; the sign of a zero may change."""
    x = torch.randn(1, 2, 9, 64, device=DEV).bfloat16()
    y = torch.empty_like(x)
    stc.stc_rotary(x, y, stc.stc_rotary_turns(64).to(DEV), 64, HALVES,
                   pos=torch.zeros(1, 9, dtype=torch.int32, device=DEV))
    assert torch.equal(x, y)


def test_rows_behind_four_gib():
    """Strides that pass 2^32 bytes."""
    far = (1 << 32) // 2 + 4096                        # elements between two tokens
    big = torch.empty(far + 2 * 64, dtype=torch.bfloat16, device=DEV)
    x = big.as_strided((1, 2, 2, 64), (0, 64, far, 1))
    src = torch.randn(1, 2, 2, 64, device=DEV).bfloat16()
    x.copy_(src)
    turns = stc.stc_rotary_turns(64)
    y, z = torch.empty_like(src), torch.empty_like(src)
    stc.stc_rotary(x, y, turns.to(DEV), 64, HALVES, pos0=3)
    stc.stc_rotary(src, z, turns.to(DEV), 64, HALVES, pos0=3)
    assert torch.equal(y, z)
    stc.stc_rotary(x, x, turns.to(DEV), 64, HALVES, pos0=3)
    assert torch.equal(x, z)


@pytest.mark.parametrize("tokens_out", [False, True])
def test_past_the_caches(tokens_out):
    """256 MiB and more go past the caches: the same bits as in two calls that do not; and in place."""
    N, H = (1 << 20) // 8 + 1, 8
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.empty(1, H, N, 128, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    t = stc.stc_rotary_turns(128, base=1e6).to(DEV)
    shape = (1, N, H, 128) if tokens_out else (1, H, N, 128)
    want, got = (torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    if tokens_out:
        want, got = want.transpose(1, 2), got.transpose(1, 2)
    half = N // 2
    stc.stc_rotary(x[:, :, :half], want[:, :, :half], t, 128, HALVES, pos0=5)
    stc.stc_rotary(x[:, :, half:], want[:, :, half:], t, 128, HALVES, pos0=5 + half)
    stc.stc_rotary(x, got, t, 128, HALVES, pos0=5)
    assert torch.equal(got, want)
    stc.stc_rotary(x, x, t, 128, HALVES, pos0=5)
    assert torch.equal(x, want)


@pytest.mark.parametrize("B,Hq,Hkv,D,rot,layout", [
    (1, 1, 1, 64, 64, HALVES), (5, 8, 2, 128, 128, HALVES), (3, 14, 2, 128, 64, INTER),
    (2, 96, 32, 128, 128, INTER), (70, 4, 4, 64, 16, HALVES), (4, 8, 8, 64, 0, HALVES)])
@pytest.mark.parametrize("given", [False, True])
def test_append(B, Hq, Hkv, D, rot, layout, given):
    """Tails of different lengths, empty, full and padded among them; rows that are not written, and
    all of a padded or full element, stay as they were."""
    rng = np.random.default_rng(B + Hq + D)
    cap = 6
    n = rng.integers(0, cap, size=B).astype(np.int32)
    if B > 2:
        n[1], n[2] = -1, cap
    if B > 3:
        n[3] = 2**31 - 1
    proj = randn_bf16(rng, (B, Hq + 2 * Hkv, D))
    dp = PT.to_dev_bf16(proj)
    Kt, Vt = (torch.full((B, Hkv, cap, D), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q_out = torch.full((B, Hq, D), 9.0, dtype=torch.bfloat16, device=DEV)
    dn, n_out = torch.from_numpy(n).to(DEV), torch.full((B,), 99, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    turns = stc.stc_rotary_turns(rot or 16)
    pos = rng.integers(0, 200000, size=B) if given else 1000 + n.astype(np.int64)
    s = stc.make_shape(B, Hq, Hkv, D, 16, 1, 16)
    stc.stc_rotary_append(s, dp[:, :Hq], dp[:, Hq:Hq + Hkv], dp[:, Hq + Hkv:], q_out, Kt, Vt, dn, cap,
                          turns.to(DEV) if rot else None, rot, layout, amplitude=1.125,
                          pos=torch.from_numpy(pos.astype(np.int32)).to(DEV) if given else None,
                          pos0=1000, n_out=n_out, dev_status=status)
    torch.cuda.synchronize()
    there = (n >= 0) & (n < cap)
    assert status.item() == int((n >= cap).any())
    assert np.array_equal(n_out.cpu().numpy(), np.where(there, n + 1, n))
    x = bits_to_f64(proj)
    b = np.nonzero(there)[0]
    if rot:
        check(host(q_out)[b], x[b, :Hq], pos[b, None], turns.numpy(), rot, layout, 1.125)
        check(host(Kt)[b, :, n[b]], x[b, Hq:Hq + Hkv], pos[b, None], turns.numpy(), rot, layout, 1.125)
    else:
        assert np.array_equal(host(q_out)[b], x[b, :Hq])
        assert np.array_equal(host(Kt)[b, :, n[b]], x[b, Hq:Hq + Hkv])
    assert np.array_equal(host(Vt)[b, :, n[b]], x[b, Hq + Hkv:])
    untouched = np.ones((B, Hkv, cap, D), dtype=bool)
    untouched[b, :, n[b]] = False
    assert (host(Kt)[untouched] == 5).all() and (host(Vt)[untouched] == 5).all()
    assert (host(q_out)[~there] == 9).all()


def test_append_agrees_with_the_prompt_form_and_advances_in_place():
    B, Hq, Hkv, D, cap = 3, 4, 2, 128, 8
    rot = stc.Rotary(128, base=1e6, device=DEV)
    s = stc.make_shape(B, Hq, Hkv, D, 16, 1, 16)
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(cap, B, Hq + 2 * Hkv, D, device=DEV, generator=g).bfloat16()
    Kt, Vt = (torch.zeros(B, Hkv, cap, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    n = torch.zeros(B, dtype=torch.int32, device=DEV)
    qs = torch.empty(cap, B, Hq, D, dtype=torch.bfloat16, device=DEV)
    for i in range(cap):
        stc.stc_rotary_append(s, x[i, :, :Hq], x[i, :, Hq:Hq + Hkv], x[i, :, Hq + Hkv:], qs[i], Kt, Vt, n,
                              cap, rot.turns, 128, HALVES, pos0=500, n_out=n)
    assert n.tolist() == [cap] * B
    want = torch.empty(B, Hq + Hkv, cap, D, dtype=torch.bfloat16, device=DEV)
    rot.apply(x[:, :, :Hq + Hkv].permute(1, 2, 0, 3), want, pos0=500)
    assert torch.equal(qs.permute(1, 2, 0, 3), want[:, :Hq]) and torch.equal(Kt, want[:, Hq:])
    assert torch.equal(Vt, x[:, :, Hq + Hkv:].permute(1, 2, 0, 3))


def test_append_in_place_over_the_queries():
    B, Hq, Hkv, D = 4, 4, 2, 64
    s = stc.make_shape(B, Hq, Hkv, D, 16, 1, 16)
    q = torch.randn(B, Hq, D, device=DEV).bfloat16()
    k, v = (torch.randn(B, Hkv, D, device=DEV).bfloat16() for _ in range(2))
    t = stc.stc_rotary_turns(64).to(DEV)
    n = torch.tensor([0, 1, -1, 2], dtype=torch.int32, device=DEV)
    tails = [torch.zeros(B, Hkv, 4, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    out = q.clone()
    stc.stc_rotary_append(s, q.clone(), k, v, out, *tails, n, 4, t, 64, HALVES)
    stc.stc_rotary_append(s, q, k, v, q, *tails, n, 4, t, 64, HALVES)
    assert torch.equal(q, out)


def test_keys_get_their_positions_on_the_way_into_a_cache():
    """RoutedCache.build with rotary equals rotation, then construction."""
    B, Hq, Hkv, D, N, G = 2, 4, 2, 128, 100, 8
    g = torch.Generator(device=DEV).manual_seed(1)
    K = torch.randn(B, N, Hkv, D, device=DEV, generator=g).bfloat16().transpose(1, 2)
    V = torch.randn(B, Hkv, N, D, device=DEV, generator=g).bfloat16()
    m = torch.randint(0, 256, (B, Hkv, N), device=DEV, generator=g).to(torch.int16)
    q = torch.randn(B, Hq, D, device=DEV, generator=g).bfloat16()
    rot = stc.Rotary(128, device=DEV)
    a, b = (stc.RoutedCache(B, Hq, Hkv, D, N, G, 3, n_cap=112, device=DEV) for _ in range(2))
    a.build(K, V, mask_in=m, rotary=rot, pos0=5)
    Kr = torch.empty(B, Hkv, N, D, dtype=torch.bfloat16, device=DEV)
    rot.apply(K, Kr, pos0=5)
    b.build(Kr, V, mask_in=m)
    assert torch.equal(a.K[:, :, :N], b.K[:, :, :N])
    assert torch.equal(a.bounds_rows(), b.bounds_rows())
    assert torch.equal(a.step(q), b.step(q))


def test_captured_and_replayed():
    """The counts lie on the device: a captured append goes on where the last replay stopped."""
    B, Hq, Hkv, D, cap = 2, 4, 2, 64, 8
    s = stc.make_shape(B, Hq, Hkv, D, 16, 1, 16)
    t = stc.stc_rotary_turns(64).to(DEV)
    x = torch.randn(B, Hq + 2 * Hkv, D, device=DEV).bfloat16()

    def fresh():
        return (torch.zeros(B, Hq, D, dtype=torch.bfloat16, device=DEV),
                *[torch.zeros(B, Hkv, cap, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)],
                torch.tensor([0, 3], dtype=torch.int32, device=DEV))

    def call(q, k, v, n):
        stc.stc_rotary_append(s, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], q, k, v, n, cap, t, 64,
                              HALVES, pos0=9, n_out=n)
    a, b = fresh(), fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*a)
    for _ in range(6):
        x.copy_(torch.randn(B, Hq + 2 * Hkv, D, device=DEV))
        graph.replay()
        call(*b)
        torch.cuda.synchronize()
        assert all(torch.equal(u, w) for u, w in zip(a, b))
    assert a[3].tolist() == [6, 8]


def test_another_stream():
    x = torch.randn(2, 4, 300, 128, device=DEV).bfloat16()
    t = stc.stc_rotary_turns(128).to(DEV)
    want, got = torch.empty_like(x), torch.empty_like(x)
    stc.stc_rotary(x, want, t, 128, INTER)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        stc.stc_rotary(x, got, t, 128, INTER)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_tensors_of_another_shape_or_type_are_refused():
    x = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16, device=DEV)
    t = stc.stc_rotary_turns(64).to(DEV)
    bad = [(ValueError, (x, x[:, :, :3], t, 64, 0)), (TypeError, (x.float(), x, t, 64, 0)),
           (TypeError, (x.cpu(), x, t, 64, 0)), (ValueError, (x[0], x[0], t, 64, 0)),
           (ValueError, (x, x, t[:16], 64, 0)), (TypeError, (x, x, t.float(), 64, 0)),
           (ValueError, (x.transpose(2, 3), x.transpose(2, 3), t, 64, 0)),
           (ValueError, (x, x, t, 64, 0, torch.zeros(3, dtype=torch.int32, device=DEV))),
           (ValueError, (x[:, :, :0], x[:, :, :0], t, 64, 0)), (stc.StcError, (x, x, t[:28], 56, 0))]
    for error, args in bad:
        with pytest.raises(error):
            stc.stc_rotary(*args)
    s = stc.make_shape(1, 2, 1, 64, 16, 1, 16)
    apart = x[0, :, :1].transpose(0, 1)              # heads that do not lie side by side
    q, k = apart.contiguous(), apart[:, :1].contiguous()
    tail, n = x[:, :1], torch.zeros(1, dtype=torch.int32, device=DEV)
    ok = [s, q, k, k, q.clone(), tail.clone(), tail.clone(), n, 4, t, 64, 0]
    stc.stc_rotary_append(*ok)
    for i, v in [(1, k), (1, apart), (2, q), (4, k.clone()), (5, tail[:, :, :3].contiguous()), (7, n.repeat(2)),
                 (8, 5), (9, t[:8])]:
        with pytest.raises(ValueError):
            stc.stc_rotary_append(*ok[:i], v, *ok[i + 1:])
