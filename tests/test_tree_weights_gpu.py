"""How exactly the attention of drafted tokens carries a weight, where a float is asked for."""
import numpy as np
import pytest
import torch

import paper_2604_21335_amd as stc
from tests import parity as PT
from tests.helpers import bits_to_f64, f32_to_bf16_bits, randn_bf16
from tests.test_tree_gpu import BF16, DEV, F32

pytestmark = pytest.mark.gpu
G, CAP, LOG2E = 4, 40, 1.4426950408889634


def two_tokens(B, T, R, Hkv, N, D, each, in_tail, dtype=F32):
    """One channel makes the logits: token a's 32 q (values 0), token b's 24 q (values of size 1), all others' -1024 q, with
    q = 1 .. 2 by row; a stands in front of b, in the same tile.  So an output is w v_b / (1 + w) with w = 2^-x, x = 8 q log2(e) / sqrt(D) of 1 .. 3, of which
    nothing is a bf16 number.  -> (outputs, v_b's share, v_b) in 64 bits."""
    rng = np.random.default_rng(N + B * T * R + D)
    P, Hq = B if each else 1, R * Hkv
    q = np.zeros((B, T, Hq, D), dtype=np.float32)
    q[..., 5] = 1 + (np.arange(B * T * Hq) * 37 % 128).reshape(B, T, Hq) / 128
    K, V = np.zeros((P, Hkv, N, D), dtype=np.float32), bits_to_f64(randn_bf16(rng, (P, Hkv, N, D)))
    Kt, Vt = np.zeros((B, Hkv, CAP + T, D), dtype=np.float32), bits_to_f64(randn_bf16(rng, (B, Hkv, CAP + T, D)))
    K[..., 5] = -1024
    Kt[..., 5] = -1024
    k, v, a, b = (Kt, Vt, CAP - 6, CAP - 5) if in_tail else (K, V, N // 16 * 16 - 7, N // 16 * 16 - 6)
    k[:, :, a, 5], k[:, :, b, 5] = 32, 24
    v[:, :, a] = 0
    v[:, :, b] = np.where(v[:, :, b] < 0, -1, 1) * (1 + np.abs(v[:, :, b]) % 1)
    v = bits_to_f64(f32_to_bf16_bits(v.astype(np.float32)))
    V, Vt = (V, v) if in_tail else (v, Vt)

    def dev(x):
        return PT.to_dev_bf16(f32_to_bf16_bits(x.astype(np.float32)))
    shape = stc.make_shape(B, Hq, Hkv, D, N, G, N * G)
    mask = torch.full((P, Hkv, N), 15, dtype=torch.int16, device=DEV)
    off = (torch.arange(N + 1, dtype=torch.int32, device=DEV) * G).expand(P, Hkv, -1).contiguous()
    k_pages = (N + 15) // 16
    ws = torch.empty(stc.stc_tree_workspace_bytes(shape, T, k_pages, CAP + T, n_prefix=P), dtype=torch.uint8, device=DEV)
    out = torch.zeros(B, T, Hq, D, dtype=dtype, device=DEV)
    stc.stc_decode_attention_tree(shape, dev(q), dev(K), dev(V).view(P, Hkv, N * G, D // G), mask, off, None, k_pages,
                                  dev(Kt), dev(Vt), torch.full((B,), CAP, dtype=torch.int32, device=DEV), CAP + T, out, ws,
                                  n_prefix=P)
    w = np.exp2(-8.0 * q[..., 5].astype(np.float64) * LOG2E / np.sqrt(D))
    vb = np.broadcast_to(v[:, :, b], (B, Hkv, D)).repeat(R, 1)[:, None]
    return out.double().cpu().numpy(), (w / (1 + w))[..., None], vb


# rows of a KV head: up to 32 (of few and of many prefixes), 64, more by 4 and by 8 wavefronts; prefixes of a few and of
# many tokens
# (floats that were made of two parts beyond 16384 tokens were off by 2^-17.2)
@pytest.mark.parametrize("in_tail", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,R,Hkv,N,each", [(1, 8, 4, 2, 1000, False), (2, 8, 4, 2, 20001, False), (32, 4, 4, 2, 500, True),
                                              (1, 64, 1, 2, 20001, False), (1, 64, 2, 1, 1000, False), (1, 40, 4, 1, 17000, False),
                                              (2, 64, 16, 8, 9000, False), (1, 64, 16, 4, 17000, False), (2, 50, 2, 2, 33000, True)])
def test_floats_are_made_of_weights_in_float(B, T, R, Hkv, N, each, D, in_tail):
    """The exponent's parts, up to 12, are rounded three times (2^-24 of them each, times ln 2): 2^-20.9; the exponential is
    off by 2^-22, the weight in three parts by 2^-24, 16 sums and the last division by 2^-24 each: 2^-19.9.  Together
    2^-18.8.  The other tokens have 2^-130 each.  Weights in two parts are off by up to 2^-16, these by 2^-17.2."""
    got, share, vb = two_tokens(B, T, R, Hkv, N, D, each, in_tail)
    off = np.abs(got / (share * vb) - 1).max()
    assert off <= 2.0 ** -18.8, np.log2(off)


def test_two_parts_would_be_seen():
    """The claim about two parts, by arithmetic on the same weights."""
    for D in (64, 128):
        w = np.exp2(-8.0 * (1 + np.arange(64) * 37 % 128 / 128) * LOG2E / np.sqrt(D)).astype(np.float32)
        one = bits_to_f64(f32_to_bf16_bits(w))
        two = one + bits_to_f64(f32_to_bf16_bits((w - one).astype(np.float32)))
        # (the sum of weights is made of whole ones, so an output is off by as much as its weight)
        assert np.abs(two / w.astype(np.float64) - 1).max() >= 2.0 ** -17.3
