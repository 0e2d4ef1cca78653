"""The operators of serving a batch over one shared prompt, and what they are measured on.

`rotary`: rotary positions of a prompt's queries or keys.  `append`: the same for one new token of
every sequence, whose key and value go to the sequence's own tail.  `shared`: decode attention of a
batch whose sequences share one compressed prefix (full-width keys, values stored as the groups that
the router kept) and have an uncompressed tail each.  `step`: the last two one after the other, layer
by layer, as a token is generated.

With `own` false `run` computes them from elementary torch operations; with `own` true it calls the
framework.  Inputs are synthetic, made on the GPU from the seed, with the value structure of the
framework's workloads: normal queries, keys and values, keys with four channels per head scaled by 8,
kept-group counts spread around their mean.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 16


# --------------------------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------------------------
def listed():
    return [
        # A prompt of 16 tokens, 8 heads of 64: the smallest call there is, a launch and nothing else.
        _rotary(name="rotary_tiny", B=1, H=8, N=16, D=64, rot=64),
        # Queries of the prompts of a Qwen2.5-7B-shaped layer as the projection leaves them (token by
        # token), 4 x 32768 tokens: the largest tensor that positions are applied to.
        _rotary(name="rotary_qwen25_7b_queries", B=4, H=28, N=32768, D=128, rot=128, base=1e6),
        # Keys of 5 left-padded prompts (given positions) from the projection's order into a cache with
        # room to grow: interleaved pairs, half of the head rotated, frequencies slowed by wavelength.
        _rotary(name="rotary_keys_ragged", B=5, H=8, N=12013, cap=12288, D=128, rot=64,
                layout="interleaved", given=True, out_tokens=False, base=5e5, scaling="wavelengths",
                factor=8.0, length=8192, slow=1.0, fast=4.0),
        # Gradient of a LLaMA-2-7B-shaped layer's queries, batch 8, 4096 tokens, head by head.
        _rotary(name="rotary_gradient_llama2_7b", B=8, H=32, N=4096, D=128, rot=128, inverse=True,
                in_tokens=False, out_tokens=False),
        # New tokens of a small batch in mid-generation, positions stretched linearly.
        _append(name="append_small", B=5, Hq=32, Hkv=8, D=128, rot=128, cap=128, scaling="linear",
                factor=4.0),
        # New tokens of a full serving batch far behind the trained length: frequencies slowed by
        # channel, cosines and sines raised to match.
        _append(name="append_batch", B=256, Hq=28, Hkv=4, D=128, rot=128, cap=256, base=1e6,
                scaling="channels", factor=4.0, length=32768, slow=1.0, fast=32.0, amplitude=1.1386),
        # Two answers to one short prompt, 8 heads of 64: the smallest step.
        _shared(name="shared_tiny", B=2, Hq=8, Hkv=8, D=64, N=1024, G=4, keep=0.5),
        # 16 answers over one 32768-token document, Qwen2.5-7B-shaped layer, up to 100 tokens each so
        # far: bound by the prefix's bytes.
        _shared(name="shared_qwen25_7b_32k", B=16, Hq=28, Hkv=4, D=128, N=32768, G=8, keep=0.5, tail=100),
        # The largest: 256 answers over the same document, bf16 output; bound by the matrix cores.
        _shared(name="shared_qwen25_7b_32k_b256", B=256, Hq=28, Hkv=4, D=128, N=32768, G=8, keep=0.5,
                tail=100, bf16=True),
        # 64 questions about one image: a LLaVA-1.5-7B-shaped prefix of 144 retained visual and 64 text
        # tokens, 32 heads, question and answer of up to 256 tokens in the tails.
        _shared(name="shared_llava15_7b_prefix", B=64, Hq=32, Hkv=32, D=128, N=208, G=8, keep=0.55,
                tail=256),
        # 3 answers over 131072 tokens of which 256 pages were selected, a quarter of the value groups.
        _shared(name="shared_selected_128k", B=3, Hq=28, Hkv=4, D=128, N=131072, G=16, keep=0.25, k=256,
                tail=33),
        # A token of 48 sequences through 4 layers: append, then attend; grouped queries 4:1, a prefix
        # that fills neither its last page nor a tile, long answers.
        _shared(name="step_4_layers", kind="step", B=48, Hq=32, Hkv=8, D=128, N=4001, G=8, keep=0.5,
                tail=1000, rot=128, layers=4, bf16=True),
    ]


def _pairs(layout="halves", base=1e4, scaling="none", factor=1.0, length=0, slow=0.0, fast=0.0,
           amplitude=1.0):
    return dict(layout=layout, base=base, scaling=scaling, factor=factor, length=length, slow=slow,
                fast=fast, amplitude=amplitude)


def _take(kw):
    return _pairs(**{k: kw.pop(k) for k in list(kw) if k in _pairs()})


def _rotary(**kw):
    d = dict(kind="rotary", cap=0, given=False, inverse=False, in_tokens=True, out_tokens=True, first=0)
    d.update(_take(kw))
    d.update(kw)
    return d


def _append(**kw):
    d = dict(kind="append", start=0)
    d.update(_take(kw))
    d.update(kw)
    return d


def _shared(**kw):
    d = dict(kind="shared", k=0, tail=0, bf16=False, layers=1, rot=0)
    d.update(_take(kw))
    d.update(kw)
    return d


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_pairs(rng, D):
    scaling = rng.choice(["none", "none", "linear", "base", "channels", "wavelengths"])
    rot = rng.choice([D, D, D // 2, D // 4, 48])
    far = scaling != "none"
    return dict(rot=rot, layout=rng.choice(["halves", "interleaved"]), base=rng.choice([1e4, 5e5, 1e6]),
                scaling=scaling, factor=rng.choice([2.0, 4.0, 8.0]) if far else 1.0,
                length=rng.choice([4096, 32768]) if far else 0, slow=1.0 if far else 0.0,
                fast=rng.choice([4.0, 32.0]) if far else 0.0,
                amplitude=1.1386 if scaling == "channels" else 1.0)


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "append", "shared", "shared", "shared", "step"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 4, 8, 8, 32])
    R = rng.choice([1, 2, 4, 5, 7, 8, 16]) if Hkv <= 8 else 1
    if kind == "rotary":
        H = rng.choice([Hkv, Hkv * R])
        N = _log(rng, 1, 131072)
        B = _log(rng, 1, max(1, min(64, 4 * 28 * 32768 // (H * N))))
        return _rotary(B=B, H=H, N=N, D=D, cap=rng.choice([0, N + rng.randint(1, 300)]),
                       given=rng.random() < 0.4, inverse=rng.random() < 0.25,
                       in_tokens=rng.random() < 0.7, out_tokens=rng.random() < 0.4,
                       first=rng.choice([0, 0, _log(rng, 1, 1000000)]), **_draw_pairs(rng, D))
    B = _log(rng, 1, 256)
    if kind == "append":
        return _append(B=B, Hq=Hkv * R, Hkv=Hkv, D=D, cap=rng.randint(1, 256),
                       start=_log(rng, 1, 1000000), **_draw_pairs(rng, D))
    N = _log(rng, 100, 131072)
    layers = 1 if kind == "shared" else rng.choice([1, 2, 3])
    tail = rng.choice([0, _log(rng, 1, 1024)]) if kind == "shared" else _log(rng, 1, 1024)
    most = 256 * 28 * 32768 // 4 // layers                     # scores of a layer
    B = max(1, min(B, most // (Hkv * R * N), (1 << 29) // (Hkv * (tail + 8) * D * 4 * layers)))
    NP = (N + PAGE - 1) // PAGE
    more = _draw_pairs(rng, D) if kind == "step" else {}
    return _shared(kind=kind, B=B, Hq=Hkv * R, Hkv=Hkv, D=D, N=N, G=rng.choice([4, 8, 8, 16 if D == 128 else 2]),
                   keep=rng.choice([0.25, 0.375, 0.5, 0.5625, 0.75]), tail=tail,
                   k=0 if rng.random() < 0.7 else max(1, int(NP * rng.uniform(0.05, 0.5))),
                   bf16=kind == "step" or rng.random() < 0.5, layers=layers, **more)


# --------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------
def _turns(c):
    """Revolutions per position of every rotated pair, in 64 bits."""
    rot, base = c["rot"], c["base"]
    if c["scaling"] == "base":                 # the base raised so that the slowest pair slows by factor
        base = base * c["factor"] ** (rot / (rot - 2))
    j = np.arange(rot // 2, dtype=np.float64)
    freq = base ** (-2.0 * j / rot)
    if c["scaling"] == "linear":
        freq = freq / c["factor"]
    elif c["scaling"] == "channels":           # slowed from one pair index on, a ramp in between
        at = lambda b: rot * math.log(c["length"] / (2 * math.pi * b)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(c["fast"])), 0), min(math.ceil(at(c["slow"])), rot - 1)
        w = np.clip((j - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        freq = freq / c["factor"] * w + freq * (1.0 - w)
    elif c["scaling"] == "wavelengths":        # slowed below so many revolutions over the trained length
        w = np.clip((c["length"] * freq / (2 * math.pi) - c["slow"]) / (c["fast"] - c["slow"]), 0.0, 1.0)
        freq = freq * (w + (1.0 - w) / c["factor"])
    return torch.from_numpy(freq / (2 * math.pi)).to(DEV)


def _normal(g, *shape):
    x = torch.empty(*shape, dtype=torch.bfloat16, device=DEV)
    return x.normal_(generator=g)


def _outliers(g, x):
    """Four channels per head times 8 (heads are the second dimension from the front)."""
    H, D = x.shape[0], x.shape[-1]
    at = torch.rand(H, D, generator=g, device=DEV).argsort(dim=1)[:, :4]
    s = torch.ones(H, D, device=DEV).scatter_(1, at, 8.0).to(x.dtype)
    return x.mul_(s[:, None, :])


def _counts(g, T, G, keep, shape):
    """Kept groups per token: at least one, G * keep in the mean."""
    n = 1 + torch.binomial(torch.full(shape + (T,), float(G - 1), device=DEV),
                           torch.full(shape + (T,), (G * keep - 1) / (G - 1), device=DEV).clamp(0, 1),
                           generator=g)
    return n.to(torch.int64)


def _prefix(g, c):
    """One layer's cache of the shared prefix, as the framework's cache construction leaves it."""
    H, N, G, D = c["Hkv"], c["N"], c["G"], c["D"]
    K = _outliers(g, _normal(g, H, N, D))
    rank = torch.rand(H, N, G, generator=g, device=DEV).argsort(dim=2).argsort(dim=2)
    kept = rank < _counts(g, N, G, c["keep"], (H,))[:, :, None]
    mask = (kept.to(torch.int32) << torch.arange(G, device=DEV, dtype=torch.int32)).sum(2)
    off = torch.zeros(H, N + 1, dtype=torch.int64, device=DEV)
    off[:, 1:] = kept.sum(2).cumsum(1)
    v = _normal(g, H, N * G, D // G)
    NP = (N + PAGE - 1) // PAGE
    pages = None
    if c["k"]:
        pages = torch.rand(H, NP, generator=g, device=DEV).argsort(dim=1)[:, :c["k"]].sort(dim=1)[0]
        pages = pages.to(torch.int32).contiguous()
    return dict(K=K, mask=mask.to(torch.int16), off=off.to(torch.int32), v=v, pages=pages,
                k=c["k"] or NP)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(c=c)
    if c["kind"] == "rotary":
        B, H, N, D = c["B"], c["H"], c["N"], c["D"]
        s["turns"] = _turns(c)
        x = _normal(g, B, N, H, D).transpose(1, 2) if c["in_tokens"] else _normal(g, B, H, N, D)
        cap = c["cap"] or N
        y = torch.zeros((B, cap, H, D) if c["out_tokens"] else (B, H, cap, D), dtype=torch.bfloat16,
                        device=DEV)
        s["x"], s["y"] = x, (y.transpose(1, 2) if c["out_tokens"] else y)[:, :, :N]
        s["pos"] = None
        if c["given"]:       # left-padded: the first tokens of a sequence all stand at its first position
            pad = torch.randint(0, N // 2 + 1, (B, 1), generator=g, device=DEV)
            s["pos"] = (c["first"] + (torch.arange(N, device=DEV) - pad).clamp(min=0)).to(torch.int32)
        return s
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    if c["kind"] in ("append", "step"):
        s["turns"] = _turns(c)
    cap = c["cap"] if c["kind"] == "append" else c["tail"] + (8 if c["kind"] == "step" else 0)
    if c["kind"] == "append":
        s["n"] = torch.randint(0, cap, (B,), generator=g, device=DEV, dtype=torch.int32)
    elif cap:
        s["n"] = torch.randint(0, c["tail"] + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["n"][0] = c["tail"]
    else:
        s["n"] = None
    s["cap"], s["layers"] = cap, []
    for _ in range(c.get("layers", 1)):
        a = {}
        if c["kind"] != "append":
            a.update(_prefix(g, c))
            a["q"] = _normal(g, B, Hq, D)
            a["out"] = torch.zeros(B, Hq, D, dtype=torch.bfloat16 if c["bf16"] else torch.float32,
                                   device=DEV)
        if cap:
            a["Kt"] = _outliers(g, _normal(g, Hkv, B * cap, D)).view(Hkv, B, cap, D).transpose(0, 1).contiguous()
            a["Vt"] = _normal(g, B, Hkv, cap, D)
        if c["kind"] != "shared":
            a["qkv"] = _normal(g, B, Hq + 2 * Hkv, D)   # what the fused projection leaves
            a["q"] = torch.zeros(B, Hq, D, dtype=torch.bfloat16, device=DEV)
        s["layers"].append(a)
    return s


# --------------------------------------------------------------------------------------------
# The plain forms
# --------------------------------------------------------------------------------------------
def _partners(c):
    """Channels of the first and second members of the pairs."""
    j = torch.arange(c["rot"] // 2, device=DEV)
    return (j, j + c["rot"] // 2) if c["layout"] == "halves" else (2 * j, 2 * j + 1)


def _rotate(c, x, pos, turns, dtype, inverse=False):
    """x [..., D] at positions pos (x's shape without D, or what broadcasts to it)."""
    part = pos.to(torch.float64)[..., None] * turns
    angle = (part - torch.floor(part)) * (2 * math.pi)
    cos, sin = (angle.cos() * c["amplitude"]).to(dtype), (angle.sin() * c["amplitude"]).to(dtype)
    if inverse:
        sin = -sin
    i0, i1 = _partners(c)
    x = x.to(dtype)
    x0, x1 = x[..., i0], x[..., i1]
    y = x.clone()
    y[..., i0], y[..., i1] = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    return y


def _positions(s):
    c = s["c"]
    if s["pos"] is not None:
        return s["pos"][:, None, :]
    return (c["first"] + torch.arange(c["N"], device=DEV))[None, None, :]


def _plain_append(s, a):
    c = s["c"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    start = c["start"] if c["kind"] == "append" else c["N"]
    pos = (start + s["n"].to(torch.int64))[:, None]
    a["q"].copy_(_rotate(c, a["qkv"][:, :Hq], pos, s["turns"], torch.float32))
    b, n = torch.arange(c["B"], device=DEV), s["n"].to(torch.int64)
    a["Kt"][b, :, n] = _rotate(c, a["qkv"][:, Hq:Hq + Hkv], pos, s["turns"], torch.float32).to(torch.bfloat16)
    a["Vt"][b, :, n] = a["qkv"][:, Hq + Hkv:]


def _attended(c, a):
    """Tokens of the listed pages [Hkv, T] and which of them exist."""
    if a["pages"] is None:
        t = torch.arange(c["N"], device=DEV).expand(c["Hkv"], -1)
    else:
        t = (a["pages"].to(torch.int64)[:, :, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten(1)
    return t.clamp(max=c["N"] - 1), t < c["N"]


def _unpacked(c, a, t, dtype):
    """Values of tokens t [Hkv, T] with zeros for dropped groups: [Hkv, T, D]."""
    H, G = c["Hkv"], c["G"]
    m = torch.gather(a["mask"].to(torch.int64) & 0xffff, 1, t)[:, :, None]
    g = torch.arange(G, device=DEV)
    bit = (m >> g) & 1
    below = bit.cumsum(2) - bit
    slot = torch.gather(a["off"].to(torch.int64), 1, t)[:, :, None] + below
    h = torch.arange(H, device=DEV)[:, None, None]
    v = a["v"][h, slot.clamp(max=a["v"].shape[1] - 1)]
    return (v.to(dtype) * bit[..., None].to(dtype)).flatten(2)


def _attend(s, a, dtype, n):
    c = s["c"]
    B, Hkv, D = c["B"], c["Hkv"], c["D"]
    R = c["Hq"] // Hkv
    t, there = _attended(c, a)
    h = torch.arange(Hkv, device=DEV)[:, None]
    q = a["q"].to(dtype).view(B, Hkv, R, D) / math.sqrt(D)
    rows = q.transpose(0, 1).reshape(Hkv, B * R, D)
    k = a["K"][h, t].to(dtype).transpose(1, 2).contiguous()
    score = torch.bmm(rows, k).masked_fill(~there[:, None, :], -math.inf)
    top = score.amax(2)
    if s["cap"]:
        kt = a["Kt"].to(dtype).flatten(0, 1).transpose(1, 2).contiguous()
        behind = torch.arange(s["cap"], device=DEV)[None, :] >= n.to(torch.int64)[:, None]
        own_score = torch.bmm(q.reshape(B * Hkv, R, D), kt).view(B, Hkv, R, s["cap"])
        own_score = own_score.masked_fill(behind[:, None, None, :], -math.inf)
        top = torch.maximum(top, own_score.amax(3).transpose(0, 1).reshape(Hkv, B * R))
    w = torch.exp(score - top[:, :, None])
    total, out = w.sum(2), torch.bmm(w, _unpacked(c, a, t, dtype))
    if s["cap"]:
        w = torch.exp(own_score - top.view(Hkv, B, R).transpose(0, 1)[..., None])
        vt = torch.where(behind[:, None, :, None], 0.0, a["Vt"].to(dtype)).flatten(0, 1)
        mine = torch.bmm(w.view(B * Hkv, R, s["cap"]), vt).view(B, Hkv, R, D)
        out = out + mine.transpose(0, 1).reshape(Hkv, B * R, D)
        total = total + w.sum(3).transpose(0, 1).reshape(Hkv, B * R)
    out = out / total[:, :, None]
    return out.view(Hkv, B, R, D).transpose(0, 1).reshape(B, c["Hq"], D)


def run(state):
    s, c = state, state["c"]
    if own:
        return _run_own(s)
    if c["kind"] == "rotary":
        s["y"].copy_(_rotate(c, s["x"], _positions(s), s["turns"], torch.float32, c["inverse"]))
        return s["y"]
    if c["kind"] == "append":
        a = s["layers"][0]
        _plain_append(s, a)
        return dict(q=a["q"], K=a["Kt"], V=a["Vt"])
    got = []
    for a in s["layers"]:
        n = s["n"]
        if c["kind"] == "step":
            _plain_append(s, a)
            n = n + 1
        a["out"].copy_(_attend(s, a, torch.float32, n))
        got.append(dict(out=a["out"], q=a["q"], K=a["Kt"]) if c["kind"] == "step" else a["out"])
    return got


# --------------------------------------------------------------------------------------------
# The framework's calls
# --------------------------------------------------------------------------------------------
def _plan(s):
    """What a program keeps between steps: shape and workspace."""
    if "shape" not in s:
        import paper_2604_21335_amd as stc
        c = s["c"]
        s["stc"] = stc
        s["layout"] = stc.STC_ROTARY_HALVES if c["layout"] == "halves" else stc.STC_ROTARY_INTERLEAVED
        s["shape"] = s["ws"] = None
        if c["kind"] != "rotary":
            N, G = c.get("N", PAGE), c.get("G", 1)
            s["shape"] = stc.make_shape(c["B"], c["Hq"], c["Hkv"], c["D"], N, G, N * G)
        if c["kind"] in ("shared", "step"):
            need = stc.stc_shared_workspace_bytes(s["shape"], s["layers"][0]["k"], s["cap"])
            s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return s["stc"]


def _own_append(stc, s, a, n_out):
    c = s["c"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    stc.stc_rotary_append(s["shape"], a["qkv"][:, :Hq], a["qkv"][:, Hq:Hq + Hkv], a["qkv"][:, Hq + Hkv:],
                          a["q"], a["Kt"], a["Vt"], s["n"], s["cap"], s["turns"], c["rot"], s["layout"],
                          amplitude=c["amplitude"], pos0=c["start"] if c["kind"] == "append" else c["N"],
                          n_out=n_out)


def _run_own(s):
    stc, c = _plan(s), s["c"]
    if c["kind"] == "rotary":
        stc.stc_rotary(s["x"], s["y"], s["turns"], c["rot"], s["layout"], pos=s["pos"], pos0=c["first"],
                       amplitude=c["amplitude"], inverse=c["inverse"])
        return s["y"]
    if c["kind"] == "append":
        a = s["layers"][0]
        _own_append(stc, s, a, None)
        return dict(q=a["q"], K=a["Kt"], V=a["Vt"])
    got = []
    for a in s["layers"]:
        n = s["n"]
        if c["kind"] == "step":
            if "n1" not in s:
                s["n1"] = torch.empty_like(n)
            _own_append(stc, s, a, s["n1"])
            n = s["n1"]
        stc.stc_decode_attention_shared(s["shape"], a["q"], a["K"], a["v"], a["mask"], a["off"], a["pages"],
                                        a["k"], a.get("Kt"), a.get("Vt"), n, s["cap"], a["out"], s["ws"])
        got.append(dict(out=a["out"], q=a["q"], K=a["Kt"]) if c["kind"] == "step" else a["out"])
    return got


# --------------------------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------------------------
def _append_work(c):
    n = c["B"] * (c["Hq"] + 2 * c["Hkv"]) * c["D"]
    return 4 * n, 3 * c["B"] * (c["Hq"] + c["Hkv"]) * c["rot"]


def _attend_work(c):
    """The tails are half full in the mean."""
    T = min(c["N"], (c["k"] or c["N"]) * PAGE)
    kept = max(c["keep"], 1.0 / c["G"])
    tail = c["B"] * c["Hkv"] * c["tail"] / 2
    rows = c["B"] * c["Hq"]
    b = c["Hkv"] * T * (2 * c["D"] * (1 + kept) + 6) + tail * 4 * c["D"]
    b += rows * c["D"] * (2 + (2 if c["bf16"] else 4))
    return b, rows * 2 * c["D"] * (T * (1 + kept) + c["tail"])


def work(case):
    c = case
    if c["kind"] == "rotary":
        n = c["B"] * c["H"] * c["N"] * c["D"]
        return dict(bytes=4 * n + (4 * c["B"] * c["N"] if c["given"] else 0), flops=3 * n * c["rot"] // c["D"])
    b = f = 0
    if c["kind"] != "shared":
        b, f = _append_work(c)
    if c["kind"] != "append":
        b2, f2 = _attend_work(c)
        b, f = b + b2, f + f2
    n = c.get("layers", 1)
    return dict(bytes=b * n, flops=f * n)


# --------------------------------------------------------------------------------------------
# The definitions in 64 bits, head by head
# --------------------------------------------------------------------------------------------
def _exact_rotation(c, x, pos, inverse=False):
    """x [rows, D] float64 at positions [rows]: pairs as complex numbers times e^(i angle)."""
    turn = torch.remainder(pos.to(torch.float64)[:, None] * _turns(c)[None, :], 1.0)
    w = torch.polar(torch.full_like(turn, c["amplitude"]), 2 * math.pi * turn)
    if inverse:
        w = w.conj()
    r, half = c["rot"], c["rot"] // 2
    if c["layout"] == "halves":
        z = torch.complex(x[:, :half], x[:, half:r]) * w
        return torch.cat([z.real, z.imag, x[:, r:]], 1)
    z = torch.complex(x[:, 0:r:2], x[:, 1:r:2]) * w
    return torch.cat([torch.view_as_real(z).flatten(1), x[:, r:]], 1)


def _exact_attention(c, a, q, Kt, Vt, n):
    B, Hkv, D, N, G = c["B"], c["Hkv"], c["D"], c["N"], c["G"]
    R, gd = c["Hq"] // Hkv, c["D"] // c["G"]
    out = torch.empty(B, c["Hq"], D, dtype=torch.float64, device=DEV)
    for h in range(Hkv):
        # every kept group back to its place: kept pairs stand in token, then group order
        bits = (a["mask"][h].to(torch.int64)[:, None] >> torch.arange(G, device=DEV)) & 1
        tok, grp = bits.nonzero(as_tuple=True)
        V = torch.zeros(N, G, gd, dtype=torch.float64, device=DEV)
        V[tok, grp] = a["v"][h, :tok.numel()].double()
        V, K = V.view(N, D), a["K"][h].double()
        if a["pages"] is not None:
            on = torch.zeros((N + PAGE - 1) // PAGE, dtype=torch.bool, device=DEV)
            on[a["pages"][h].to(torch.int64)] = True
            on = on.repeat_interleave(PAGE)[:N]
            K, V = K[on], V[on]
        rows = q[:, h * R:(h + 1) * R].reshape(B * R, D).double()
        for r0 in range(0, B * R, 512):
            w = rows[r0:r0 + 512] @ K.t() / math.sqrt(D)
            m = w.amax(1, keepdim=True)
            w = torch.exp(w - m)
            l, o = w.sum(1, keepdim=True), w @ V
            if Kt is not None:
                b = torch.arange(r0, min(r0 + 512, B * R), device=DEV) // R
                for i in torch.unique(b).tolist():
                    k = int(n[i])
                    if k == 0:
                        continue
                    mine = b == i
                    x = rows[r0:r0 + 512][mine] @ Kt[i, h, :k].double().t() / math.sqrt(D)
                    m2 = torch.maximum(m[mine], x.amax(1, keepdim=True))
                    f, e = torch.exp(m[mine] - m2), torch.exp(x - m2)
                    l[mine] = l[mine] * f + e.sum(1, keepdim=True)
                    o[mine] = o[mine] * f + e @ Vt[i, h, :k].double()
            o = o / l
            for r in range(o.shape[0]):
                out[(r0 + r) // R, h * R + (r0 + r) % R] = o[r]
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rotary":
        B, H, N, D = c["B"], c["H"], c["N"], c["D"]
        y = torch.empty(B, H, N, D, dtype=torch.float64, device=DEV)
        for b in range(B):
            pos = s["pos"][b] if s["pos"] is not None else c["first"] + torch.arange(N, device=DEV)
            for h in range(H):
                y[b, h] = _exact_rotation(c, s["x"][b, h].double(), pos, c["inverse"])
        return y
    got = []
    for a in s["layers"]:
        q, Kt, Vt, n = a["q"], a.get("Kt"), a.get("Vt"), s["n"]
        Hq, Hkv = c["Hq"], c["Hkv"]
        if c["kind"] != "shared":
            pos = (c["start"] if c["kind"] == "append" else c["N"]) + n
            q, Kt = a["q"].double(), Kt.double()
            for h in range(Hq):
                q[:, h] = _exact_rotation(c, a["qkv"][:, h].double(), pos)
            for h in range(Hkv):
                k = _exact_rotation(c, a["qkv"][:, Hq + h].double(), pos)
                for b in range(c["B"]):
                    Kt[b, h, int(n[b])] = k[b]
                    Vt[b, h, int(n[b])] = a["qkv"][b, Hq + Hkv + h]
        if c["kind"] == "append":
            return dict(q=q, K=Kt, V=Vt.double())
        if c["kind"] == "step":
            # the attention reads what the step stores: rotated queries and keys in bf16
            out = _exact_attention(c, a, q.bfloat16(), Kt.bfloat16(), Vt, n + 1)
            got.append(dict(out=out, q=q, K=Kt))
        else:
            got.append(_exact_attention(c, a, q, Kt, Vt, n))
    return got
