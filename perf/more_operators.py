"""The operators of drafted tokens over a compressed cache, and what they are measured on.

Up to 64 tokens of a sequence are drafted as a tree: node t sees the nodes whose bits are set in
tree[t], its ancestors and itself (no tree: a chain).  `append`: rotary positions of the drafted tokens,
their keys and values to the rows behind the sequence's own tail.  `attend`: every node's query over a
compressed prefix (one for all sequences, or one each), the sequence's tail and the nodes that it sees.
`accept`: the accepted nodes move together, in place, the tail grows by them, in all layers at once.
`fork`: sequences take over others' tails (beams, samples, another try from an earlier token), in place,
in all layers at once.  `round`: the first three as one verification runs them, layer by layer.

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
        # A chain of 5 drafted tokens of one sequence: the smallest call, a launch and nothing else.
        _append(name="append_chain_of_5", B=1, T=5, Hq=32, Hkv=8, D=128, rot=128, tail=100, chain=True),
        # Trees of up to 63 nodes of 64 sequences of a Qwen2.5-7B-shaped layer, of different sizes, some
        # elements of the batch padding.
        _append(name="append_trees_batch", B=64, T=63, Hq=28, Hkv=4, D=128, rot=128, tail=300, base=1e6,
                ragged=True, padded=True),
        # 4 drafted tokens of 2 sequences over a short prompt, 8 heads of 64: the smallest attention.
        _attend_case(name="tree_tiny", B=2, T=4, Hq=8, Hkv=8, D=64, N=1024, G=4, keep=0.5, tail=8),
        # One sequence far into a 32768-token document, a tree of 64 nodes, Qwen2.5-7B-shaped layer:
        # what a single user waits for.
        _attend_case(name="tree_qwen25_7b_32k", B=1, T=64, Hq=28, Hkv=4, D=128, N=32768, G=8, keep=0.5,
                     tail=700),
        # The largest: 16 answers over the same document, 16 nodes each, of different sizes, bf16 output.
        _attend_case(name="tree_qwen25_7b_32k_b16", B=16, T=16, Hq=28, Hkv=4, D=128, N=32768, G=8, keep=0.5,
                     tail=300, bf16=True, ragged=True),
        # 8 prompts of their own, LLaMA-2-7B-shaped layer, 64 of 256 pages selected, 7 nodes.
        _attend_case(name="tree_llama2_7b_4k_own", B=8, T=7, Hq=32, Hkv=32, D=128, N=4096, G=8, keep=0.5,
                     tail=200, k=64, each=True),
        # 64 conversations about one image, 32 heads over 208 tokens, long tails, 6 nodes: tails count.
        _attend_case(name="tree_llava15_7b_prefix", B=64, T=6, Hq=32, Hkv=32, D=128, N=208, G=8, keep=0.55,
                     tail=1000, bf16=True, ragged=True, padded=True),
        # Accepted nodes of one layer of a small batch; then of all 28 layers of a Qwen2.5-7B-shaped model.
        _accept(name="accept_small", B=5, T=8, Hkv=8, D=128, tail=100),
        _accept(name="accept_28_layers", B=16, T=32, Hkv=4, D=128, tail=300, layers=28, padded=True),
        # Beams: 8 sequences of one layer change places after a token; 48 of 4 layers with long tails.
        _fork(name="fork_8_beams", B=8, Hkv=4, D=128, tail=120),
        # The largest move: a third of 48 sequences become copies of others, some from an earlier token on.
        _fork(name="fork_4_layers", B=48, Hkv=8, D=128, tail=1500, layers=4, rewind=True, padded=True),
        # A verification through 4 layers: 12 sequences, 13 nodes, a prefix that fills no tile, half of the
        # head rotated; then what was accepted moves together.
        _attend_case(name="round_4_layers", kind="round", B=12, T=13, Hq=32, Hkv=8, D=128, N=4001, G=8, keep=0.5,
                     tail=400, rot=64, layout="interleaved", layers=4, bf16=True, ragged=True),
    ]


def _base(**kw):
    d = dict(layout="halves", base=1e4, rot=0, layers=1, chain=False, ragged=False, padded=False, tail=0)
    d.update(kw)
    return d


def _append(**kw):
    return _base(**dict(dict(kind="append", start=1000), **kw))


def _attend_case(**kw):
    return _base(**dict(dict(kind="attend", k=0, bf16=False, each=False), **kw))


def _accept(**kw):
    return _base(**dict(dict(kind="accept", Hq=kw["Hkv"]), **kw))


def _fork(**kw):
    return _base(**dict(dict(kind="fork", Hq=kw["Hkv"], T=0, rewind=False), **kw))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "attend", "accept", "fork", "round"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 4, 8, 8, 32])
    R = rng.choice([1, 2, 4, 5, 7, 8, 16]) if Hkv <= 8 else 1
    T = rng.choice([1, _log(rng, 2, 64), _log(rng, 2, 64)])
    more = dict(chain=rng.random() < 0.3, ragged=rng.random() < 0.5, padded=rng.random() < 0.3)
    pairs = dict(rot=rng.choice([D, D, D // 2, 48]), layout=rng.choice(["halves", "interleaved"]),
                 base=rng.choice([1e4, 5e5, 1e6]))
    B = _log(rng, 1, 256)
    if kind == "append":
        tail = rng.randint(1, 512)
        B = max(1, min(B, (1 << 27) // (Hkv * (tail + T) * D), (1 << 26) // (T * Hkv * R * D)))
        return _append(B=B, T=T, Hq=Hkv * R, Hkv=Hkv, D=D, tail=tail, start=_log(rng, 1, 1000000), **pairs,
                       **more)
    if kind in ("accept", "fork"):
        layers = rng.choice([1, 1, 2, 4, 28])
        tail = _log(rng, 1, 2000)
        most = 48 * 8 * 128 * 1500 * 4 if kind == "fork" else 1 << 27
        B = max(1, min(B, most // (Hkv * D * (tail + T) * layers)))
        tail = max(1, min(tail, most // (Hkv * D * B * layers) - T))
        if kind == "accept":
            return _accept(B=B, T=T, Hkv=Hkv, D=D, tail=tail, layers=layers, chain=more["chain"],
                           padded=more["padded"])
        return _fork(B=B, Hkv=Hkv, D=D, tail=tail, layers=layers, rewind=rng.random() < 0.4,
                     padded=more["padded"])
    layers = 1 if kind == "attend" else rng.choice([1, 2, 3])
    each = rng.random() < 0.4
    keys = (3 << 24) // (Hkv * D * layers)                     # tokens of all prefixes
    N = _log(rng, 100, min(131072, keys))
    tail = _log(rng, 1, 1500)
    most = 256 * 28 * 32768 // 4 // layers                     # scores of a layer
    B = max(1, min(B, most // (Hkv * R * T * N), keys // N if each else B))
    T = max(1, min(T, most // (Hkv * R * N * B)))
    tail = max(1, min(tail, (1 << 27) // (Hkv * B * D * layers), most // (Hkv * R * T * B)))
    NP = (N + PAGE - 1) // PAGE
    if kind == "round":
        more.update(pairs)
    return _attend_case(kind=kind, B=B, T=T, Hq=Hkv * R, Hkv=Hkv, D=D, N=N, G=rng.choice([4, 8, 8, 16 if D == 128 else 2]),
                        keep=rng.choice([0.25, 0.375, 0.5, 0.5625, 0.75]), tail=tail,
                        k=0 if rng.random() < 0.6 else max(1, int(NP * rng.uniform(0.05, 0.5))),
                        bf16=kind == "round" or rng.random() < 0.5, each=each, layers=layers, **more)


# --------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------
def _turns(c):
    """Revolutions per position of every rotated pair, in 64 bits."""
    j = np.arange(c["rot"] // 2, dtype=np.float64)
    return torch.from_numpy(c["base"] ** (-2.0 * j / c["rot"]) / (2 * math.pi)).to(DEV)


def _normal(g, *shape):
    x = torch.empty(*shape, dtype=torch.bfloat16, device=DEV)
    return x.normal_(generator=g)


def _outliers(g, x):
    """Four channels per head times 8; x [B, H, tokens, D], heads of all b alike."""
    H, D = x.shape[1], x.shape[-1]
    at = torch.rand(H, D, generator=g, device=DEV).argsort(dim=1)[:, :4]
    s = torch.ones(H, D, device=DEV).scatter_(1, at, 8.0).to(x.dtype)
    return x.mul_(s[:, None, :])


def _trees(c, rng):
    """Sets of visible nodes [B, T] as int64: a node's parent is one of the 8 nodes before it."""
    B, T = c["B"], c["T"]
    seen = np.zeros((B, T), dtype=np.uint64)
    for t in range(T):
        seen[:, t] = np.uint64(1) << np.uint64(t)
        if t:
            low = t - 1 if c["chain"] else max(0, t - 8)
            seen[:, t] |= seen[np.arange(B), rng.integers(low, t, size=B)]
    return seen.view(np.int64)


def _prefix(g, c):
    """One layer's compressed prefixes, as the framework's cache construction leaves them."""
    P, H, N, G, D = c["B"] if c["each"] else 1, c["Hkv"], c["N"], c["G"], c["D"]
    K = _outliers(g, _normal(g, P, H, N, D))
    n = 1 + torch.binomial(torch.full((P, H, N), float(G - 1), device=DEV),
                           torch.full((P, H, N), (G * c["keep"] - 1) / (G - 1), device=DEV).clamp(0, 1),
                           generator=g)
    rank = torch.rand(P, H, N, G, generator=g, device=DEV).argsort(dim=3).argsort(dim=3)
    kept = rank < n[..., None]                                 # at least one group, G * keep in the mean
    mask = (kept.to(torch.int32) << torch.arange(G, device=DEV, dtype=torch.int32)).sum(3)
    off = torch.zeros(P, H, N + 1, dtype=torch.int64, device=DEV)
    off[..., 1:] = kept.sum(3).cumsum(2)
    v = _normal(g, P, H, N * G, D // G)
    pages = None
    if c["k"]:
        NP = (N + PAGE - 1) // PAGE
        pages = torch.rand(P, H, NP, generator=g, device=DEV).argsort(dim=2)[..., :c["k"]].sort(dim=2)[0]
        pages = pages.to(torch.int32).contiguous()
    return dict(K=K, mask=mask.to(torch.int16), off=off.to(torch.int32), v=v, pages=pages)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = np.random.default_rng(seed)
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    cap = c["tail"] + T
    n = rng.integers(0, c["tail"] + 1, size=B)
    n[0] = c["tail"]
    if c["padded"]:
        n[rng.random(B) < 0.1] = -1
        n[0] = c["tail"]
    s = dict(c=c, cap=cap, n=torch.from_numpy(n.astype(np.int32)).to(DEV), tree=None, drafted=None,
             n1=torch.zeros(c["layers"], B, dtype=torch.int32, device=DEV), layers=[])
    if c["rot"]:
        s["turns"] = _turns(c)
    if T:
        seen = _trees(c, rng)
        drafted = rng.integers(1, T + 1, size=B) if c["ragged"] else np.full(B, T)
        last = rng.integers(0, drafted)                        # the last accepted node
        s["keep"] = torch.from_numpy(seen[np.arange(B), last]).to(DEV)
        if not c["chain"]:
            s["tree"] = torch.from_numpy(seen).to(DEV)
        if c["ragged"]:
            s["drafted"] = torch.from_numpy(drafted.astype(np.int32)).to(DEV)
    if c["kind"] == "fork":
        src = np.arange(B)
        moved = rng.random(B) < (1.0 if B <= 8 else 1.0 / 3.0)  # few beams: a new choice of all
        src[moved] = rng.integers(0, B, size=moved.sum())
        if c["padded"]:
            src[rng.random(B) < 0.05] = -1                     # ended
        s["src"] = torch.from_numpy(src.astype(np.int32)).to(DEV)
        s["kept"] = None
        if c["rewind"]:
            kept = np.where(rng.random(B) < 0.5, c["tail"], rng.integers(0, c["tail"] + 1, size=B))
            s["kept"] = torch.from_numpy(kept.astype(np.int32)).to(DEV)
    for _ in range(c["layers"]):
        a = {}
        if c["kind"] in ("attend", "round"):
            a.update(_prefix(g, c))
            a["q"] = _normal(g, B, T, Hq, D)
            a["out"] = torch.zeros(B, T, Hq, D, dtype=torch.bfloat16 if c["bf16"] else torch.float32,
                                   device=DEV)
        a["Kt"] = _outliers(g, _normal(g, B, Hkv, cap, D))
        a["Vt"] = _normal(g, B, Hkv, cap, D)
        if c["kind"] in ("append", "round"):
            a["qkv"] = _normal(g, B, T, Hq + 2 * Hkv, D)       # what the fused projection leaves
            a["q"] = torch.zeros(B, T, Hq, D, dtype=torch.bfloat16, device=DEV)
        s["layers"].append(a)
    return s


# --------------------------------------------------------------------------------------------
# The plain forms
# --------------------------------------------------------------------------------------------
def _sees(s):
    """[B, T, T]: node t sees node u, of those that are drafted."""
    c = s["c"]
    u = torch.arange(c["T"], device=DEV)
    if s["tree"] is None:
        see = (u[None, :] <= u[:, None]).expand(c["B"], -1, -1)
    else:
        see = ((s["tree"][:, :, None] >> u) & 1) != 0
    if s["drafted"] is not None:
        see = see & (u < s["drafted"][:, None])[:, None, :]
    return see


def _drafted(s):
    """[B, T]: the nodes that are there."""
    c = s["c"]
    on = (s["n"] >= 0)[:, None].expand(-1, c["T"])
    if s["drafted"] is not None:
        on = on & (torch.arange(c["T"], device=DEV) < s["drafted"][:, None])
    return on


def _plain_append(s, a):
    c = s["c"]
    Hq, Hkv, T = c["Hq"], c["Hkv"], c["T"]
    t = torch.arange(T, device=DEV)
    if s["tree"] is None:
        depth = t.expand(c["B"], -1)
    else:
        depth = (((s["tree"][:, :, None] >> t) & 1) * (t[None, :] < t[:, None])).sum(2)
    pos = (c["start"] if c["kind"] == "append" else c["N"]) + s["n"].to(torch.int64)[:, None] + depth
    part = pos.to(torch.float64)[..., None] * s["turns"]
    angle = (part - torch.floor(part)) * (2 * math.pi)
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    j = torch.arange(c["rot"] // 2, device=DEV)
    i0, i1 = (j, j + c["rot"] // 2) if c["layout"] == "halves" else (2 * j, 2 * j + 1)
    x = a["qkv"][:, :, :Hq + Hkv].float()
    x0, x1 = x[..., i0], x[..., i1]
    y = x.clone()
    y[..., i0], y[..., i1] = x0 * cos - x1 * sin, x0 * sin + x1 * cos
    y = y.to(torch.bfloat16)
    on = _drafted(s)
    a["q"].copy_(torch.where(on[:, :, None, None], y[:, :, :Hq], a["q"]))
    b, t = on.nonzero(as_tuple=True)
    row = s["n"].to(torch.int64)[b] + t
    a["Kt"][b, :, row] = y[b, t, Hq:]
    a["Vt"][b, :, row] = a["qkv"][b, t, Hq + Hkv:]


def _attended(c, a):
    """Tokens of the listed pages [prefixes * Hkv, tokens] and which of them exist."""
    streams = a["K"].shape[0] * c["Hkv"]
    if a["pages"] is None:
        t = torch.arange(c["N"], device=DEV).expand(streams, -1)
    else:
        t = (a["pages"].to(torch.int64).flatten(0, 1)[:, :, None] * PAGE +
             torch.arange(PAGE, device=DEV)).flatten(1)
    return t.clamp(max=c["N"] - 1), t < c["N"]


def _unpacked(c, a, t):
    """Values of tokens t with zeros for dropped groups: [streams, tokens, D]."""
    m = torch.gather(a["mask"].flatten(0, 1).to(torch.int64) & 0xffff, 1, t)[:, :, None]
    bit = (m >> torch.arange(c["G"], device=DEV)) & 1
    slot = torch.gather(a["off"].flatten(0, 1).to(torch.int64), 1, t)[:, :, None] + bit.cumsum(2) - bit
    v = a["v"].flatten(0, 1)
    h = torch.arange(v.shape[0], device=DEV)[:, None, None]
    return (v[h, slot.clamp(max=v.shape[1] - 1)].float() * bit[..., None]).flatten(2)


def _plain_attend(s, a):
    c = s["c"]
    B, T, Hkv, D = c["B"], c["T"], c["Hkv"], c["D"]
    R, P = c["Hq"] // Hkv, a["K"].shape[0]
    t, there = _attended(c, a)
    q = a["q"].float().view(B, T, Hkv, R, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * R, D) / math.sqrt(D)

    def by_prefix(x):       # rows of all sequences that share a prefix, head by head
        return x.view(P, B // P, Hkv, T * R, -1).transpose(1, 2).reshape(P * Hkv, B // P * T * R, x.shape[-1])

    def by_sequence(x):
        return x.view(P, Hkv, B // P, T * R, -1).transpose(1, 2).reshape(B, Hkv, T * R, x.shape[-1])
    h = torch.arange(P * Hkv, device=DEV)[:, None]
    k = a["K"].flatten(0, 1)[h, t].float().transpose(1, 2).contiguous()
    score = torch.bmm(by_prefix(q), k).masked_fill(~there[:, None, :], -math.inf)
    # rows of the tail: committed ones, then nodes
    n = s["n"].to(torch.int64)
    j = torch.arange(s["cap"], device=DEV)
    node = j[None, :] - n[:, None]                                               # [B, cap]
    visible = torch.gather(_sees(s), 2, node.clamp(0, T - 1)[:, None, :].expand(-1, T, -1))
    visible = (node < 0)[:, None, :] | (visible & (node < T)[:, None, :])        # [B, T, cap]
    kt = a["Kt"].float().flatten(0, 1).transpose(1, 2).contiguous()
    mine = torch.bmm(q.flatten(0, 1), kt).view(B, Hkv, T, R, s["cap"])
    mine = mine.masked_fill(~visible[:, None, :, None, :], -math.inf).view(B, Hkv, T * R, s["cap"])
    top = torch.maximum(by_sequence(score.amax(2, keepdim=True)), mine.amax(3, keepdim=True))
    w = torch.exp(score - by_prefix(top))
    total, out = by_sequence(w.sum(2, keepdim=True)), by_sequence(torch.bmm(w, _unpacked(c, a, t)))
    w = torch.exp(mine - top)
    total = total + w.sum(3, keepdim=True)
    out = out + torch.bmm(w.flatten(0, 1), a["Vt"].float().flatten(0, 1)).view_as(out)
    out = (out / total).view(B, Hkv, T, R, D).permute(0, 2, 1, 3, 4).reshape(B, T, c["Hq"], D)
    a["out"].copy_(torch.where(_drafted(s)[:, :, None, None], out.to(a["out"].dtype), a["out"]))


def _plain_accept(s):
    """Sources of the kept nodes first, in order: a stable sort by what is dropped."""
    c = s["c"]
    u = torch.arange(c["T"], device=DEV)
    kept = (((s["keep"][:, None] >> u) & 1) != 0) & (s["n"] >= 0)[:, None]
    node = torch.sort((~kept).to(torch.int8), dim=1, stable=True)[1]
    count = kept.sum(1)
    b, i = (u < count[:, None]).nonzero(as_tuple=True)
    first = s["n"].to(torch.int64)[b]
    for a in s["layers"]:
        for x in (a["Kt"], a["Vt"]):
            x[b, :, first + i] = x[b, :, first + node[b, i]]
    s["n1"].copy_((s["n"] + count.to(torch.int32)).expand_as(s["n1"]))


def _plain_fork(s):
    src = s["src"].to(torch.int64)
    b = torch.arange(s["c"]["B"], device=DEV)
    at = src.clamp(min=0)
    n = s["n"][at]
    if s["kept"] is not None:
        n = torch.where(n >= 0, torch.minimum(n, s["kept"]), n)
    n = torch.where(src == -1, -1, n).to(torch.int32)
    j = torch.arange(s["cap"], device=DEV)
    moved = ((j[None, :] < n[:, None]) & (src != b)[:, None])[:, None, :, None]
    for a in s["layers"]:
        for x in (a["Kt"], a["Vt"]):
            x.copy_(torch.where(moved, x[at], x))
    s["n1"].copy_(n.expand_as(s["n1"]))


def _outputs(s):
    kind, got = s["c"]["kind"], []
    for a in s["layers"]:
        if kind == "attend":
            got.append(dict(out=a["out"]))
        elif kind == "append":
            got.append(dict(q=a["q"], K=a["Kt"], V=a["Vt"]))
        elif kind == "round":
            got.append(dict(out=a["out"], q=a["q"], K=a["Kt"], V=a["Vt"]))
        else:
            got.append(dict(K=a["Kt"], V=a["Vt"]))
    return dict(layers=got, n=s["n1"]) if kind in ("accept", "fork", "round") else got


def run(state):
    s, kind = state, state["c"]["kind"]
    if own:
        _run_own(s)
        return _outputs(s)
    for a in s["layers"]:
        if kind in ("append", "round"):
            _plain_append(s, a)
        if kind in ("attend", "round"):
            _plain_attend(s, a)
    if kind in ("accept", "round"):
        _plain_accept(s)
    elif kind == "fork":
        _plain_fork(s)
    return _outputs(s)


# --------------------------------------------------------------------------------------------
# The framework's calls
# --------------------------------------------------------------------------------------------
def _plan(s):
    """What a program keeps between steps: shape, workspace, the layers' tails."""
    if "shape" not in s:
        import paper_2604_21335_amd as stc
        c = s["c"]
        s["stc"] = stc
        N, G = c.get("N", PAGE), c.get("G", 1)
        s["shape"] = stc.make_shape(c["B"], c["Hq"], c["Hkv"], c["D"], N, G, N * G)
        s["layout"] = stc.STC_ROTARY_HALVES if c["layout"] == "halves" else stc.STC_ROTARY_INTERLEAVED
        s["Kts"], s["Vts"] = [a["Kt"] for a in s["layers"]], [a["Vt"] for a in s["layers"]]
        s["ns"], s["n1s"] = [s["n"]] * c["layers"], list(s["n1"])
        if c["kind"] in ("attend", "round"):
            s["prefixes"] = c["B"] if c["each"] else 1
            s["k"] = c["k"] or (N + PAGE - 1) // PAGE
            need = stc.stc_tree_workspace_bytes(s["shape"], c["T"], s["k"], s["cap"], n_prefix=s["prefixes"])
            s["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return s["stc"]


def _run_own(s):
    stc, c = _plan(s), s["c"]
    kind, Hq, Hkv = c["kind"], c["Hq"], c["Hkv"]
    for a in s["layers"]:
        if kind in ("append", "round"):
            stc.stc_rotary_append_tree(
                s["shape"], a["qkv"][:, :, :Hq], a["qkv"][:, :, Hq:Hq + Hkv], a["qkv"][:, :, Hq + Hkv:], a["q"],
                a["Kt"], a["Vt"], s["n"], s["cap"], s["turns"], c["rot"], s["layout"], tree=s["tree"],
                n_draft=s["drafted"], pos0=c["start"] if kind == "append" else c["N"])
        if kind in ("attend", "round"):
            stc.stc_decode_attention_tree(
                s["shape"], a["q"], a["K"], a["v"], a["mask"], a["off"], a["pages"], s["k"], a["Kt"], a["Vt"],
                s["n"], s["cap"], a["out"], s["ws"], tree=s["tree"], n_draft=s["drafted"],
                n_prefix=s["prefixes"])
    if kind in ("accept", "round"):
        stc.stc_accept_tail(s["shape"], c["T"], s["Kts"], s["Vts"], s["ns"], s["cap"], s["keep"],
                            n_outs=s["n1s"])
    elif kind == "fork":
        stc.stc_fork_tail(s["shape"], s["Kts"], s["Vts"], s["ns"], s["cap"], s["src"], n_keep=s["kept"],
                          n_outs=s["n1s"])


# --------------------------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------------------------
def work(case):
    """Tails are half full in the mean, ragged trees half as large, a path takes half of a chain's nodes
    and the depth of a tree whose parents lie 4 nodes back."""
    c = case
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    nodes = B * T / (2.0 if c["ragged"] else 1.0)
    b = f = 0.0
    if c["kind"] in ("append", "round"):
        b += 4 * nodes * (Hq + 2 * Hkv) * D
        f += 3 * nodes * (Hq + Hkv) * c["rot"]
    if c["kind"] in ("attend", "round"):
        P = B if c["each"] else 1
        n = min(c["N"], (c["k"] or c["N"]) * PAGE)
        kept = max(c["keep"], 1.0 / c["G"])
        mine = c["tail"] / 2.0
        b += P * Hkv * n * (2 * D * (1 + kept) + 6) + (B * mine + nodes) * Hkv * 4 * D
        b += nodes * Hq * D * (2 + (2 if c["bf16"] else 4))
        f += nodes * Hq * 2 * D * (n * (1 + kept) + 2 * mine + T / (1.0 if c["chain"] else 4.0))
    if c["kind"] in ("accept", "round"):
        moved = 0 if c["chain"] else T / 8.0
        b += 8.0 * B * Hkv * D * moved + 8.0 * B
    if c["kind"] == "fork":
        share = (1.0 if B <= 8 else 1.0 / 3.0) * (1 - 1.0 / B) * (0.9 if c["padded"] else 1.0)
        b += 8.0 * B * share * Hkv * D * c["tail"] / 2.0 * (0.65 if c["rewind"] else 1.0) + 12.0 * B
    return dict(bytes=max(b, 8.0) * c["layers"], flops=f * c["layers"])


# --------------------------------------------------------------------------------------------
# The definitions in 64 bits, sequence by sequence and head by head
# --------------------------------------------------------------------------------------------
def _bits(x):
    x = int(x) & 0xFFFFFFFFFFFFFFFF
    return [i for i in range(64) if x >> i & 1]


def _exact_rotation(c, x, pos, turns):
    """x [heads, D] float64 at one position: pairs as complex numbers times e^(i angle)."""
    turn = torch.remainder(pos * turns, 1.0)
    w = torch.polar(torch.ones_like(turn), 2 * math.pi * turn)
    r, half = c["rot"], c["rot"] // 2
    if c["layout"] == "halves":
        z = torch.complex(x[:, :half], x[:, half:r]) * w
        return torch.cat([z.real, z.imag, x[:, r:]], 1)
    z = torch.complex(x[:, 0:r:2], x[:, 1:r:2]) * w
    return torch.cat([torch.view_as_real(z).flatten(1), x[:, r:]], 1)


def _exact_append(c, a, n, drafted, trees):
    Hq, Hkv = c["Hq"], c["Hkv"]
    q, K, turns = a["q"].double(), a["Kt"].double(), _turns(c)
    for b in range(c["B"]):
        if n[b] < 0:
            continue
        for t in range(drafted[b]):
            pos = (c["start"] if c["kind"] == "append" else c["N"]) + n[b] + sum(u < t for u in trees[b][t])
            x = _exact_rotation(c, a["qkv"][b, t, :Hq + Hkv].double(), float(pos), turns)
            q[b, t], K[b, :, n[b] + t] = x[:Hq], x[Hq:]
            a["Vt"][b, :, n[b] + t] = a["qkv"][b, t, Hq + Hkv:]
    return q, K


def _exact_attention(c, a, q, Kt, Vt, n, drafted, trees):
    """Heads of one prefix: keys and values of the attended tokens once, then a sequence at a time."""
    B, T, Hkv, D, N, G = c["B"], c["T"], c["Hkv"], c["D"], c["N"], c["G"]
    R, P = c["Hq"] // Hkv, a["K"].shape[0]
    out = a["out"].double()
    for p in range(P):
        for h in range(Hkv):
            # every kept group back to its place: kept pairs stand in token, then group order
            held = (a["mask"][p, h].to(torch.int64)[:, None] >> torch.arange(G, device=DEV)) & 1
            tok, grp = held.nonzero(as_tuple=True)
            V = torch.zeros(N, G, D // G, dtype=torch.float64, device=DEV)
            V[tok, grp] = a["v"][p, h, :tok.numel()].double()
            V, K = V.view(N, D), a["K"][p, h].double()
            if a["pages"] is not None:
                on = torch.zeros((N + PAGE - 1) // PAGE, dtype=torch.bool, device=DEV)
                on[a["pages"][p, h].to(torch.int64)] = True
                on = on.repeat_interleave(PAGE)[:N]
                K, V = K[on], V[on]
            for b in range(p * (B // P), (p + 1) * (B // P)):
                if n[b] < 0:
                    continue
                m = drafted[b]
                rows = q[b, :m, h * R:(h + 1) * R].reshape(m * R, D).double()
                hide = torch.full((m, n[b] + m), -math.inf, dtype=torch.float64)
                hide[:, :n[b]] = 0
                for t in range(m):
                    hide[t, [n[b] + u for u in trees[b][t] if u < m]] = 0
                hide = hide.to(DEV).repeat_interleave(R, 0)
                x = torch.cat([rows @ K.t(), rows @ Kt[b, h, :n[b] + m].double().t()], 1) / math.sqrt(D)
                x[:, K.shape[0]:] += hide
                w = torch.softmax(x, 1)
                got = w[:, :K.shape[0]] @ V + w[:, K.shape[0]:] @ Vt[b, h, :n[b] + m].double()
                out[b, :m, h * R:(h + 1) * R] = got.view(m, R, D)
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, T, kind = c["B"], c["T"], c["kind"]
    n = s["n"].tolist()
    drafted = s["drafted"].tolist() if s["drafted"] is not None else [T] * B
    seen = s["tree"].tolist() if s["tree"] is not None else [[(2 << t) - 1 for t in range(T)]] * B
    trees = [[_bits(x) for x in row] for row in seen]
    got = []
    for a in s["layers"]:
        q, K = a.get("q"), a["Kt"].double()
        if kind in ("append", "round"):
            q, K = _exact_append(c, a, n, drafted, trees)
        out = None
        if kind in ("attend", "round"):
            # the attention reads what the append stores: rotated queries and keys in bf16
            out = _exact_attention(c, a, q.bfloat16(), K.bfloat16(), a["Vt"], n, drafted, trees)
        V = a["Vt"].double()
        if kind in ("accept", "round"):
            for b in range(B):
                for i, t in enumerate(_bits(s["keep"][b]) if n[b] >= 0 else []):
                    K[b, :, n[b] + i], V[b, :, n[b] + i] = K[b, :, n[b] + t], V[b, :, n[b] + t]
        if kind == "fork":
            old = K.clone(), V.clone()
            for b, f in enumerate(s["src"].tolist()):
                if f >= 0 and f != b and n[f] > 0:
                    m = n[f] if s["kept"] is None else min(n[f], int(s["kept"][b]))
                    K[b, :, :m], V[b, :, :m] = old[0][f, :, :m], old[1][f, :, :m]
        got.append({"attend": dict(out=out), "append": dict(q=q, K=K, V=V), "accept": dict(K=K, V=V),
                    "fork": dict(K=K, V=V), "round": dict(out=out, q=q, K=K, V=V)}[kind])
    return dict(layers=got, n=None) if kind in ("accept", "fork", "round") else got
