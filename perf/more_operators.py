"""What stands around softmax attention when a hybrid model is served with drafted tokens, as cases that can be timed and compared.

Softmax attention is in the layers that the linearized layer is distilled from and in those that a hybrid keeps. Its queries
and keys carry rotary positions; and a serving loop that has several tokens drafted per step needs all of them verified by one
pass over the cache, and the accepted ones' keys and values put into it. The operators:

rotary positions (forward and gradient): the leading `rot` channels of a head form rot / 2 pairs, (i, i + rot / 2) in the half layout and
(2 i, 2 i + 1) in the interleaved one; pair i of a token at position n is turned by the angle n f_i and multiplied by m:
    (x, y) -> m (x cos a - y sin a, x sin a + y cos a),  a = n f_i,  f_i = base^(-2 i / rot), slowed down for long contexts:
    by wavelength: with r = original f_i / (2 pi) turns over the original length, w = clamp((r - low) / (high - low), 0, 1):
        f_i (w + (1 - w) / factor)
    by channel: with c(r) = rot ln(original / (2 pi r)) / (2 ln base), a = max(0, floor c(high)), z = min(rot - 1, ceil c(low)),
        w = 1 - clamp((i - a) / max(z - a, 0.001), 0, 1): f_i (w + (1 - w) / factor)
The other channels stay as they are. The gradient turns the other way.

attention of drafted tokens: N nodes per sequence, each with a parent (an earlier node, -1: the sequence's last token; anything else
than those: neither it nor what hangs from it is there, its output is 0). A node of depth e (0 behind the last token) stands at position
pos + e and sees what a step-by-step generation would have it see: the cached positions j in [pos - C, pos) and the nodes of its path, itself
included, that lie less than W (the window, or the C slots of the ring) behind it. Scores as in the attention of this framework:
    u = q.k / sqrt(d), cap tanh(u / cap) where asked, less slope times the distance where asked.
The same over a cache held in 4 bits, where a node's key and value are what the cache would hold of them.

accepting: the keys and values of a path of nodes (a list per sequence, up to its first negative entry) go to slots pos, pos + 1, ... of the
ring, in the storage type or in 4 bits; the new position comes back.

A case is a dict of plain values; `kind` is rope | rope_train | tree | tree_quant | accept | accept_quant.
"""
import math
import random

import torch


own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SMALL = dict(H=32, H_kv=8, d=64)    # the 1B shape
LARGE = dict(H=32, H_kv=8, d=128)   # the 7B shape
BASE = 10000.0


def _api():
    from paper_2509_18467_b200 import api
    return api


def _rope(name, kind, dtype, B, T, last, docs="", layout="half", rot=0, scaling="", factor=1.0, original=0, **heads):
    c = dict(kind=kind, dtype=dtype, B=B, T=T, last=last, docs=docs, layout=layout, rot=rot or heads["d"], scaling=scaling, factor=factor,
             original=original, **heads)
    return dict(name=name, **c) if name else c


def _tree(name, kind, B, N, C, last, shape="tree", window=0, cap=0.0, slopes=False, dtype="bf16", M=0, **heads):
    c = dict(kind=kind, dtype=dtype, B=B, N=N, C=C, last=last, shape=shape, window=window, cap=cap, slopes=slopes, M=M, **heads)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one token for each of a serving batch, far out in a context that was stretched sixteen times: all launches and latency
        _rope("rope-step", "rope", "bf16", 64, 1, 131072, scaling="channel", factor=16.0, original=8192, **LARGE),
        # queries and keys of a whole 32K-token prompt, in a context that was stretched eight times
        _rope("rope-prompt", "rope", "bf16", 1, 32768, 0, scaling="wavelength", factor=8.0, original=4096, **LARGE),
        # the four training lengths as documents of one packed sequence, half of each head turned: forward and gradient
        _rope("rope-train", "rope_train", "bf16", 1, 4856, 0, docs="1162,1171,1223,1300", layout="interleaved", rot=32, **SMALL),
        # one conversation, five tokens drafted in a row
        _tree("tree-one", "tree", 1, 5, 8192, 8190, shape="chain", **LARGE),
        # a serving batch of 16 sequences of different lengths, a tree of 32 tokens for each
        _tree("tree-batch", "tree", 16, 32, 8192, 8190, **LARGE),
        # the largest product here: wide trees with distance biases and capped scores, at width 64
        _tree("tree-wide", "tree", 8, 64, 8192, 8190, cap=30.0, slopes=True, **SMALL),
        # a sliding-window layer (window 64): a short ring that has wrapped, a tree for each of eight sequences
        _tree("tree-window", "tree", 8, 26, 64, 1223, window=64, **SMALL),
        # the small exact configuration in fp32
        _tree("tree-fp32", "tree", 2, 13, 512, 500, dtype="f32", H=4, H_kv=4, d=64),
        # one sequence over a long past held in 4 bits
        _tree("tree-quant-one", "tree_quant", 1, 16, 32768, 32700, slopes=True, **LARGE),
        # a serving batch over pasts held in 4 bits, eight tokens drafted for each
        _tree("tree-quant-batch", "tree_quant", 64, 8, 16384, 16383, **LARGE),
        # the accepted tokens of a serving batch go into their rings
        _tree("accept-batch", "accept", 64, 32, 1300, 1290, M=8, **LARGE),
        # the same into a cache in 4 bits
        _tree("accept-quant", "accept_quant", 16, 64, 1300, 1290, M=12, **SMALL),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "rope_train", "tree", "tree", "tree", "tree", "tree_quant", "tree_quant", "accept", "accept_quant"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"]) if kind != "tree_quant" else "bf16"
    d = rng.choice([64, 128])
    H_kv = rng.choice([1, 2, 4, 8])
    H = H_kv * rng.choice([1, 2, 4, 8][:3 if H_kv == 8 else 4])
    heads = dict(H=H, H_kv=H_kv, d=d)
    if kind in ("rope", "rope_train"):
        B = rng.choice([1, 1, 2, 8, 64])
        T = _log(rng, 1, (32768 if kind == "rope" and dtype == "bf16" else 8192) // B)
        rot = rng.choice([d, d, d // 2, d // 4])
        scaling = rng.choice(["", "wavelength", "channel"])
        docs = ""
        if B == 1 and T >= 8 and rng.random() < 0.4:
            cuts = sorted(rng.randint(0, T) for _ in range(rng.randint(1, 7)))
            docs = ",".join(str(y - x) for x, y in zip([0] + cuts, cuts + [T]))
        return _rope("", kind, dtype, B, T, rng.choice([0, _log(rng, 1, 131072)]), docs=docs, layout=rng.choice(["half", "interleaved"]), rot=rot,
                     scaling=scaling, factor=rng.choice([2.0, 8.0, 32.0]) if scaling else 1.0, original=rng.choice([2048, 4096, 8192]) if scaling else 0, **heads)
    C = _log(rng, 64, 1500 if dtype == "f32" or kind.startswith("accept") else 8192)
    window = rng.choice([0, 0, _log(rng, 1, C)])
    N = _log(rng, 1, 64)
    return _tree("", kind, rng.randint(1, min(16, 384 // N)) if dtype == "bf16" else rng.randint(1, 4), N, C, _log(rng, 1, 2 * C), shape=rng.choice(["tree", "tree", "chain"]),
                 window=window, cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=rng.random() < 0.3, dtype=dtype,
                 M=min(N, _log(rng, 1, 12)) if kind.startswith("accept") else 0, **heads)


# ------------------------------------------------------------------------------------------------ what a case's names stand for
def _freq(c):
    """Host list: the angle per token of each pair; and the factor of the turned values."""
    rot, base, factor, original = c["rot"], BASE, c["factor"], c["original"]
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if c["scaling"] == "wavelength":
        low, high = 1.0, 4.0
        w = [min(1.0, max(0.0, (original * x / (2 * math.pi) - low) / (high - low))) for x in f]
    elif c["scaling"] == "channel":
        low, high = 1.0, 32.0
        at = lambda r: rot * math.log(original / (2 * math.pi * r)) / (2 * math.log(base))  # noqa: E731
        a, z = max(0, math.floor(at(high))), min(rot - 1, math.ceil(at(low)))
        w = [1.0 - min(1.0, max(0.0, (i - a) / max(z - a, 0.001))) for i in range(rot // 2)]
    else:
        return f, 1.0
    return [x * (v + (1 - v) / factor) for x, v in zip(f, w)], 0.1 * math.log(factor) + 1.0 if c["scaling"] == "channel" else 1.0


def _starts(c):
    """Host list: the position that each sequence begins at (rope: of its first token; tree: of the first token that is not cached):
    ragged, from `last` down to a half of it."""
    return [max(0, c["last"] - (c["last"] // 2) * ((7 * b) % 16) // 15) for b in range(c["B"])]


def _positions(c):
    """Host list of lists [B][T] of a rope case: they start over with each packed document."""
    if c["docs"]:
        return [[t for n in c["docs"].split(",") for t in range(int(n))]]
    return [list(range(p, p + c["T"])) for p in _starts(c)]


def _parents(c, seed):
    """Host list of lists [B][N]. A chain has each node behind the one in front; a tree has a few nodes per depth, as the most likely
    continuations give it (depth 8 at most), and its last nodes are missing in some sequences (a padded batch)."""
    rng, out = random.Random(seed), []
    for b in range(c["B"]):
        if c["shape"] == "chain":
            out.append([i - 1 for i in range(c["N"])])
            continue
        row, depth = [], []
        there = c["N"] if b % 3 else max(1, c["N"] - rng.randint(0, c["N"] // 4))
        for i in range(c["N"]):
            p = -1 if i == 0 or rng.random() < 0.1 else rng.randint(max(0, i - 8), i - 1)
            while p >= 0 and depth[p] >= 7:
                p = row[p]
            row.append(p)
            depth.append(depth[p] + 1 if p >= 0 else 0)
        out.append(row[:there] + [-2] * (c["N"] - there))
    return out


def _paths(parents, M, seed):
    """Host list of lists [B][M]: for each sequence a path from a root down, padded with -1 (in one of eight nothing is accepted)."""
    rng, out = random.Random(seed + 1), []
    for b, row in enumerate(parents):
        n = rng.choice([i for i, p in enumerate(row) if p >= -1])
        path = []
        while n >= 0:
            path.append(n)
            n = row[n]
        path = path[::-1][:M] if b % 8 != 5 else []
        out.append(path + [-1] * (M - len(path)))
    return out


def _slope_values(c):
    return [2.0 ** (-8.0 * (h + 1) / c["H"]) for h in range(c["H"])]


def _group(d):
    return min(32, d)


def _behind(c):
    """W: keys that lie this far behind a node, or farther, are not seen."""
    return c["window"] or c["C"]


def prepare(case, seed):
    c = case
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = torch.Generator(device=dev).manual_seed(seed)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=dev) * std).to(DT[c["dtype"]])  # noqa: E731
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    B, H, H_kv, d = (c[n] for n in ("B", "H", "H_kv", "d"))
    s = dict(c=c)
    if c["kind"] in ("rope", "rope_train"):
        T = c["T"]
        s.update(q=rnd(B, T, H, d, std=1.5), k=rnd(B, T, H_kv, d))
        if c["kind"] == "rope_train":
            s.update(dq=rnd(B, T, H, d), dk=rnd(B, T, H_kv, d))
        # a packed batch says where each token stands, any other where its sequences begin
        s["positions"], s["start"] = (ints(_positions(c)), None) if c["docs"] else (None, ints(_starts(c)))
        f, s["scale"] = _freq(c)
        s["freq"] = torch.tensor(f, dtype=torch.float64, device=dev)
    else:
        N, C = c["N"], c["C"]
        s.update(q=rnd(B, N, H, d, std=1.5), k=rnd(B, N, H_kv, d), v=rnd(B, N, H_kv, d))
        parents = _parents(c, seed)
        s.update(pos=ints(_starts(c)), parent=ints(parents))
        if c["M"]:
            s["path"] = ints(_paths(parents, c["M"], seed))
        if c["kind"] in ("tree", "accept"):
            s.update(K=rnd(B, C, H_kv, d), V=rnd(B, C, H_kv, d))
        else:  # a cache as the quantization of normal values leaves it: a minimum near -2, a scale near 4 / 15
            q = lambda: torch.randint(0, 256, (B, H_kv, C, d // 2), generator=g, device=dev, dtype=torch.uint8)  # noqa: E731
            s["cache"] = dict(kq=q(), vq=q())
            for n in ("kp", "vp"):
                u = torch.rand(B, H_kv, C, d // _group(d), 2, generator=g, device=dev)
                s["cache"][n] = torch.stack([0.2 + 0.1 * u[..., 0], u[..., 1] - 2.5], -1).bfloat16()
        s["slopes"] = torch.tensor(_slope_values(c), device=dev) if c["slopes"] else None
    if own:
        s.update(_own_plan(c))
    return s


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own_plan(c):
    api = _api()
    if c["kind"] in ("rope", "rope_train"):
        ramp = dict(wavelength=dict(scaling="wavelength", low=1.0, high=4.0), channel=dict(scaling="channel", low=1.0, high=32.0)).get(c["scaling"], {})
        freq = api.rope_frequencies(c["rot"], BASE, factor=c["factor"], original=c["original"], **ramp)
        return dict(p=api.rope_params(c["B"], c["T"], c["H"], c["H_kv"], c["d"], rot=c["rot"], layout=c["layout"], dtype=c["dtype"], scale=_freq(c)[1]), own_freq=freq)
    return dict(p=api.attn_params(c["B"], c["N"], c["H"], c["H_kv"], c["d"], T_k=c["C"], dtype=c["dtype"], window=c["window"], cap=c["cap"]),
                read=api.attn_params(c["B"], c["M"] or 1, c["H"], c["H_kv"], c["d"], T_k=c["C"], dtype=c["dtype"]))


def _run_own(s):
    api, c, p = _api(), s["c"], s["p"]
    if c["kind"] in ("rope", "rope_train"):
        at = dict(positions=s["positions"], start=s["start"])
        q, k = api.lawcat_rope_fwd(p, s["own_freq"], s["q"], s["k"], **at)
        if c["kind"] == "rope":
            return dict(q=q, k=k)
        dq, dk = api.lawcat_rope_bwd(p, s["own_freq"], s["dq"], s["dk"], **at)
        return dict(q=q, k=k, dq=dq, dk=dk)
    parent = None if c["shape"] == "chain" else s["parent"]
    if c["kind"] == "tree":
        return api.lawcat_attn_tree(p, s["q"], s["k"], s["v"], s["K"], s["V"], s["pos"], parent=parent, slopes=s["slopes"])
    if c["kind"] == "accept":
        pos = api.lawcat_cache_accept(p, s["k"], s["v"], s["pos"], s["K"], s["V"], path=s["path"])
        return dict(pos=pos, K=s["K"], V=s["V"])
    x = s["cache"]
    cache = (x["kq"], x["kp"], x["vq"], x["vp"])
    if c["kind"] == "tree_quant":
        return api.lawcat_attn_tree_quant(p, s["q"], s["k"], s["v"], *cache, s["pos"], parent=parent, slopes=s["slopes"])
    pos = api.lawcat_cache_accept_quant(p, s["k"], s["v"], s["pos"], *cache, path=s["path"])
    # (the slots of the longest path, as the values that they stand for)
    return dict(pos=pos, **api.lawcat_cache_dequantize(s["read"], *cache, s["pos"]))


# ------------------------------------------------------------------------------------------------ the plain forms
def _turn(s, x, back):
    """x [B, T, heads, d] turned by its positions' angles (back: the other way)."""
    c = s["c"]
    rot, n = c["rot"], c["rot"] // 2
    at = s["positions"] if s["positions"] is not None else s["start"][:, None] + torch.arange(c["T"], device=x.device)
    angle = at[..., None].double() * s["freq"]                              # (64 bits: 131072 tokens are 20860 turns)
    co, si = (s["scale"] * f(angle).float()[:, :, None] for f in (torch.cos, torch.sin))
    si = -si if back else si
    y = x.float()
    if c["layout"] == "half":
        a, b = y[..., :n], y[..., n:rot]
        turned = torch.cat([a * co - b * si, a * si + b * co], -1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _plain_rope(s):
    out = dict(q=_turn(s, s["q"], False), k=_turn(s, s["k"], False))
    if s["c"]["kind"] == "rope_train":
        out.update(dq=_turn(s, s["dq"], True), dk=_turn(s, s["dk"], True))
    return out


def _plain_paths(s):
    """on [B, N, N]: node j lies on node i's path (itself included); depth [B, N]; there [B, N]."""
    c, parent = s["c"], s["parent"].long()
    N = c["N"]
    i = torch.arange(N, device=parent.device)
    fine = (parent >= -1) & (parent < i)
    step = (parent[..., None] == i).float()
    on = (step + torch.eye(N, device=parent.device)).clamp_max(1)
    for _ in range(max(1, (N - 1).bit_length())):
        on = (on @ on).clamp_max(1)
    on = on > 0
    there = ~(on & ~fine[:, None]).any(-1)
    return on, on.sum(-1) - 1, there


def _plain_quantize(x):
    """[..., d] -> codes [..., d / 2] and (scale, minimum) [..., groups, 2]."""
    d = x.shape[-1]
    g = x.float().reshape(*x.shape[:-1], d // _group(d), _group(d))
    lo, hi = g.amin(-1, keepdim=True).bfloat16().float(), g.amax(-1, keepdim=True)
    sc = ((hi - lo) / 15).bfloat16().float()
    code = torch.where(sc > 0, (g - lo) / torch.where(sc > 0, sc, torch.ones_like(sc)), torch.zeros_like(g)).round().clamp(0, 15)
    code = code.to(torch.uint8).reshape(*x.shape[:-1], d // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), torch.cat([sc, lo], -1).bfloat16()


def _plain_dequantize(q, p):
    n = q.shape[-1] * 2
    code = torch.stack([q & 15, q >> 4], -1).reshape(*q.shape[:-1], n // _group(n), _group(n)).float()
    return (code * p[..., :1].float() + p[..., 1:].float()).reshape(*q.shape[:-1], n)


def _plain_tree(s):
    c = s["c"]
    B, N, C, H, H_kv, d = (c[n] for n in ("B", "N", "C", "H", "H_kv", "d"))
    G, W = H // H_kv, _behind(c)
    on, depth, there = _plain_paths(s)
    pos = s["pos"].long()
    slot = torch.arange(C, device=pos.device)[None]
    back = (pos[:, None] - 1 - slot) % C + 1                                 # how far in front of `pos` the slot's token stands
    far = torch.cat([back[:, None] + depth[..., None], (depth[..., None] - depth[:, None]).abs()], -1)   # [B, N, C + N]
    see = torch.cat([(back <= pos[:, None])[:, None].expand(B, N, C), on], -1) & (far < W) & there[..., None]
    if c["kind"] == "tree":
        K, V = (s[n].float().permute(0, 2, 1, 3) for n in ("K", "V"))       # [B, H_kv, C, d]
        k, v = s["k"].float(), s["v"].float()
    else:
        x = s["cache"]
        K, V = _plain_dequantize(x["kq"], x["kp"]), _plain_dequantize(x["vq"], x["vp"])
        k, v = (_plain_dequantize(*_plain_quantize(s[n])) for n in ("k", "v"))
    # (nodes that are not there may hold anything)
    k, v = (torch.where(there[..., None, None], y, torch.zeros_like(y)).permute(0, 2, 1, 3) for y in (k, v))
    q = s["q"].float().reshape(B, N, H_kv, G, d).permute(0, 2, 3, 1, 4).reshape(B, H_kv, G * N, d)
    w = torch.cat([q @ K.transpose(-1, -2), q @ k.transpose(-1, -2)], -1).mul_(d ** -0.5).reshape(B, H_kv, G, N, C + N)
    if c["cap"]:
        w = w.div_(c["cap"]).tanh_().mul_(c["cap"])
    if s["slopes"] is not None:
        w = w - s["slopes"].reshape(1, H_kv, G, 1, 1) * far[:, None, None]
    w = w.masked_fill_(~see[:, None, None], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)).exp_()
    l = w.sum(-1, keepdim=True)
    w = w.div_(torch.where(l > 0, l, torch.ones_like(l))).reshape(B, H_kv, G * N, C + N)
    o = w[..., :C] @ V + w[..., C:] @ v
    return o.reshape(B, H_kv, G, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, H, d).to(s["q"].dtype)


def _plain_accept(s):
    c = s["c"]
    B, M, C = c["B"], c["M"], c["C"]
    path, pos = s["path"].long(), s["pos"].long()
    taken = (path >= 0).cumprod(-1).bool()                                   # up to the first negative entry
    b = torch.arange(B, device=pos.device)[:, None]
    t = torch.arange(M, device=pos.device)
    at = (pos[:, None] + t) % C
    rows = [s[n][b, path.clamp_min(0)] for n in ("k", "v")]                  # [B, M, H_kv, d]
    out = dict(pos=(pos + taken.sum(-1)).to(torch.int32))
    if c["kind"] == "accept":
        for n, x in zip(("K", "V"), rows):
            s[n][b, at] = torch.where(taken[..., None, None], x, s[n][b, at])
            out[n] = s[n]
        return out
    x = s["cache"]
    for n, q, p, y in (("k", "kq", "kp", rows[0]), ("v", "vq", "vp", rows[1])):
        codes, sc = _plain_quantize(y)
        x[q][b, :, at] = torch.where(taken[..., None, None], codes, x[q][b, :, at])
        x[p][b, :, at] = torch.where(taken[..., None, None, None], sc, x[p][b, :, at])
        out[n] = _plain_dequantize(x[q][b, :, at], x[p][b, :, at]).to(s[n].dtype)
    return out


def run(state):
    if own:
        return _run_own(state)
    kind = state["c"]["kind"]
    return _plain_rope(state) if kind.startswith("rope") else _plain_tree(state) if kind.startswith("tree") else _plain_accept(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] in ("rope", "rope_train"):
        n = c["B"] * c["T"] * (c["H"] + c["H_kv"])
        passes = 2 if c["kind"] == "rope_train" else 1
        return dict(bytes=passes * (2 * n * c["d"] * es + 4 * (c["T"] if c["docs"] else c["B"])), flops=passes * 3 * n * c["rot"])
    quant = c["d"] // 2 + 4 * c["d"] // _group(c["d"])                       # bytes of a row in 4 bits
    if c["kind"] in ("accept", "accept_quant"):
        rows = 2 * sum(max(1, c["M"] // 2) for b in range(c["B"])) * c["H_kv"]   # (about half of the entries are a path's)
        if c["kind"] == "accept":
            return dict(bytes=2 * rows * c["d"] * es, flops=rows * c["d"])
        back = 2 * c["B"] * c["M"] * c["H_kv"] * (quant + c["d"] * es)           # the slots read back
        return dict(bytes=rows * (c["d"] * es + quant) + back, flops=8 * rows * c["d"])
    seen = [min(p, c["C"], _behind(c) - 1) for p in _starts(c)]
    rows = sum(seen) * c["H_kv"]
    own_rows = c["B"] * c["N"] * c["d"] * es * (2 * c["H"] + 2 * c["H_kv"])
    pairs = (sum(seen) + c["B"] * min(4, c["N"])) * c["N"] * c["H"]          # (a node sees a few nodes of its path)
    return dict(bytes=2 * rows * (quant if c["kind"] == "tree_quant" else c["d"] * es) + own_rows, flops=4 * c["d"] * pairs)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_turn(c, x, way):
    """One pair as a complex number times m e^(i n f)."""
    f, m = _freq(c)
    n = torch.tensor(_positions(c), dtype=torch.float64, device=x.device)
    z = torch.polar(torch.full((), m, dtype=torch.float64, device=x.device), way * n[..., None] * torch.tensor(f, dtype=torch.float64, device=x.device))[:, :, None]
    y = x.double().clone()
    rot = c["rot"]
    even, odd = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    w = torch.complex(y[..., even], y[..., odd]) * z
    y[..., even], y[..., odd] = w.real, w.imag
    return y


def _exact_held(x):
    """What a 4-bit cache holds of the row values x [..., d], as the definition has it, in 64 bits."""
    d = x.shape[-1]
    y = x.double().reshape(*x.shape[:-1], -1, _group(d))
    lo = y.min(-1, keepdim=True).values.to(torch.bfloat16).double()
    sc = ((y.max(-1, keepdim=True).values - lo) / 15).to(torch.bfloat16).double()
    n = torch.nan_to_num((y - lo) / sc, nan=0.0).round().clamp(0, 15)
    return (lo + n * sc).reshape(x.shape)


def _exact_rows(cache, q, p, b, slots):
    """Values [H_kv, n, d] of a 4-bit cache's slots."""
    byte, pr = cache[q][b][:, slots].to(torch.int64), cache[p][b][:, slots].double()
    d = 2 * byte.shape[-1]
    code = torch.zeros(*byte.shape[:-1], d, dtype=torch.float64, device=byte.device)
    code[..., 0::2], code[..., 1::2] = (byte % 16).double(), (byte // 16).double()
    scale, low = pr.repeat_interleave(_group(d), -2).unbind(-1)
    return low + code * scale


def exact(case, seed):
    global own
    c, was = case, own
    own = False
    s = prepare(case, seed)
    own = was
    if c["kind"] in ("rope", "rope_train"):
        out = dict(q=_exact_turn(c, s["q"], 1), k=_exact_turn(c, s["k"], 1))
        if c["kind"] == "rope_train":
            out.update(dq=_exact_turn(c, s["dq"], -1), dk=_exact_turn(c, s["dk"], -1))
        return out
    B, N, C, H, H_kv, d = (c[n] for n in ("B", "N", "C", "H", "H_kv", "d"))
    dev, W = s["k"].device, _behind(c)
    parents, starts = s["parent"].tolist(), _starts(c)
    if c["kind"] in ("accept", "accept_quant"):
        out = dict(pos=None)
        if c["kind"] == "accept":
            for n in ("K", "V"):
                out[n] = s[n].double()
                for b, path in enumerate(s["path"].tolist()):
                    for t in range(len(path)):
                        if min(path[:t + 1]) >= 0:
                            out[n][b, (starts[b] + t) % C] = s[n.lower()][b, path[t]].double()
            return out
        for n, q, p in (("k", "kq", "kp"), ("v", "vq", "vp")):
            out[n] = torch.zeros(B, c["M"], H_kv, d, dtype=torch.float64, device=dev)
            for b, path in enumerate(s["path"].tolist()):
                slots = [(starts[b] + t) % C for t in range(c["M"])]
                out[n][b] = _exact_rows(s["cache"], q, p, b, slots).transpose(0, 1)
                for t, node in enumerate(path):
                    if node < 0:
                        break
                    out[n][b, t] = _exact_held(s[n][b, node])
        return out
    o = torch.zeros(B, N, H, d, dtype=torch.float64, device=dev)
    slopes = _slope_values(c) if c["slopes"] else [0.0] * H
    slopes = torch.tensor(slopes).double().to(dev)
    for b, pos in enumerate(starts):
        paths = []
        for i, p in enumerate(parents[b]):
            paths.append(paths[p] + [i] if 0 <= p < i and paths[p] else [i] if p == -1 else [])
        first = max(0, pos - min(C, W - 1))
        cached = torch.arange(first, pos, device=dev)
        if c["kind"] == "tree_quant":
            K, V = (_exact_rows(s["cache"], q, p, b, cached % C) for q, p in (("kq", "kp"), ("vq", "vp")))
            k, v = (_exact_held(s[n][b]).transpose(0, 1) for n in ("k", "v"))
        else:
            K, V = (s[n][b, cached % C].double().transpose(0, 1) for n in ("K", "V"))
            k, v = (s[n][b].double().transpose(0, 1) for n in ("k", "v"))
        k, v = torch.cat([K, k], 1), torch.cat([V, v], 1)                    # [H_kv, cached + N, d]
        at = torch.full((N, len(cached) + N), math.inf, dtype=torch.float64, device=dev)   # distances; infinite where not seen
        for i, path in enumerate(paths):
            if not path:
                continue
            here = pos + len(path) - 1
            at[i, :len(cached)] = (here - cached).double()
            for e, j in enumerate(path):
                at[i, len(cached) + j] = float(len(path) - 1 - e)
        at[at >= W] = math.inf
        rows = [i for i, path in enumerate(paths) if path]
        for h in range(H):
            g = h * H_kv // H
            x = s["q"][b, rows, h].double() @ k[g].T / math.sqrt(d)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            dist = at[rows]
            x = torch.where(torch.isinf(dist), -math.inf, x - slopes[h] * torch.nan_to_num(dist, posinf=0.0))
            y = torch.softmax(x, -1)
            o[b, rows, h] = y @ torch.where((y.sum(0) > 0)[:, None], v[g], 0.0)
    return o
