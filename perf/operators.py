"""Softmax attention beside the linearized layer, as cases that can be timed and compared.

Softmax attention is what the layer is distilled from (the teacher of the layer-wise stage) and what a hybrid model keeps
in some of its layers (the sliding-window rows of the ablation). Its operators: the forward over prompts, pieces of prompts
and packed documents; its gradient; one decode step over a cache of keys and values in the storage type; the same over a
cache held in 4 bits, and the writing and reading back of such a cache.

The scores are s = scale q.k, then (where asked) cap tanh(s / cap), then (where asked) a bias of -slope |i - j|. A query at
position i sees the keys of its own document with j <= i (and, under a window w, i - j < w), and the document's prefix.

A cache in 4 bits holds, for every group of 32 channels of a token's key or value row (16 at width 16), a scale and a
minimum in bf16 and one code of 4 bits per channel: value = minimum + code scale, scale = bf16((max - min) / 15),
code = round-half-even((x - minimum) / scale) in 0 ... 15.

Sizes are those of the benchmark configurations and tests: 32 query / 8 key-value heads of width 64 or 128, 4 heads of 64
in fp32, prompts of up to 8192 tokens, training sequences of 1162 ... 1300 and 8 x 1024 tokens, 64 sequences decoded at once.
A case is a dict of plain values; `kind` is fwd | train | decode | decode_quant | quantize.
"""
import math

import torch


own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SMALL = dict(H=32, H_kv=8, d=64)    # the 1B shape
LARGE = dict(H=32, H_kv=8, d=128)   # the 7B shape


def _api():
    from paper_2509_18467_b200 import api
    return api


def _attn(name, kind, dtype, B, T, T_k=0, docs="", causal=1, window=0, cap=0.0, slopes=False, prefix=False, **heads):
    c = dict(kind=kind, dtype=dtype, B=B, T=T, T_k=T_k or T, docs=docs, causal=causal, window=window, cap=cap, slopes=slopes,
             prefix=prefix, **heads)
    return dict(name=name, **c) if name else c


def _dec(name, kind, B, C, last, window=0, cap=0.0, slopes=False, dtype="bf16", **heads):
    c = dict(kind=kind, dtype=dtype, B=B, C=C, last=last, window=window, cap=cap, slopes=slopes, **heads)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # the teacher's outputs for a batch of distillation sequences; a prefix model with distance biases
        _attn("teacher-prefix", "fwd", "bf16", 8, 1024, slopes=True, prefix=True, **SMALL),
        # the teacher's outputs for a whole long prompt, the largest product here
        _attn("teacher-prompt", "fwd", "bf16", 1, 8192, **LARGE),
        # a turn of a conversation: few queries behind a long past, scores capped
        _attn("teacher-turn", "fwd", "bf16", 1, 77, T_k=8192, cap=30.0, **LARGE),
        # the small exact configuration, forward and gradients in fp32
        _attn("train-fp32", "train", "f32", 1, 512, H=4, H_kv=4, d=64),
        # the four training lengths as documents of one packed sequence, scores capped
        _attn("train-packed", "train", "bf16", 1, 4856, docs="1162,1171,1223,1300", cap=30.0, **LARGE),
        # fine-tuning of a hybrid's sliding-window layer (window 64) on the distillation batch
        _attn("train-window", "train", "bf16", 8, 1024, window=64, **SMALL),
        # one sequence being generated by a sliding-window layer: a ring of 64 slots, all launches and latency
        _dec("decode-one", "decode", 1, 64, 1223, window=64, **SMALL),
        # one token for each of a serving batch of 64 sequences of different lengths
        _dec("decode-batch", "decode", 64, 8192, 8190, **LARGE),
        # one sequence over a long past held in 4 bits
        _dec("quant-one", "decode_quant", 1, 32768, 32700, slopes=True, **LARGE),
        # a serving batch over pasts held in 4 bits
        _dec("quant-batch", "decode_quant", 64, 16384, 16383, **LARGE),
        # a prompt's keys and values go into the 4-bit cache, and come back for the next piece of the prompt
        dict(name="cache-prompt", kind="quantize", dtype="bf16", B=1, T=8192, C=8192, at=0, H_kv=8, d=128),
        # the tokens of a turn, appended for four sequences in a ring that wraps
        dict(name="cache-turn", kind="quantize", dtype="bf16", B=4, T=77, C=1300, at=1290, H_kv=8, d=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "train", "train", "decode", "decode_quant", "quantize"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"]) if kind in ("fwd", "train", "decode") else "bf16"
    d = rng.choice([64, 128])
    H_kv = rng.choice([1, 2, 4, 8])
    H = H_kv * rng.choice([1, 2, 4, 8][:3 if H_kv == 8 else 4])
    heads = dict(H=H, H_kv=H_kv, d=d)
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    slopes = rng.random() < 0.3
    if kind == "quantize":
        C = _log(rng, 64, 8192)
        return dict(kind=kind, dtype=dtype, B=rng.randint(1, 8), T=_log(rng, 1, C), C=C, at=rng.randint(0, C), H_kv=H_kv, d=d)
    if kind in ("decode", "decode_quant"):
        B = _log(rng, 1, 64)
        C = _log(rng, 64, 8192)
        window = rng.choice([0, 0, _log(rng, 1, C)])
        return _dec("", kind, B, C, _log(rng, 1, 2 * C), window=window, cap=cap, slopes=slopes, dtype=dtype, **heads)
    T = _log(rng, 1, 5000 if kind == "fwd" else 4000)
    if dtype == "f32":
        T = min(T, 1500)
    B = rng.randint(1, max(1, min(8, 4000 // T)))
    form = rng.choice(["causal", "full", "window", "docs", "prefix", "past"])
    if form == "docs":
        n = rng.randint(2, 9)
        cuts = sorted(rng.randint(0, T) for _ in range(n - 1))
        docs = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [T]))
        return _attn("", kind, dtype, 1, T, docs=docs, cap=cap, slopes=slopes, **heads)
    if form == "past":
        return _attn("", kind, dtype, B, max(1, T // 8), T_k=T, cap=cap, slopes=slopes, **heads)
    return _attn("", kind, dtype, B, T, causal=int(form != "full"), window=_log(rng, 1, T) if form == "window" else 0, cap=cap,
                 slopes=slopes, prefix=form == "prefix", **heads)


# ------------------------------------------------------------------------------------------------ what a case's names stand for
def _lens(c):
    return [int(x) for x in c["docs"].split(",")] if c["docs"] else [c["T_k"]] * c["B"]


def _prefixes(c):
    """Host list: the prefix of each sequence (ragged, from nothing to two thirds of it)."""
    n = _lens(c)
    return [(2 * x * ((5 * i + 3) % 8)) // 21 for i, x in enumerate(n)] if c["prefix"] else None


def _intervals(c):
    """Host list over sequences: (length, prefix) of each; with documents the sequences are packed."""
    return list(zip(_lens(c), _prefixes(c) or [0] * len(_lens(c))))


def _positions(c):
    """Host list: the position of the new token of each decoded sequence: ragged, from `last` down to a half of it."""
    return [max(0, c["last"] - (c["last"] // 2) * ((7 * b) % 16) // 15) for b in range(c["B"])]


def _seen(c, pos):
    return min(pos + 1, c["C"], c["window"] or c["C"])


def _slope_values(c):
    return [2.0 ** (-8.0 * (h + 1) / c["H"]) for h in range(c["H"])]


def _group(d):
    return min(32, d)


def prepare(case, seed):
    c = case
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = torch.Generator(device=dev).manual_seed(seed)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=dev) * std).to(DT[c["dtype"]])  # noqa: E731
    s = dict(c=c)
    if c["kind"] in ("fwd", "train"):
        B, T, T_k, H, H_kv, d = (c[n] for n in ("B", "T", "T_k", "H", "H_kv", "d"))
        s.update(q=rnd(B, T, H, d, std=1.5), k=rnd(B, T_k, H_kv, d), v=rnd(B, T_k, H_kv, d))
        if c["kind"] == "train":
            s["dO"] = rnd(B, T, H, d)
        s["cu"] = [sum(_lens(c)[:i]) for i in range(len(_lens(c)) + 1)] if c["docs"] else None
        s["prefix"] = _prefixes(c)
        # (the same on the device, for the plain form's masks)
        s["doc"] = torch.repeat_interleave(torch.arange(len(_lens(c))), torch.tensor(_lens(c))).to(dev) if c["docs"] else None
        s["prefix_dev"] = torch.tensor(s["prefix"], device=dev) if s["prefix"] else None
    elif c["kind"] == "quantize":
        B, T, H_kv, d = (c[n] for n in ("B", "T", "H_kv", "d"))
        # keys have channels that stand out, as behind a projection; values do not
        s.update(k=(rnd(B, T, H_kv, d) * (1 + 4 * (torch.arange(d, device=dev) % 17 == 3))).to(DT[c["dtype"]]), v=rnd(B, T, H_kv, d))
        s["pos"] = torch.tensor([c["at"] + 3 * b for b in range(B)], dtype=torch.int32, device=dev)
        s["cache"] = _empty_cache(B, c["C"], H_kv, d, dev)
    else:
        B, C, H, H_kv, d = (c[n] for n in ("B", "C", "H", "H_kv", "d"))
        s.update(q=rnd(B, H, d, std=1.5), k=rnd(B, H_kv, d), v=rnd(B, H_kv, d))
        s["pos"] = torch.tensor(_positions(c), dtype=torch.int32, device=dev)
        if c["kind"] == "decode":
            s.update(K=rnd(B, C, H_kv, d), V=rnd(B, C, H_kv, d))
        else:  # a cache as the quantization of normal values leaves it: a minimum near -2, a scale near 4 / 15
            ng = d // _group(d)
            cache = _empty_cache(B, C, H_kv, d, dev)
            for n in ("kq", "vq"):
                cache[n].copy_(torch.randint(0, 256, cache[n].shape, generator=g, device=dev, dtype=torch.uint8))
            for n in ("kp", "vp"):
                cache[n][..., 0] = 0.2 + 0.1 * torch.rand(B, H_kv, C, ng, generator=g, device=dev)
                cache[n][..., 1] = -2.5 + torch.rand(B, H_kv, C, ng, generator=g, device=dev)
            s["cache"] = cache
    s["slopes"] = torch.tensor(_slope_values(c), device=dev) if c.get("slopes") else None
    if own:
        s["p"] = _own_params(c)
    return s


def _empty_cache(B, C, H_kv, d, dev):
    """Codes of two channels per byte (the even one low) and (scale, minimum) per group, a head's tokens side by side."""
    q = lambda: torch.zeros(B, H_kv, C, d // 2, dtype=torch.uint8, device=dev)  # noqa: E731
    p = lambda: torch.zeros(B, H_kv, C, d // _group(d), 2, dtype=torch.bfloat16, device=dev)  # noqa: E731
    return dict(kq=q(), kp=p(), vq=q(), vp=p())


# ------------------------------------------------------------------------------------------------ the framework's calls
def _own_params(c):
    api = _api()
    if c["kind"] in ("fwd", "train"):
        return api.attn_params(c["B"], c["T"], c["H"], c["H_kv"], c["d"], T_k=c["T_k"], dtype=c["dtype"], causal=c["causal"],
                               window=c["window"], cap=c["cap"])
    if c["kind"] == "quantize":
        return api.attn_params(c["B"], c["T"], c["H_kv"], c["H_kv"], c["d"], T_k=c["C"], dtype=c["dtype"])
    return api.attn_params(c["B"], 1, c["H"], c["H_kv"], c["d"], T_k=c["C"], dtype=c["dtype"], window=c["window"], cap=c["cap"])


def _run_own(s):
    api, c, p = _api(), s["c"], s["p"]
    if c["kind"] in ("fwd", "train"):
        more = dict(slopes=s["slopes"], cu_seqlens=s["cu"], prefix=s["prefix"])
        r = api.lawcat_attn_fwd(p, s["q"], s["k"], s["v"], **more)
        if c["kind"] == "train":
            r.update(api.lawcat_attn_bwd(p, s["q"], s["k"], s["v"], r["o"], r["lse"], s["dO"], **more))
        return r
    if c["kind"] == "quantize":
        x = s["cache"]
        api.lawcat_cache_quantize(p, s["k"], s["v"], s["pos"], x["kq"], x["kp"], x["vq"], x["vp"])
        return api.lawcat_cache_dequantize(p, x["kq"], x["kp"], x["vq"], x["vp"], s["pos"])
    if c["kind"] == "decode":
        o = api.lawcat_attn_decode(p, s["q"], s["k"], s["v"], s["K"], s["V"], s["pos"], slopes=s["slopes"])
        return dict(o=o, K=s["K"], V=s["V"])
    x = s["cache"]
    o = api.lawcat_attn_decode_quant(p, s["q"], s["k"], s["v"], x["kq"], x["kp"], x["vq"], x["vp"], s["pos"], slopes=s["slopes"])
    # (the state's one new row, as the values that it stands for)
    return dict(o=o, **api.lawcat_cache_dequantize(p, x["kq"], x["kp"], x["vq"], x["vp"], s["pos"]))


# ------------------------------------------------------------------------------------------------ the plain forms
def _plain_mask(s):
    """[B or 1, T, T_k] truth values: key j is seen by query i; and the distances |i - j| [T, T_k]."""
    c, dev = s["c"], s["q"].device
    i = torch.arange(c["T"], device=dev)[:, None] + (c["T_k"] - c["T"])
    j = torch.arange(c["T_k"], device=dev)[None, :]
    see = (j <= i) if c["causal"] else torch.ones_like(j <= i)
    if c["window"]:
        see = see & (i - j < c["window"]) & (j - i < c["window"])
    see = see[None]
    if s["prefix_dev"] is not None:
        see = see | (j < s["prefix_dev"][:, None, None])
    if s["doc"] is not None:
        see = see & (s["doc"][None, :, None] == s["doc"][None, None, :])
    return see, (i - j).abs()


def _plain_attention(s):
    c = s["c"]
    B, T, T_k, H, H_kv, d = (c[n] for n in ("B", "T", "T_k", "H", "H_kv", "d"))
    G = H // H_kv
    q = s["q"].float().reshape(B, T, H_kv, G, d).permute(0, 2, 3, 1, 4)  # [B, H_kv, G, T, d]
    k = s["k"].float().permute(0, 2, 1, 3)[:, :, None]                   # [B, H_kv, 1, T_k, d]
    v = s["v"].float().permute(0, 2, 1, 3)[:, :, None]
    see, far = _plain_mask(s)
    x = q @ k.transpose(-1, -2)
    x.mul_(d ** -0.5)
    th = None
    if c["cap"]:
        th = x.div_(c["cap"]).tanh_()
        x = th * c["cap"]
    if s["slopes"] is not None:
        x.sub_(s["slopes"].reshape(1, H_kv, G, 1, 1) * far)
    x.masked_fill_(~see[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(m.clamp_min(torch.finfo(torch.float32).min)).exp_()
    l = x.sum(-1, keepdim=True)
    lse = (m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(B, T, H)
    x.div_(torch.where(l > 0, l, torch.ones_like(l)))
    rows = lambda y: y.permute(0, 3, 1, 2, 4).reshape(B, T, H, d)  # noqa: E731
    out = dict(o=rows(x @ v).to(s["q"].dtype), lse=lse)
    if c["kind"] == "fwd":
        return out
    del see, far
    dO = s["dO"].float().reshape(B, T, H_kv, G, d).permute(0, 2, 3, 1, 4)
    keys = lambda y: y.permute(0, 2, 1, 3).to(s["q"].dtype)  # noqa: E731
    out["dv"] = keys((x.transpose(-1, -2) @ dO).sum(2))
    dx = dO @ v.transpose(-1, -2)
    dx.sub_((dx * x).sum(-1, keepdim=True)).mul_(x)
    if th is not None:
        dx.mul_(th.square_().neg_().add_(1))
    dx.mul_(d ** -0.5)
    out["dq"] = rows(dx @ k).to(s["q"].dtype)
    out["dk"] = keys((dx.transpose(-1, -2) @ q).sum(2))
    return out


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


def _plain_decode(s):
    c = s["c"]
    B, C, H, H_kv, d = (c[n] for n in ("B", "C", "H", "H_kv", "d"))
    G = H // H_kv
    pos = s["pos"].long()
    at, b = pos % C, torch.arange(B, device=pos.device)
    if c["kind"] == "decode":
        s["K"][b, at], s["V"][b, at] = s["k"], s["v"]
        K, V = s["K"].float().permute(0, 2, 1, 3), s["V"].float().permute(0, 2, 1, 3)  # [B, H_kv, C, d]
    else:
        x = s["cache"]
        for t, q, p in (("k", "kq", "kp"), ("v", "vq", "vp")):
            x[q][b, :, at], x[p][b, :, at] = _plain_quantize(s[t])
        K, V = _plain_dequantize(x["kq"], x["kp"]), _plain_dequantize(x["vq"], x["vp"])
    slot = torch.arange(C, device=pos.device)[None]
    back = (pos[:, None] - slot) % C                     # how far behind the new token the slot's token is
    see = (back <= pos[:, None]) & (back < (c["window"] or C))
    w = (s["q"].float().reshape(B, H_kv, G, d) @ K.transpose(-1, -2)) * d ** -0.5
    if c["cap"]:
        w = c["cap"] * torch.tanh(w / c["cap"])
    if s["slopes"] is not None:
        w = w - s["slopes"].reshape(1, H_kv, G, 1) * back[:, None, None]
    w = torch.where(see[:, None, None], w, -math.inf)
    w = torch.exp(w - w.amax(-1, keepdim=True))
    o = ((w @ V) / w.sum(-1, keepdim=True)).reshape(B, H, d).to(s["q"].dtype)
    if c["kind"] == "decode":
        return dict(o=o, K=s["K"], V=s["V"])
    row = lambda q, p: _plain_dequantize(x[q][b, :, at], x[p][b, :, at])[:, None].to(s["q"].dtype)  # noqa: E731
    return dict(o=o, k=row("kq", "kp"), v=row("vq", "vp"))


def _plain_cache(s):
    c, x = s["c"], s["cache"]
    T, C = c["T"], c["C"]
    at = (s["pos"].long()[:, None] + torch.arange(T, device=s["pos"].device)) % C   # [B, T]
    b = torch.arange(c["B"], device=at.device)[:, None]
    out = {}
    for t, q, p in (("k", "kq", "kp"), ("v", "vq", "vp")):
        codes, sc = _plain_quantize(s[t])
        x[q][b, :, at], x[p][b, :, at] = codes, sc
        out[t] = _plain_dequantize(x[q][b, :, at], x[p][b, :, at]).to(s[t].dtype)
    return out


def run(state):
    if own:
        return _run_own(state)
    kind = state["c"]["kind"]
    return _plain_attention(state) if kind in ("fwd", "train") else _plain_cache(state) if kind == "quantize" else _plain_decode(state)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _pairs(c):
    """(query, key) pairs that are seen, per head."""
    n = 0
    for length, pre in _intervals(c):
        T = length if c["docs"] else c["T"]
        for t in range(T):
            i = t + length - T
            lo = max(0, i - c["window"] + 1) if c["window"] else 0
            hi = max(i + 1, pre) if c["causal"] else min(length, i + c["window"]) if c["window"] else length
            n += max(0, hi - lo)
    return n


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] in ("fwd", "train"):
        nq, nk = c["B"] * c["T"] * c["H"] * c["d"], c["B"] * c["T_k"] * c["H_kv"] * c["d"]
        pairs = _pairs(c) * c["H"]
        if c["kind"] == "fwd":
            return dict(bytes=es * (2 * nq + 2 * nk) + 4 * c["B"] * c["T"] * c["H"], flops=4 * c["d"] * pairs)
        return dict(bytes=es * (4 * nq + 4 * nk) + 4 * c["B"] * c["T"] * c["H"], flops=14 * c["d"] * pairs)
    rows = {"quantize": lambda: 0}.get(c["kind"], lambda: sum(_seen(c, x) for x in _positions(c)))() * c["H_kv"]
    quant = c["d"] // 2 + 4 * c["d"] // _group(c["d"])                  # bytes of a row in 4 bits
    if c["kind"] == "quantize":
        n = c["B"] * min(c["T"], c["C"]) * c["H_kv"]
        return dict(bytes=2 * n * (2 * es * c["d"] + 2 * quant), flops=2 * n * 6 * c["d"])
    new = c["B"] * (2 * c["H"] + 4 * c["H_kv"]) * c["d"] * es
    if c["kind"] == "decode":
        return dict(bytes=2 * rows * c["d"] * es + new, flops=4 * c["d"] * rows * c["H"] // c["H_kv"])
    return dict(bytes=2 * rows * quant + new, flops=(4 * c["H"] // c["H_kv"] + 4) * c["d"] * rows)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_row_block(c, q, k, v, i, slope, pre):
    """One head of one sequence: q [n, d], k, v [m, d] in 64 bits, positions i [n]; returns what the definition gives."""
    j = torch.arange(k.shape[0], device=k.device, dtype=torch.float64)
    raw = torch.einsum("nd,md->nm", q, k) / math.sqrt(c["d"])
    x = raw
    if c["cap"]:
        x = c["cap"] * torch.tanh(raw / c["cap"])
    dist = torch.abs(i[:, None] - j[None, :])
    x = x - slope * dist
    hidden = torch.zeros_like(dist, dtype=torch.bool)
    if c["causal"]:
        hidden |= (j[None, :] > i[:, None]) & (j[None, :] >= pre)
    if c["window"]:
        hidden |= dist >= c["window"]
    x[hidden] = -math.inf
    return raw, x


def _exact_attention(c, s):
    B, T, T_k, H, H_kv, d = (c[n] for n in ("B", "T", "T_k", "H", "H_kv", "d"))
    dev = s["q"].device
    o = torch.zeros(B, T, H, d, dtype=torch.float64, device=dev)
    lse = torch.zeros(B, T, H, dtype=torch.float64, device=dev)
    train = c["kind"] == "train"
    if train:
        dq = torch.zeros_like(o)
        dk, dv = (torch.zeros(B, T_k, H_kv, d, dtype=torch.float64, device=dev) for _ in range(2))
    slopes = _slope_values(c) if c["slopes"] else [0.0] * H
    start = 0
    for n, (length, pre) in enumerate(_intervals(c)):
        b, k0, nq = (0, start, length) if c["docs"] else (n, 0, T)
        start += length
        if not length:
            continue
        i = torch.arange(nq, device=dev, dtype=torch.float64) + (length - nq)
        for h in range(H):
            g = h * H_kv // H
            q = s["q"][b, k0:k0 + nq, h].double()
            k, v = s["k"][b, k0:k0 + length, g].double(), s["v"][b, k0:k0 + length, g].double()
            raw, x = _exact_row_block(c, q, k, v, i, float(torch.tensor(slopes[h])), pre)
            z = torch.logsumexp(x, -1)
            w = torch.where(torch.isinf(z)[:, None], torch.zeros_like(x), torch.exp(x - z[:, None]))
            y = w @ v
            o[b, k0:k0 + nq, h], lse[b, k0:k0 + nq, h] = y, z
            if train:
                dy = s["dO"][b, k0:k0 + nq, h].double()
                dv[b, k0:k0 + length, g] += w.T @ dy
                dx = w * (dy @ v.T - (dy * y).sum(-1, keepdim=True))
                if c["cap"]:
                    dx = dx / torch.cosh(raw / c["cap"]) ** 2
                dq[b, k0:k0 + nq, h] = dx @ k / math.sqrt(d)
                dk[b, k0:k0 + length, g] += dx.T @ q / math.sqrt(d)
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv) if train else dict(o=o, lse=lse)


def _exact_held(x):
    """What a 4-bit cache holds of the row values x [..., d], as the definition has it, in 64 bits."""
    d = x.shape[-1]
    y = x.double().reshape(*x.shape[:-1], -1, _group(d))
    lo = y.min(-1, keepdim=True).values.to(torch.bfloat16).double()
    sc = ((y.max(-1, keepdim=True).values - lo) / 15).to(torch.bfloat16).double()
    n = torch.nan_to_num((y - lo) / sc, nan=0.0).round().clamp(0, 15)
    return (lo + n * sc).reshape(x.shape)


def exact(case, seed):
    global own
    c, was = case, own
    own = False
    s = prepare(case, seed)
    own = was
    if c["kind"] in ("fwd", "train"):
        return _exact_attention(c, s)
    if c["kind"] == "quantize":
        return dict(k=_exact_held(s["k"]), v=_exact_held(s["v"]))
    B, C, H, H_kv, d = (c[n] for n in ("B", "C", "H", "H_kv", "d"))
    o = torch.zeros(B, H, d, dtype=torch.float64, device=s["q"].device)
    slopes = _slope_values(c) if c["slopes"] else [0.0] * H
    quant = c["kind"] == "decode_quant"
    new_k, new_v = (_exact_held(s[n]) if quant else s[n].double() for n in ("k", "v"))
    for b, pos in enumerate(_positions(c)):
        first = pos + 1 - _seen(c, pos)
        slots = torch.arange(first, pos, device=o.device) % C     # the past's slots, oldest first
        for g in range(H_kv):
            if quant:
                past = []
                for q, p in (("kq", "kp"), ("vq", "vp")):
                    byte = s["cache"][q][b, g, slots].to(torch.int64)
                    scale, low = s["cache"][p][b, g, slots].double().repeat_interleave(_group(d), 1).unbind(-1)
                    code = torch.zeros(len(slots), d, dtype=torch.float64, device=o.device)
                    code[:, 0::2], code[:, 1::2] = (byte % 16).double(), (byte // 16).double()
                    past.append(low + code * scale)
            else:
                past = [s[n][b, slots, g].double() for n in ("K", "V")]
            k, v = torch.cat([past[0], new_k[b, g][None]]), torch.cat([past[1], new_v[b, g][None]])
            back = torch.arange(len(k) - 1, -1, -1, device=o.device, dtype=torch.float64)
            for h in range(g * H // H_kv, (g + 1) * H // H_kv):
                x = k @ s["q"][b, h].double() / math.sqrt(d)
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                o[b, h] = torch.softmax(x - float(torch.tensor(slopes[h])) * back, 0) @ v
    if quant:
        return dict(o=o, k=new_k[:, None], v=new_v[:, None])
    at = torch.tensor(_positions(c), device=o.device) % C
    rows = torch.arange(B, device=o.device)
    K, V = s["K"].double(), s["V"].double()
    K[rows, at], V[rows, at] = new_k, new_v
    return dict(o=o, K=K, V=V)
