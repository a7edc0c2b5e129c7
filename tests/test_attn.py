"""Softmax attention forward and backward through the C ABI against 64 bits (attn_reference.py, which derives the tolerances):
masks that cut tiles, leave rows empty or cover several documents, one token to several tiles, shared heads, both storage types
and both sets of kernels; and the calls that are refused."""
import ctypes
import math

import pytest
import torch

from attn_reference import U16, U32, attention, check, visible
from paper_2509_18467_b200 import api, build

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(shape, seed, dtype, std=1.0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(DT[dtype]).to(device)


def case(B=1, T=64, T_k=None, H=4, H_kv=2, d=64, dtype="bf16", causal=1, window=0, cap=0.0, slopes=False, cu=None, prefix=None,
         exact=0, grad=True, seed=0, ref_cap=None):
    T_k = T if T_k is None else T_k
    q, k, v = draw((B, T, H, d), seed, dtype, 1.5), draw((B, T_k, H_kv, d), seed + 1, dtype), draw((B, T_k, H_kv, d), seed + 2, dtype)
    dO = draw((B, T, H, d), seed + 3, dtype)
    sl = torch.tensor([2.0 ** (-1 - h) for h in range(H)], device="cuda") if slopes else None
    p = api.attn_params(B, T, H, H_kv, d, T_k=T_k, dtype=dtype, causal=causal, window=window, cap=cap, exact=exact)
    more = dict(slopes=sl, cu_seqlens=cu, prefix=prefix)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = api.lawcat_attn_fwd(p, q, k, v, dev_status=status, **more)
    see = visible(T, T_k, causal, window, cu, prefix, B)
    ref = attention(q, k, v, see, float(torch.tensor(d ** -0.5)), cap if ref_cap is None else ref_cap, sl, dO, r["o"])
    coarse = U16 if dtype == "bf16" and not exact else 0.0     # the tensor-core kernels round weights to bf16
    out = U16 if dtype == "bf16" else U32
    check(r["o"], ref["o"], ref["o_sum"] + coarse * ref["o_mag"], out, "o")
    check(r["lse"], ref["lse"], ref["lse_err"], U32, "lse")
    if grad:
        g = api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, dev_status=status, **more)
        err = ref["grad_err"](coarse, out)
        for n in ("dq", "dk", "dv"):
            check(g[n], ref[n], err[n], out, n)
        r.update(g)
    assert int(status.item()) == 0
    return p, (q, k, v, dO), r


KINDS = [("f32", 0), ("bf16", 1), ("bf16", 0)]  # (storage type, exact)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("T", [1, 2, 17, 63, 64, 65, 127, 128, 129, 200, 257, 385])
def test_lengths(T, dtype, exact):
    case(T=T, dtype=dtype, exact=exact, B=2, seed=T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (6, 2), (8, 1), (5, 5)])
def test_heads_and_widths(H, H_kv, d, dtype, exact):
    case(T=150, H=H, H_kv=H_kv, d=d, dtype=dtype, exact=exact, seed=H + d)


MASKS = [
    dict(causal=0), dict(causal=0, cap=8.0, slopes=True), dict(window=1), dict(window=64), dict(window=7, causal=0), dict(window=1000),
    dict(window=130, slopes=True), dict(window=2 ** 31 - 1, causal=0), dict(cap=5.0), dict(slopes=True), dict(cap=30.0, slopes=True),
    dict(prefix=[0, 300]), dict(prefix=[129, 64], slopes=True, cap=20.0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("i", range(len(MASKS)))
def test_masks(i, d, dtype, exact):
    case(B=2, T=300, d=d, dtype=dtype, exact=exact, seed=50 + i, **MASKS[i])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
def test_a_cap_far_above_the_scores(dtype, exact):
    """No cap, up to some steps of 2^-24 of the scores, which their bound has room for: none of the cap's."""
    case(T=200, dtype=dtype, exact=exact, seed=9, cap=1e6, ref_cap=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("T,T_k", [(1, 300), (5, 300), (77, 500), (130, 131), (300, 1), (300, 200), (64, 0), (0, 64), (129, 600)])
@pytest.mark.parametrize("kw", [dict(), dict(causal=0), dict(window=40), dict(window=40, causal=0, cap=6.0, slopes=True)])
def test_other_number_of_keys(T, T_k, kw, dtype, exact):
    """Pieces of a prompt behind a past; more queries than keys (the first ones see nothing); no keys, no queries at all."""
    p, _, r = case(B=2, T=T, T_k=T_k, dtype=dtype, exact=exact, seed=T + T_k, **kw)
    if T > T_k and kw.get("causal", 1):
        assert not r["o"][:, :T - T_k].any() and (r["lse"][:, :T - T_k] == -math.inf).all() and not r["dq"][:, :T - T_k].any()
    if T == 0:
        assert not r["dk"].any() and not r["dv"].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("kw", [dict(), dict(causal=0), dict(causal=0, T_k=1100), dict(causal=0, T_k=150), dict(prefix=[0, 390, 200]), dict(causal=0, cap=7.0), dict(window=90)])
def test_steep_biases(kw, dtype, exact):
    """Slopes from far above one to below zero, keys on both sides, queries in front of the first key."""
    steep_case(dtype, exact, **kw)


def steep_case(dtype, exact, causal=1, T_k=None, prefix=None, cap=0.0, window=0):
    B, T, H, H_kv, d = 3, 400, 6, 2, 64
    T_k = T if T_k is None else T_k
    q, k, v, dO = [draw((B, n, h, d), 60 + i, dtype, 1.5 if i == 0 else 1.0) for i, (n, h) in enumerate(((T, H), (T_k, H_kv), (T_k, H_kv), (T, H)))]
    sl = torch.tensor([1.3, -0.4, 9.0, 0.84, 2.9, -1.2], device="cuda")
    p = api.attn_params(B, T, H, H_kv, d, T_k=T_k, dtype=dtype, causal=causal, window=window, cap=cap, exact=exact)
    r = api.lawcat_attn_fwd(p, q, k, v, slopes=sl, prefix=prefix)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, slopes=sl, prefix=prefix))
    ref = attention(q, k, v, visible(T, T_k, causal, window, None, prefix, B), float(torch.tensor(d ** -0.5)), cap, sl, dO, r["o"])
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    err = dict(ref["grad_err"](coarse, out), o=ref["o_sum"] + coarse * ref["o_mag"], lse=ref["lse_err"])
    # A key far from every query has weights around fp32's least normal number 2^-126; one below it counts as zero, so that each of a key's
    # T H / H_kv weights is off by 2^-126 at most. dv sums p dO; dk sums scale p (dP - D) q with |dP|, |D| <= d max|dO| max|v|.
    top = [float(x.double().abs().max()) for x in (q, v, dO)]
    lost = T * H // H_kv * 2.0 ** -126
    tiny = dict(dv=lost * top[2], dk=lost * d ** -0.5 * 2 * d * top[2] * top[1] * top[0])
    for n in ("o", "lse", "dq", "dk", "dv"):
        check(r[n], ref[n], err[n], U32 if n == "lse" else out, n, 1e-37 + tiny.get(n, 0.0))


DOCS = [
    ([0, 300], None), ([0, 1, 300], None), ([0, 0, 128, 128, 256, 300, 300], None), ([0, 63, 64, 65, 130, 299, 300], None),
    ([0, 100, 300], [100, 0]), ([0, 40, 41, 300], [13, 1, 200]), (list(range(0, 301)), None), (list(range(0, 301, 4)), [3] * 75),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cu,prefix", DOCS)
def test_documents(cu, prefix, d, dtype, exact):
    case(T=300, d=d, dtype=dtype, exact=exact, cu=cu, prefix=prefix, seed=len(cu), cap=0.0 if prefix else 10.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_documents_than_one_table(dtype):
    """700 documents (three launches of the interval table) among them empty ones; and a window inside documents."""
    cu = [0]
    for i in range(700):
        cu.append(cu[-1] + (i * 7) % 4)
    case(T=cu[-1], H=2, H_kv=1, dtype=dtype, cu=cu, seed=9)
    case(T=cu[-1], H=2, H_kv=1, dtype=dtype, cu=[0, 500, cu[-1]], window=33, seed=10)


@pytest.mark.gpu
def test_more_tiles_of_documents_than_are_put_in_order():
    """140400 packed tokens, 1097 tiles of keys: the first, the last and some other documents."""
    n, T, d = 260, 540, 64
    q, k, v, dO = [draw((1, n * T, h, d), i, "bf16") for i, h in enumerate((2, 1, 1, 2))]
    p = api.attn_params(1, n * T, 2, 1, d)
    cu = list(range(0, n * T + 1, T))
    r = api.lawcat_attn_fwd(p, q, k, v, cu_seqlens=cu)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, cu_seqlens=cu))
    one = [0, 1, 130, 255, 256, 259]
    part = lambda x: x.reshape(n, T, *x.shape[2:])[one]  # noqa: E731
    ref = attention(part(q), part(k), part(v), visible(T, T, 1, 0, B=len(one)), float(torch.tensor(d ** -0.5)), 0.0, None, part(dO), part(r["o"]))
    err = dict(ref["grad_err"](U16, U16), o=ref["o_sum"] + U16 * ref["o_mag"], lse=ref["lse_err"])
    for x in ("o", "lse", "dq", "dk", "dv"):
        check(part(r[x]), ref[x], err[x], U32 if x == "lse" else U16, x)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
def test_the_same_call_gives_the_same_bits(dtype, exact):
    a = case(B=2, T=333, H=8, H_kv=2, dtype=dtype, exact=exact, cap=9.0, seed=3)[2]
    b = case(B=2, T=333, H=8, H_kv=2, dtype=dtype, exact=exact, cap=9.0, seed=3)[2]
    for n in a:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("T", [70, 300])
def test_rows_that_are_not_seen_stay_out(T, bad, dtype, exact):
    """A NaN or an infinity in keys and values that only later queries see, and in another document's rows, changes no bit of
    the other queries' results. (The tensor-core kernels compute the rows of a block that came out not finite again on the CUDA
    cores, where the weights are not rounded to bf16: those stay within the tolerance instead.)"""
    d, H, H_kv, at = 64, 4, 2, T - 13
    q, k, v = draw((1, T, H, d), 1, dtype), draw((1, T, H_kv, d), 2, dtype), draw((1, T, H_kv, d), 3, dtype)
    dO = draw((1, T, H, d), 4, dtype)
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    for kw in (dict(), dict(cu_seqlens=[0, at, T])):
        p = api.attn_params(1, T, H, H_kv, d, dtype=dtype, exact=exact)
        clean = api.lawcat_attn_fwd(p, q, k, v, **kw)
        clean.update(api.lawcat_attn_bwd(p, q, k, v, clean["o"], clean["lse"], dO, **kw))
        k2, v2, q2, dO2 = k.clone(), v.clone(), q.clone(), dO.clone()
        for x in (k2, v2, q2, dO2):
            x[:, at:, :, 5] = bad
        r = api.lawcat_attn_fwd(p, q2, k2, v2, **kw)
        r.update(api.lawcat_attn_bwd(p, q2, k2, v2, r["o"], r["lse"], dO2, **kw))
        names = ["o", "lse", "dq"] + (["dk", "dv"] if "cu_seqlens" in kw else [])
        if not coarse:
            for n in names:
                assert torch.equal(r[n][:, :at], clean[n][:, :at]), n
            continue
        ref = attention(q, k, v, visible(T, T, 1, 0, kw.get("cu_seqlens")), 0.125, 0.0, None, dO, r["o"].nan_to_num(0, 0, 0))
        err = dict(ref["grad_err"](coarse, out), o=ref["o_sum"] + coarse * ref["o_mag"], lse=ref["lse_err"])
        for n in names:
            check(r[n][:, :at], ref[n][:, :at], err[n][:, :at], U32 if n == "lse" else out, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
def test_large_scores(dtype, exact):
    """Scores of several hundred: the running maximum moves by more than an exponential holds, down and up along the keys."""
    d, T = 64, 400
    q, k, v = draw((1, T, 2, d), 1, dtype, 8.0), draw((1, T, 2, d), 2, dtype, 8.0), draw((1, T, 2, d), 3, dtype)
    k *= torch.linspace(-2, 2, T, device="cuda").reshape(1, T, 1, 1).to(k.dtype)
    p = api.attn_params(1, T, 2, 2, d, dtype=dtype, exact=exact)
    r = api.lawcat_attn_fwd(p, q, k, v)
    ref = attention(q, k, v, visible(T, T, 1, 0), 0.125)
    coarse = U16 if dtype == "bf16" and not exact else 0.0
    check(r["o"], ref["o"], ref["o_sum"] + coarse * ref["o_mag"], U16 if dtype == "bf16" else U32, "o")
    check(r["lse"], ref["lse"], ref["lse_err"], U32, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(), dict(cap=4.0, slopes=True), dict(window=9), dict(cu=[0, 11, 40])])
def test_gradients_against_differences(kw):
    """Along a random direction of (q, k, v): the gradients' product with it against central differences of sum(dO o) in 64 bits. The
    differences' truncation (what they are off the 64-bit gradients) and the gradients' own tolerance add up."""
    p, (q, k, v, dO), r = case(T=40, H=4, H_kv=2, d=32, dtype="f32", seed=21, **kw)
    slopes = torch.tensor([2.0 ** (-1 - h) for h in range(4)], device="cuda") if kw.get("slopes") else None
    see = visible(40, 40, 1, kw.get("window", 0), kw.get("cu"))
    d = [draw(x.shape, 30 + i, "f32").double() for i, x in enumerate((q, k, v))]
    h = 2.0 ** -12
    scale = float(torch.tensor(32 ** -0.5))
    loss = lambda s: float((attention(*[x.double() + s * e for x, e in zip((q, k, v), d)], see, scale, kw.get("cap", 0.0), slopes)["o"] * dO.double()).sum())  # noqa: E731
    diff = (loss(h) - loss(-h)) / (2 * h)
    full = attention(q, k, v, see, scale, kw.get("cap", 0.0), slopes, dO, r["o"])
    dot = lambda g: float(sum((g[n].double() * e).sum() for n, e in zip(("dq", "dk", "dv"), d)))  # noqa: E731
    err = full["grad_err"](0.0, U32)
    tol = float(sum(((err[n] + U32 * full[n].abs()) * e.abs()).sum() for n, e in zip(("dq", "dk", "dv"), d)))
    trunc = abs(diff - dot(full))
    assert abs(diff - dot(r)) <= tol + trunc, (diff, dot(r), tol, trunc)
    assert trunc < 1e-4 * (1 + abs(diff))   # (the 64-bit gradients are those of the 64-bit definition)


@pytest.mark.gpu
def test_streams_graphs_and_given_outputs():
    """On a side stream, captured and replayed with other inputs in the same places (two graphs in turn), into given outputs."""
    T, H, H_kv, d = 200, 4, 2, 64
    p = api.attn_params(1, T, H, H_kv, d)
    x = [draw((1, T, h, d), i, "bf16") for i, h in enumerate((H, H_kv, H_kv, H))]
    y = [draw((1, T, h, d), 10 + i, "bf16") for i, h in enumerate((H, H_kv, H_kv, H))]
    kw = dict(cu_seqlens=[0, 77, T], prefix=[5, 100])

    def run(z):
        r = api.lawcat_attn_fwd(p, *z[:3], **kw)
        r.update(api.lawcat_attn_bwd(p, *z[:3], r["o"], r["lse"], z[3], **kw))
        return r
    want_x, want_y = run(x), run(y)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = torch.full_like(x[0], 7.0)
    api.lawcat_attn_fwd(p, *x[:3], o=o, want_lse=False, stream=side, **kw)
    side.synchronize()
    assert torch.equal(o, want_x["o"])
    buf = [t.clone() for t in x]
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run(buf)
        graphs.append((g, out))
    for z, want in ((x, want_x), (y, want_y), (x, want_x)):
        for b, s in zip(buf, z):
            b.copy_(s)
        for g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for n in want:
                assert torch.equal(out[n], want[n]), n


@pytest.mark.gpu
def test_teacher_student_and_hybrid_together():
    """As they are used: softmax attention gives the target of a layer's distillation (packed documents), the layer its output, the
    difference of the two goes back through the layer; and a window layer's forward over a prompt continues as decode steps, in
    the storage type and in 4 bits."""
    T, H, H_kv, d, lens = 160, 4, 2, 64, [0, 70, 160]
    q, k, v = draw((1, T, H, d), 1, "bf16"), draw((1, T, H_kv, d), 2, "bf16"), draw((1, T, H_kv, d), 3, "bf16")
    p = api.attn_params(1, T, H, H_kv, d)
    target = api.lawcat_attn_fwd(p, q, k, v, cu_seqlens=lens, want_lse=False)["o"]
    lp = api.params(1, 70, H, H_kv, d, d)
    gate = draw((1, 70, H, d), 4, "bf16")
    w = [draw((H * d, 4), 5, "bf16", 0.5), draw((H_kv * d, 4), 6, "bf16", 0.5), draw((H, d, d), 7, "bf16", d ** -0.5)]
    o = api.lawcat_layer_fwd(lp, q[:, :70].contiguous(), k[:, :70].contiguous(), v[:, :70].contiguous(), gate, *w)["o"]
    dO = ((o.float() - target[:, :70].float()) * (2.0 / o.numel())).bfloat16()
    g = api.lawcat_layer_bwd(lp, q[:, :70].contiguous(), k[:, :70].contiguous(), v[:, :70].contiguous(), gate, *w, dO)
    assert all(torch.isfinite(t).all() for t in g.values()) and float(g["dW"].abs().max()) > 0
    # a window layer: the prompt at once, and its last 30 tokens one by one over a ring of 48 slots
    win, n = 48, 130
    pw = api.attn_params(1, T, H, H_kv, d, window=win)
    whole = attention(q, k, v, visible(T, T, 1, win), 0.125)
    o = api.lawcat_attn_fwd(pw, q, k, v, want_lse=False)["o"]
    check(o, whole["o"], whole["o_sum"] + U16 * whole["o_mag"], U16, "prompt")
    pd = api.attn_params(1, 1, H, H_kv, d, T_k=win, window=win)
    K, V = torch.zeros(1, win, H_kv, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, win, H_kv, d, dtype=torch.bfloat16, device="cuda")
    for t in range(n - win, n):
        K[:, t % win], V[:, t % win] = k[:, t], v[:, t]
    pc = api.attn_params(1, n, H, H_kv, d, T_k=win, window=win)
    cache = api.quant_cache(pc)
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.lawcat_cache_quantize(pc, k[:, :n].contiguous(), v[:, :n].contiguous(), pos, *cache)
    pos += n
    for t in range(n, T):
        step = [x[:, t].contiguous() for x in (q, k, v)]
        o1 = api.lawcat_attn_decode(pd, *step, K, V, pos)
        check(o1, whole["o"][:, t], whole["o_sum"][:, t] + U16 * whole["o_mag"][:, t], U16, f"step {t}")
        o4 = api.lawcat_attn_decode_quant(pd, *step, *cache, pos)
        assert torch.isfinite(o4).all() and float((o4 - o1).float().norm() / o1.float().norm()) < 0.5  # (a 16-level cache)
        pos += 1


@pytest.mark.gpu
def test_which_kernels_run():
    """bf16 and widths 64 and 128 run on the tensor cores unless exact results are asked for."""
    def names(**kw):
        api.trace_begin()
        case(T=70, seed=1, **kw)
        return set(api.trace_end())
    tc, exact = {"attn_fwd_tc", "attn_dq_tc", "attn_dkdv_tc"}, {"attn_fwd_exact", "attn_dq_exact", "attn_dkdv_exact"}
    for d in (64, 128):
        assert names(d=d) == tc
        assert names(d=d, exact=1) >= exact and not names(d=d, exact=1) & tc
    assert names(d=32) >= exact and names(d=64, dtype="f32") >= exact
    assert "attn_rows" in names(cu=[0, 30, 70])


@pytest.mark.gpu
@pytest.mark.parametrize("d,kw", [(64, dict()), (128, dict(cap=25.0)), (64, dict(window=3000, slopes=True))])
def test_long_sequence_on_its_last_rows(d, kw):
    """70001 tokens: the last 200 queries (which see all of them, or the window), and the last 200 keys, which no other query sees."""
    T, n, H = 70001, 200, 2
    q, k, v, dO = [draw((1, T, h, d), i, "bf16", 1.5 if i == 0 else 1.0) for i, h in enumerate((H, 1, 1, H))]
    sl = torch.tensor([0.01, 0.001], device="cuda") if kw.get("slopes") else None
    p = api.attn_params(1, T, H, 1, d, window=kw.get("window", 0), cap=kw.get("cap", 0.0))
    r = api.lawcat_attn_fwd(p, q, k, v, slopes=sl)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, slopes=sl))
    last = lambda x: x[:, -n:]  # noqa: E731
    ref = attention(last(q), k, v, visible(n, T, 1, kw.get("window", 0)), float(torch.tensor(d ** -0.5)), kw.get("cap", 0.0), sl, last(dO), last(r["o"]))
    err = dict(ref["grad_err"](U16, U16), o=ref["o_sum"] + U16 * ref["o_mag"], lse=ref["lse_err"])
    for x in ("o", "lse", "dq", "dk", "dv"):
        want, e = (ref[x], err[x]) if ref[x].shape[1] == n else (last(ref[x]), last(err[x]))
        check(last(r[x]), want, e, U32 if x == "lse" else U16, x)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,window", [(50, 0), (1000, 1)])
def test_many_items_of_one_tile(T, window, d):
    """Thousands of items that meet one or two tiles of keys each: the roles of a block are then several items apart."""
    B, H, H_kv = (1500, 4, 2) if T == 50 else (40, 8, 4)
    q, k, v, dO = [draw((B, T, h, d), i, "bf16") for i, h in enumerate((H, H_kv, H_kv, H))]
    p = api.attn_params(B, T, H, H_kv, d, window=window)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for again in range(3):
        r = api.lawcat_attn_fwd(p, q, k, v, dev_status=status)
        r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, dev_status=status))
        assert int(status.item()) == 0
        for b in range(0, B, 100 if T == 50 else 10):
            s = slice(b, b + 20 if T == 50 else b + 2)
            ref = attention(q[s], k[s], v[s], visible(T, T, 1, window, B=len(q[s])), float(torch.tensor(d ** -0.5)), 0.0, None, dO[s], r["o"][s])
            err = dict(ref["grad_err"](U16, U16), o=ref["o_sum"] + U16 * ref["o_mag"], lse=ref["lse_err"])
            for n in ("o", "lse", "dq", "dk", "dv"):
                check(r[n][s], ref[n], err[n], U32 if n == "lse" else U16, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("kw", [dict(T=200), dict(T=77, T_k=900), dict(T=150, causal=0, cap=9.0), dict(T=300, cu=[0, 90, 300])])
def test_what_the_scratch_held_makes_no_difference(kw, dtype, exact):
    """The same bits over scratch full of zeros and full of NaN (a row that came out not finite would be computed in another way)."""
    T, T_k, cu = kw["T"], kw.get("T_k", kw["T"]), kw.get("cu")
    B, H, H_kv, d = 1 if cu else 2, 4, 2, 64
    q, k, v, dO = [draw((B, n, h, d), i, dtype) for i, (n, h) in enumerate(((T, H), (T_k, H_kv), (T_k, H_kv), (T, H)))]
    p = api.attn_params(B, T, H, H_kv, d, T_k=T_k, dtype=dtype, exact=exact, causal=kw.get("causal", 1), cap=kw.get("cap", 0.0))
    n = [api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), op) for op in (api.OP_ATTN_FWD, api.OP_ATTN_BWD)]
    got = []
    for fill in (0, 255):
        ws = [torch.full((max(x, 1),), fill, dtype=torch.uint8, device="cuda") for x in n]
        r = api.lawcat_attn_fwd(p, q, k, v, cu_seqlens=cu, ws=ws[0])
        r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, cu_seqlens=cu, ws=ws[1]))
        got.append(r)
    for x in got[0]:
        assert torch.equal(got[0][x], got[1][x]), x


@pytest.mark.gpu
def test_two_calls_at_once():
    """Different calls on two streams, many blocks each, over and over: the results of the calls one after the other."""
    T, H, H_kv, d = 700, 8, 2, 64
    p = api.attn_params(2, T, H, H_kv, d, cap=9.0)
    sets = [[draw((2, T, h, d), 10 * s + i, "bf16") for i, h in enumerate((H, H_kv, H_kv, H))] for s in range(2)]

    def run(x, stream=None):
        r = api.lawcat_attn_fwd(p, *x[:3], stream=stream)
        r.update(api.lawcat_attn_bwd(p, *x[:3], r["o"], r["lse"], x[3], stream=stream))
        return r
    want = [run(x) for x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(6):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(run(sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            for n in want[i]:
                assert torch.equal(r[n], want[i][n]), n


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_a_wait_that_runs_out_is_reported(d):
    """With a bound of a few hundred clock cycles, less than any copy or product takes, the kernels' roles give up on one another: each
    call ends and says so, and the next one, with the bound restored, is right."""
    T, H, H_kv, B = 500, 4, 2, 2
    x = [draw((B, T, h, d), i, "bf16") for i, h in enumerate((H, H_kv, H_kv, H))]
    p, pd = api.attn_params(B, T, H, H_kv, d), api.attn_params(B, 1, H, H_kv, d, T_k=T)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = torch.full((B,), T - 1, dtype=torch.int32, device="cuda")
    cache = api.quant_cache(pd)
    api.lawcat_cache_quantize(api.attn_params(B, T, H, H_kv, d, T_k=T), x[1], x[2], torch.zeros_like(pos), *cache)
    step = [t[:, -1].contiguous() for t in x[:3]]
    calls = dict(fwd=lambda: api.lawcat_attn_fwd(p, *x[:3], dev_status=status)["o"],
                 bwd=lambda: api.lawcat_attn_bwd(p, *x[:3], good["o"], good["lse"], x[3], dev_status=status)["dk"],
                 decode=lambda: api.lawcat_attn_decode(pd, *step, x[1].clone(), x[2].clone(), pos, dev_status=status),
                 quant=lambda: api.lawcat_attn_decode_quant(pd, *step, *[t.clone() for t in cache], pos, dev_status=status))
    good = api.lawcat_attn_fwd(p, *x[:3])
    want = {n: f() for n, f in calls.items()}
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for n, f in calls.items():
        api.test_set_wait_limit(300)
        try:
            f()
            torch.cuda.synchronize()
        finally:
            api.test_set_wait_limit(0)
        assert int(status.item()) == 5, n
        status.zero_()
        assert torch.equal(f(), want[n]), n
        assert int(status.item()) == 0


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
@pytest.fixture(scope="module")
def L():
    build.build()
    return api.lib()


OK, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)
BASE = dict(B=1, T=8, H=4, H_kv=2, d=64)


def fwd_status(L, kw, cu=None, prefix=None, nseq=0, ptrs=None, ws=OK, nws=1 << 20):
    p = api.attn_params(**{**BASE, **kw})
    arr = lambda x: None if x is None else (ctypes.c_int32 * max(1, len(x)))(*x)  # noqa: E731
    return L.lawcat_attn_fwd(ctypes.byref(p), arr(cu), arr(prefix), nseq, *(ptrs or [OK, OK, OK, None, OK, None]), ws, nws, None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(H_kv=3), 1), (dict(T=-1), 1), (dict(T_k=-1), 1), (dict(B=-1), 1), (dict(H=0), 1), (dict(H_kv=0), 1), (dict(dtype=2), 1),
    (dict(causal=2), 1), (dict(exact=-1), 1), (dict(window=-1), 1), (dict(scale=math.nan), 1), (dict(scale=math.inf), 1),
    (dict(cap=-1.0), 1), (dict(cap=math.inf), 1), (dict(d=48), 2), (dict(d=256), 2), (dict(T=(1 << 30) + 1), 2),
    (dict(T_k=(1 << 30) + 1), 2), (dict(B=1 << 27), 2)])
def test_bad_parameters(L, kw, status):
    assert fwd_status(L, kw) == status
    p = api.attn_params(**{**BASE, **kw})
    assert L.lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_FWD) == 0
    assert L.lawcat_attn_bwd(ctypes.byref(p), None, None, 0, *[OK] * 3, None, *[OK] * 6, OK, 1 << 20, None, None) == status
    assert L.lawcat_attn_decode(ctypes.byref(p), *[OK] * 6, None, OK, OK, 1 << 20, None, None) == status


@pytest.mark.parametrize("kw,cu,prefix,nseq", [
    (dict(), [1, 8], None, 1), (dict(), [0, 7], None, 1), (dict(), [0, 9], None, 1), (dict(), [0, 5, 4, 8], None, 3), (dict(B=2), [0, 8], None, 1),
    (dict(T_k=9), [0, 8], None, 1), (dict(), [0, 8], None, -1), (dict(), None, None, 1), (dict(), None, [0, 0], 2), (dict(), None, [9], 1),
    (dict(), None, [-1], 1), (dict(causal=0), None, [1], 1), (dict(window=3), None, [1], 1), (dict(), [0, 4, 8], [4, 5], 2), (dict(), None, [1], -1)])
def test_bad_documents(L, kw, cu, prefix, nseq):
    assert fwd_status(L, kw, cu, prefix, nseq) == 1


def test_bad_pointers_and_scratch(L):
    good = [OK, OK, OK, None, OK, None]
    for i in (0, 1, 2, 4):
        assert fwd_status(L, {}, ptrs=[None if j == i else x for j, x in enumerate(good)]) == 1
    for i in range(6):
        assert fwd_status(L, {}, ptrs=[ODD if j == i else x for j, x in enumerate(good)]) == 1
    p = api.attn_params(**BASE)
    need = L.lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_FWD)
    assert need > 0
    assert fwd_status(L, {}, nws=need - 1) == 4 and fwd_status(L, {}, ws=None) == 4
    assert fwd_status(L, dict(B=0), ptrs=[None] * 6, ws=None, nws=0) == 0   # nothing to do
    b = lambda x, ws=OK, n=1 << 20: L.lawcat_attn_bwd(ctypes.byref(p), None, None, 0, *x, ws, n, None, None)  # noqa: E731
    good = [OK, OK, OK, None, OK, OK, OK, OK, OK, OK]
    for i in (0, 1, 2, 4, 5, 6, 7, 8, 9):
        assert b([None if j == i else x for j, x in enumerate(good)]) == 1
        assert b([ODD if j == i else x for j, x in enumerate(good)]) == 1
    assert b(good, n=16) == 4 and b(good, ws=None) == 4


@pytest.mark.parametrize("name,nptr,opt", [("lawcat_attn_decode", 8, {6}), ("lawcat_attn_decode_quant", 10, {8}), ("lawcat_cache_quantize", 7, set()),
                                           ("lawcat_cache_dequantize", 7, set())])
def test_bad_cache_calls(L, name, nptr, opt):
    f = getattr(L, name)
    call = lambda p, x, ws=OK, n=1 << 30: f(ctypes.byref(p), *x, ws, n, None, None)  # noqa: E731
    p = api.attn_params(1, 1, 4, 2, 64, T_k=100)
    for i in range(nptr):
        if i not in opt:
            assert call(p, [None if j == i else OK for j in range(nptr)]) == 1
        assert call(p, [ODD if j == i else OK for j in range(nptr)]) == 1
    assert call(api.attn_params(1, 1, 4, 2, 64, T_k=0), [OK] * nptr) == 1               # no slots
    assert call(api.attn_params(1, 1, 4, 2, 64, T_k=100, window=101), [OK] * nptr) == 1  # a window that the ring does not hold
    assert call(api.attn_params(1, 1, 4, 2, 48, T_k=100), [OK] * nptr) == 2
    assert call(api.attn_params(0, 1, 4, 2, 64, T_k=100), [None] * nptr, None, 0) == 0
    if "decode" in name:
        big = api.attn_params(1, 1, 4, 2, 64, T_k=4096)
        assert L.lawcat_attn_workspace_bytes(ctypes.byref(big), api.OP_ATTN_DECODE) > 0
        assert call(big, [OK] * nptr, OK, 16) == 4 and call(big, [OK] * nptr, None, 0) == 4


def test_python_checks_shapes_and_types():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    p = api.attn_params(1, 8, 4, 2, 64)
    q, k = z(1, 8, 4, 64), z(1, 8, 2, 64)
    bad = [dict(q=z(1, 8, 2, 64)), dict(k=z(1, 7, 2, 64)), dict(v=z(1, 8, 2, 64, dt=torch.float16)), dict(q=q.float()),
           dict(slopes=z(4)), dict(slopes=z(5, dt=torch.float32)), dict(o=z(1, 8, 4, 32)), dict(cu_seqlens=[]),
           dict(cu_seqlens=[0, 8], prefix=[1, 2])]
    for kw in bad:
        with pytest.raises(ValueError):
            api.lawcat_attn_fwd(p, **{**dict(q=q, k=k, v=k), **kw})
    pd = api.attn_params(1, 1, 4, 2, 64, T_k=16)
    for pos in (z(1, dt=torch.int64), z(2, dt=torch.int32)):
        with pytest.raises(ValueError):
            api.lawcat_attn_decode(pd, z(1, 4, 64), z(1, 2, 64), z(1, 2, 64), z(1, 16, 2, 64), z(1, 16, 2, 64), pos)


def test_struct_matches_header():
    import os
    import re
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lawcat.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\} lawcat_attn_params;", re.sub(r"/\*.*?\*/", "", hdr, flags=re.S), re.S).group(1)
    names = [n.strip() for d in body.split(";") if d.strip() for n in d.strip().split(None, 1)[1].split(",")]
    assert names == [f[0] for f in api.AttnParams._fields_]
    assert ctypes.sizeof(api.AttnParams) == 4 * len(names)
