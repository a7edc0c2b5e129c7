"""One step of softmax attention over a cache, in the storage type and in 4 bits, and the 4-bit cache itself, against 64 bits
(attn_reference.py): rings that wrap, windows, slots that hold no token, sequences that are not there, every head grouping."""
import ctypes
import math

import pytest
import torch

from attn_reference import U16, U32, attention, check, quantized
from paper_2509_18467_b200 import api
from test_attn import DT, draw

pytestmark = pytest.mark.gpu


def rows_of(cache, b, slots):
    """A 4-bit cache's rows as 64-bit values: two of [n, H_kv, d]."""
    out = []
    for q, p in (cache[:2], cache[2:]):
        byte, pr = q[b][:, slots].long(), p[b][:, slots].double()
        n = q.shape[-1] * 2
        code = torch.stack([byte % 16, byte // 16], -1).reshape(*byte.shape[:-1], n).double()
        rep = n // pr.shape[-2]
        out.append((pr[..., 1].repeat_interleave(rep, -1) + code * pr[..., 0].repeat_interleave(rep, -1)).transpose(0, 1))
    return out


def step(quant, pos, C=100, H=4, H_kv=2, d=64, dtype="bf16", window=0, cap=0.0, slopes=False, exact=0, seed=0, garbage=math.nan, ref_cap=None):
    """One step for sequences at positions `pos`; slots without a token hold `garbage`."""
    B = len(pos)
    q, k, v = draw((B, H, d), seed, dtype, 1.5), draw((B, H_kv, d), seed + 1, dtype), draw((B, H_kv, d), seed + 2, dtype)
    pasts = [draw((B, C, H_kv, d), seed + 3 + i, dtype) for i in range(2)]
    sl = torch.tensor([2.0 ** (-3 - h % 8) for h in range(H)], device="cuda") if slopes else None
    p = api.attn_params(B, 1, H, H_kv, d, T_k=C, dtype=dtype, window=window, cap=cap, exact=exact)
    at = torch.tensor(pos, dtype=torch.int32, device="cuda")
    if quant:
        cache = api.quant_cache(p)
        pc = api.attn_params(B, C, H, H_kv, d, T_k=C, dtype=dtype)
        api.lawcat_cache_quantize(pc, pasts[0], pasts[1], torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    else:
        cache = tuple(x.clone() for x in pasts)
    for b, x in enumerate(pos):
        if x < 0 or x < C - 1:
            for t in cache:
                part = t[b][:, max(0, x + 1):] if quant else t[b][max(0, x + 1):]
                part.fill_(garbage if t.dtype != torch.uint8 else 255)
    before = [t.clone() for t in cache]
    if quant:
        o = api.lawcat_attn_decode_quant(p, q, k, v, *cache, at, slopes=sl)
    else:
        o = api.lawcat_attn_decode(p, q, k, v, *cache, at, slopes=sl)
    coarse = U16 if dtype == "bf16" and not exact else 0.0
    out = U16 if dtype == "bf16" else U32
    for b, x in enumerate(pos):
        if x < 0:
            assert not o[b].any()
            for t, was in zip(cache, before):
                assert torch.equal(t[b].view(torch.uint8), was[b].view(torch.uint8))
            continue
        n = min(x + 1, C, window or C)
        slots = torch.arange(x - n + 1, x + 1, device="cuda") % C
        if quant:
            K, V = rows_of(cache, b, slots)
            for new, got in ((k, K), (v, V)):
                assert torch.equal(got[-1], quantized(new[b])[3])
        else:
            K, V = cache[0][b][slots], cache[1][b][slots]
            assert torch.equal(K[-1], k[b]) and torch.equal(V[-1], v[b])
        other = torch.ones(C, dtype=torch.bool, device="cuda")
        other[x % C] = False
        for t, was in zip(cache, before):   # no other slot is written
            a, c = (t[b][:, other], was[b][:, other]) if quant else (t[b][other], was[b][other])
            assert torch.equal(a.contiguous().view(torch.uint8), c.contiguous().view(torch.uint8))
        see = torch.ones(1, 1, n, dtype=torch.bool)
        ref = attention(q[b][None, None], K[None], V[None], see, float(torch.tensor(d ** -0.5)), cap if ref_cap is None else ref_cap, sl)
        more = 0.0
        if quant:  # products with codes and with the minimum apart: each is as large as 32 times the largest value at most in fp32,
            # and a rounded weight meets scale times code, at most twice the largest value
            kmax, vmax = float(K.abs().max()), float(V.abs().max())
            dx = (2 * d + 16) * U32 * float(q[b].double().abs().sum(-1).max()) * 32 * kmax * d ** -0.5
            more = 2 * dx * ref["o_mag"] + (n + 64) * U32 * 32 * vmax + coarse * 2 * vmax
        check(o[b][None, None], ref["o"], ref["o_sum"] + coarse * ref["o_mag"] + more, out, f"o of sequence {b} at {x}")
    return o


@pytest.mark.parametrize("dtype,exact", [("f32", 0), ("bf16", 1), ("bf16", 0)])
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("pos,C", [([0], 1), ([0, 1, 62, 63, 64, 65], 100), ([99, 100, 101, 250, -1, 7], 100), ([5, 700, -5, 1299], 1300), ([12345], 1300)])
def test_positions(pos, C, quant, dtype, exact):
    step(quant, pos, C, dtype=dtype, exact=exact, seed=len(pos) + C)


@pytest.mark.parametrize("dtype,exact", [("f32", 0), ("bf16", 1), ("bf16", 0)])
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (8, 8), (12, 4), (8, 1), (20, 2), (32, 1)])
def test_heads_and_widths(H, H_kv, d, quant, dtype, exact):
    step(quant, [40, 333, 600], 400, H=H, H_kv=H_kv, d=d, dtype=dtype, exact=exact, seed=H + d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("kw", [dict(window=1), dict(window=64), dict(window=333, slopes=True), dict(cap=4.0), dict(cap=20.0, slopes=True), dict(slopes=True)])
def test_windows_caps_and_biases(kw, quant, dtype):
    step(quant, [0, 63, 64, 500, 1111], 600, dtype=dtype, d=128, H=8, H_kv=2, seed=7, **kw)


@pytest.mark.parametrize("dtype,exact", [("f32", 0), ("bf16", 1), ("bf16", 0)])
@pytest.mark.parametrize("quant", [False, True])
def test_a_cap_far_above_the_scores(quant, dtype, exact):
    """No cap, up to some steps of 2^-24 of the scores, which their bound has room for: none of the cap's."""
    step(quant, [0, 77, 300, 1111], 400, dtype=dtype, exact=exact, H=8, H_kv=2, seed=11, cap=1e6, ref_cap=0.0)


@pytest.mark.parametrize("quant", [False, True])
def test_long_cache(quant):
    """Many parts per sequence, lengths from one token on, and positions near the end of 32 bits."""
    step(quant, [0, 300, 9000, 20000, 2 ** 31 - 1], 9000, H=8, H_kv=2, d=128, seed=5)


def test_offsets_beyond_32_bits():
    """A cache of more than 2^31 elements: the last sequence's slots lie behind them."""
    B, C, H, H_kv, d = 17, 262144, 4, 4, 128
    p = api.attn_params(B, 1, H, H_kv, d, T_k=C, window=50)
    K = torch.zeros(B, C, H_kv, d, dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    pos = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    x = 5 * C + C - 3
    pos[-1] = x
    sl = [(x - i) % C for i in range(1, 50)]
    past = [draw((49, H_kv, d), i, "bf16") for i in (1, 2)]
    for t, s in zip((K, V), past):
        t[-1, sl] = s
    q, k, v = draw((B, H, d), 3, "bf16"), draw((B, H_kv, d), 4, "bf16"), draw((B, H_kv, d), 5, "bf16")
    o = api.lawcat_attn_decode(p, q, k, v, K, V, pos)
    rows = [torch.cat([new[-1][None], s]) for new, s in zip((k, v), past)]
    ref = attention(q[-1][None, None], rows[0][None], rows[1][None], torch.ones(1, 1, 50, dtype=torch.bool), float(torch.tensor(d ** -0.5)))
    check(o[-1][None, None], ref["o"], ref["o_sum"] + U16 * ref["o_mag"], U16, "o")
    assert torch.equal(K[-1, x % C], k[-1]) and torch.equal(V[-1, x % C], v[-1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("T,C,start", [(1, 1, 0), (7, 100, 0), (50, 100, 80), (100, 100, 3), (257, 100, 5)])
def test_quantize_and_back(T, C, start, d, dtype):
    B, H_kv = 3, 2
    k, v = draw((B, T, H_kv, d), 1, dtype), draw((B, T, H_kv, d), 2, dtype)
    k[:, ::3, :, ::7] *= 40
    v[0, 0] = 1.25                                   # (a group of one value: no scale)
    v[1, T // 2] = torch.linspace(-7.5, 7.5, d).to(v.dtype)  # (quotients on the borders between codes)
    p = api.attn_params(B, T, H_kv, H_kv, d, T_k=C, dtype=dtype)
    cache = api.quant_cache(p)
    for t in cache:
        t.view(torch.uint8).fill_(0xAB)
    before = [t.clone() for t in cache]
    pos = torch.tensor([start, start + 2 * C + 1, -1], dtype=torch.int32, device="cuda")
    api.lawcat_cache_quantize(p, k, v, pos, *cache)
    keep = min(T, C)
    for b in range(2):
        slots = (int(pos[b]) + torch.arange(T - keep, T, device="cuda")) % C
        for x, q, pr in ((k, 0, 1), (v, 2, 3)):
            code, scale, low, _ = quantized(x[b, T - keep:])
            got = cache[q][b][:, slots].transpose(0, 1)
            want = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
            assert torch.equal(cache[pr][b][:, slots].transpose(0, 1).double(), torch.stack([scale, low], -1))
            if dtype == "bf16":
                assert torch.equal(got, want)
            else:   # (fp32 rows: a quotient within a step of fp32 of a border may fall on either side)
                assert float((got != want).double().mean()) < 1e-3
        rest = torch.ones(C, dtype=torch.bool, device="cuda")
        rest[slots] = False
        for t, was in zip(cache, before):
            assert torch.equal(t[b][:, rest].contiguous().view(torch.uint8), was[b][:, rest].contiguous().view(torch.uint8))
    for t, was in zip(cache, before):
        assert torch.equal(t[2].view(torch.uint8), was[2].view(torch.uint8))
    back = api.lawcat_cache_dequantize(p, *cache, pos)
    for n, i in (("k", 0), ("v", 1)):
        assert not back[n][2].any()
        for b in range(2):
            slots = (int(pos[b]) + torch.arange(T, device="cuda")) % C
            # (one fp32 rounding of minimum + code scale, then the storage type's)
            want = rows_of(cache, b, slots)[i].float().to(DT[dtype])
            assert torch.equal(back[n][b], want)


def test_quantize_values_that_are_not_finite():
    """Their group reads back as NaN, the row's other groups and the neighbours as ever."""
    d, T = 64, 4
    k, v = draw((1, T, 1, d), 1, "bf16"), draw((1, T, 1, d), 2, "bf16")
    k[0, 1, 0, 3], k[0, 2, 0, 40], v[0, 0, 0, 0] = math.nan, math.inf, -math.inf
    v[0, 3, 0, :2] = torch.tensor([3e38, -3e38], dtype=torch.bfloat16)
    p = api.attn_params(1, T, 1, 1, d, T_k=8)
    cache = api.quant_cache(p)
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.lawcat_cache_quantize(p, k, v, pos, *cache)
    back = api.lawcat_cache_dequantize(p, *cache, pos)
    for n, x in (("k", k), ("v", v)):
        bad = torch.zeros(1, T, 1, 2, dtype=torch.bool, device="cuda")
        for t, g in ([(1, 0), (2, 1)] if n == "k" else [(0, 0), (3, 0)]):
            bad[0, t, 0, g] = True
        bad = bad.repeat_interleave(32, -1)
        assert torch.isnan(back[n][bad]).all()
        assert torch.equal(back[n][~bad], quantized(x)[3].float().bfloat16()[~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("quant", [False, True])
def test_what_the_scratch_held_makes_no_difference(quant, dtype):
    """The same bits over scratch full of zeros and full of NaN, most parts of the slots without a key."""
    B, C, H, H_kv, d = 4, 9000, 8, 2, 64
    p = api.attn_params(B, 1, H, H_kv, d, T_k=C, dtype=dtype)
    q, k, v = draw((B, H, d), 1, dtype, 1.5), draw((B, H_kv, d), 2, dtype), draw((B, H_kv, d), 3, dtype)
    pos = torch.tensor([-1, 0, 700, 8999], dtype=torch.int32, device="cuda")
    pasts = [draw((B, C, H_kv, d), 4 + i, dtype) for i in range(2)]
    cache = api.quant_cache(p) if quant else tuple(pasts)
    if quant:
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C, dtype=dtype), *pasts, torch.zeros_like(pos), *cache)
    n = api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_DECODE)
    assert n > 0
    f = api.lawcat_attn_decode_quant if quant else api.lawcat_attn_decode
    got = [f(p, q, k, v, *[t.clone() for t in cache], pos, ws=torch.full((n,), fill, dtype=torch.uint8, device="cuda")) for fill in (0, 255)]
    assert torch.equal(*got) and not got[0][0].any() and torch.isfinite(got[0]).all()


@pytest.mark.parametrize("quant", [False, True])
def test_a_captured_step_is_replayed_at_every_length(quant):
    B, C, H, H_kv, d = 2, 700, 8, 2, 64
    p = api.attn_params(B, 1, H, H_kv, d, T_k=C, window=600)
    q, k, v = draw((B, H, d), 1, "bf16"), draw((B, H_kv, d), 2, "bf16"), draw((B, H_kv, d), 3, "bf16")
    pos = torch.tensor([0, 690], dtype=torch.int32, device="cuda")
    new = lambda: api.quant_cache(p) if quant else tuple(torch.zeros(B, C, H_kv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))  # noqa: E731
    f = api.lawcat_attn_decode_quant if quant else api.lawcat_attn_decode
    a, e = new(), new()
    f(p, q, k, v, *new(), pos.clone())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = f(p, q, k, v, *a, pos)
        pos += 1
    pe = torch.tensor([0, 690], dtype=torch.int32, device="cuda")
    for i in range(20):
        q.copy_(draw((B, H, d), 100 + i, "bf16"))
        k.copy_(draw((B, H_kv, d), 200 + i, "bf16"))
        g.replay()
        want = f(p, q, k, v, *e, pe)
        pe += 1
        assert torch.equal(o, want)
    for x, y in zip(a, e):
        assert torch.equal(x, y)
