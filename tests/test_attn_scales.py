"""Softmax attention with scales that are zero or negative. With a negative scale the attention is that of -q with the scale's size:
the same o, lse, dk and dv, and dq with its sign turned (so that the 64-bit reference and its bounds are those of a positive scale).
With a scale of zero every key that is seen weighs the same (but for the biases) and no gradient flows into q and k."""
import math

import pytest
import torch

from attn_reference import U16, U32, attention, check, visible
from paper_2509_18467_b200 import api
from test_attn import KINDS, draw

pytestmark = pytest.mark.gpu

FORMS = [dict(), dict(cap=3.0), dict(slopes=True), dict(cap=20.0, slopes=True), dict(causal=0, cap=1.0), dict(window=70), dict(cu=[0, 90, 300]),
         dict(prefix=[129], slopes=True)]


@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.125, -1.5])
@pytest.mark.parametrize("kw", FORMS)
def test_forward_and_gradients(kw, scale, d, dtype, exact):
    T, H, H_kv = 300, 4, 2
    q, k, v, dO = [draw((1, T, h, d), 70 + i, dtype) for i, h in enumerate((H, H_kv, H_kv, H))]
    sl = torch.tensor([2.0 ** (-1 - h) for h in range(H)], device="cuda") if kw.get("slopes") else None
    causal, window, cap, cu, prefix = kw.get("causal", 1), kw.get("window", 0), kw.get("cap", 0.0), kw.get("cu"), kw.get("prefix")
    p = api.attn_params(1, T, H, H_kv, d, dtype=dtype, exact=exact, scale=scale, causal=causal, window=window, cap=cap)
    more = dict(slopes=sl, cu_seqlens=cu, prefix=prefix)
    r = api.lawcat_attn_fwd(p, q, k, v, **more)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, **more))
    ref = attention(-q if scale < 0 else q, k, v, visible(T, T, causal, window, cu, prefix), abs(scale), cap, sl, dO, r["o"])
    if scale < 0:
        ref["dq"] = -ref["dq"]
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    err = dict(ref["grad_err"](coarse, out), o=ref["o_sum"] + coarse * ref["o_mag"], lse=ref["lse_err"])
    for n in ("o", "lse", "dq", "dk", "dv"):
        check(r[n], ref[n], err[n], U32 if n == "lse" else out, n)
    if scale == 0:
        assert not r["dq"].any() and not r["dk"].any()


@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("scale", [0.0, -0.125])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (3.0, False), (0.0, True), (20.0, True)])
def test_decode(cap, slopes, scale, dtype, exact):
    B, C, H, H_kv, d = 3, 300, 8, 2, 64
    q, k, v = draw((B, H, d), 1, dtype), draw((B, H_kv, d), 2, dtype), draw((B, H_kv, d), 3, dtype)
    K, V = draw((B, C, H_kv, d), 4, dtype), draw((B, C, H_kv, d), 5, dtype)
    sl = torch.tensor([2.0 ** (-3 - h % 8) for h in range(H)], device="cuda") if slopes else None
    pos = [0, 200, 777]
    p = api.attn_params(B, 1, H, H_kv, d, T_k=C, dtype=dtype, exact=exact, scale=scale, cap=cap)
    o = api.lawcat_attn_decode(p, q, k, v, K, V, torch.tensor(pos, dtype=torch.int32, device="cuda"), slopes=sl)
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    for b, x in enumerate(pos):
        n = min(x + 1, C)
        at = torch.arange(x - n + 1, x + 1, device="cuda") % C
        ref = attention((-q if scale < 0 else q)[b][None, None], K[b][at][None], V[b][at][None], torch.ones(1, 1, n, dtype=torch.bool), abs(scale), cap, sl)
        check(o[b][None, None], ref["o"], ref["o_sum"] + coarse * ref["o_mag"], out, f"o of sequence {b}")


@pytest.mark.parametrize("dtype,exact", KINDS)
def test_a_scale_of_zero_is_the_mean(dtype, exact):
    """A plain mean of the value rows that are seen, and lse the logarithm of their number."""
    T, H, d = 150, 2, 64
    q, k, v = [draw((1, T, H, d), i, dtype) for i in range(3)]
    r = api.lawcat_attn_fwd(api.attn_params(1, T, H, H, d, dtype=dtype, exact=exact, scale=0.0), q, k, v)
    n = torch.arange(1, T + 1, device="cuda", dtype=torch.float64)[None, :, None]
    mean, mag = (x.double().cumsum(1) / n[..., None] for x in (v, v.abs()))
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    check(r["o"], mean, ((T + 32) * U32 + coarse) * mag, out, "o")
    check(r["lse"], n.log().expand(1, T, H), (T + 32) * U32 * torch.ones(1, T, H, dtype=torch.float64), 4 * U32, "lse")
    assert math.isclose(float(r["lse"][0, 0, 0]), 0.0, abs_tol=1e-6)
