"""Two checks of the attention gradients that the element-wise bounds do not make.

Where D = dO.o comes from. The stored o is rounded to the storage type, and the tensor-core kernels do not take D from it: the
queries' kernel sums D = sum_j p_j dP_j in fp32, corrects dq by (dO.o - D) sum_j p_j k_j at its end, and hands D to the keys' kernel.
The inputs here make that correction the whole of the gradient's error: every value row has the same sum over channels and dO is one, so
that all dP_j are equal, dx = p (dP - D) is zero and so are dq and dk; o lies 0.4 of a bf16 step above one in every channel and is
stored as one; keys and queries have a common offset, so that nothing else cancels it.

Against differences. Along directions that follow the sign of the 64-bit gradient (every element counts in the same sense), against
extrapolated differences of the loss, whose own error is estimated from the differences alone.
"""
import math

import pytest
import torch

from attn_reference import U16, U32, attention, check, visible
from paper_2509_18467_b200 import api
from test_attn import draw


def level_case(d, causal, device, T=200, H=4, H_kv=2):
    """Inputs whose dP is the same for every key; and what the kernels' roundings allow."""
    g = torch.Generator().manual_seed(d + causal)
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    q = (0.5 + 0.25 * rnd(1, T, H, d)).bfloat16()
    k = (2.0 + rnd(1, T, H_kv, d)).bfloat16()
    up = torch.rand(1, T, H_kv, d, generator=g).argsort(-1) < int(0.4 * d)   # 0.4 d channels of every row, one bf16 step up
    v = (1.0 + up.float() * 2.0 ** -7).bfloat16()
    return [x.to(device) for x in (q, k, v, torch.ones(1, T, H, d).bfloat16())]


def level_terms(q, k, v, dO, o, causal):
    """In 64 bits: ref (dq, dk), their bounds, and what kernels that took D from the stored o, or turned the correction's sign, would give.

    With D^ = sum p^ dP^ in fp32, off by e_D <= p_err sum p |dP| + (n + d + 16) 2^-24 sum p sum|dO||v|, and f = |dO.o - D| + e_D:
      dq = scale [sum bf16(p^ (dP - dO.o)) k + (dO.o - D^) sum bf16(p^) k]: two roundings to bf16 (2^-8 of p (|dP - D| + f) and of p f), the
        weights' relative error on p (dP - D), (d + 16) 2^-24 sum|dO||v| of dP and e_D on p, n + 16 steps of the fp32 sums; rounded once
      dk = scale sum bf16(p^ (dP - D^)) q, the same without the terms of f
    (2 % on top for products of these errors.)"""
    T, H, d = q.shape[1:]
    H_kv, scale = k.shape[2], d ** -0.5
    G = H // H_kv
    see = visible(T, T, causal, 0)
    r = attention(q, k, v, see, scale)
    q, dO, o = q.double(), dO.double(), o.double()
    k, v = (x.double().repeat_interleave(G, 2) for x in (k, v))
    x = torch.einsum("bthd,bshd->bhts", q, k) * scale
    p = torch.softmax(x.masked_fill(~see.to(q.device)[:, None], -math.inf), -1)
    dP, mag = torch.einsum("bthd,bshd->bhts", dO, v), torch.einsum("bthd,bshd->bhts", dO.abs(), v.abs())
    D, Do = ((p * dP).sum(-1, keepdim=True), torch.einsum("bthd,bthd->bht", dO, o)[..., None])
    n, p_err = see.sum(-1)[:, None, :, None].to(q.device).double(), r["p_err"]
    e_D = p_err * (p * dP.abs()).sum(-1, keepdim=True) + (n + d + 16) * U32 * (p * mag).sum(-1, keepdim=True)
    f, w = (Do - D).abs() + e_D, (dP - D).abs()
    both = lambda y, z: torch.einsum("bhts,bshd->bthd", y, z) * scale  # noqa: E731
    keys = lambda y, z: (torch.einsum("bhts,bthd->bshd", y, z) * scale).reshape(1, T, H_kv, G, d).sum(3)  # noqa: E731
    e = (p_err + U16) * w + (d + 16) * U32 * mag + e_D
    err = dict(dq=both(1.02 * p * (e + 2 * U16 * f + 2 * (n + 16) * U32 * (w + f)), k.abs()),
               dk=keys(1.02 * p * (e + G * (T + 16) * U32 * (w + e_D)), q.abs()))
    ref = dict(dq=both(p * (dP - D), k), dk=keys(p * (dP - D), q))
    stored = dict(dq=both(p * (dP - Do), k), dk=keys(p * (dP - Do), q))
    turned = dict(dq=both(p * (dP - 2 * Do + D), k), dk=keys(p * (dP + D - 2 * Do), q))
    return ref, err, stored, turned


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_the_bounds_see_where_D_comes_from(d, causal):
    """(On the CPU, with the mistakes made in the reference.) Gradients with D from the stored o, or with the correction's sign turned,
    are off by more than twice the bound in most elements: nothing within the bound of them is within the bound of the right ones."""
    x = level_case(d, causal, "cpu")
    o = attention(*x[:3], visible(200, 200, causal, 0), d ** -0.5)["o"].bfloat16()
    ref, err, stored, turned = level_terms(*x, o, causal)
    for wrong in (stored, turned):
        for n in ("dq", "dk"):
            over = ((wrong[n] - ref[n]).abs() / (err[n] + U16 * ref[n].abs())).flatten()
            assert float(over.median()) > 2, n
            with pytest.raises(AssertionError):
                check(wrong[n].bfloat16(), ref[n], err[n], U16, n)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_D_is_not_taken_from_the_rounded_output(d, causal):
    q, k, v, dO = level_case(d, causal, "cuda")
    T, H = q.shape[1:3]
    p = api.attn_params(1, T, H, k.shape[2], d, causal=causal)
    r = api.lawcat_attn_fwd(p, q, k, v)
    g = api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO)
    ref, err, _, _ = level_terms(q, k, v, dO, r["o"], causal)
    for n in ("dq", "dk"):
        check(g[n], ref[n], err[n], U16, n)


DIFF = [dict(), dict(causal=0), dict(cap=4.0, slopes=True), dict(window=9), dict(cu=[0, 11, 40])]


def along_the_gradient(dtype, kw, device):
    """Inputs, 64-bit results, directions, the loss's extrapolated difference quotient along each and that one's own error."""
    T, H, H_kv, d = 40, 4, 2, 64
    x = [draw((1, T, h, d), 21 + i, dtype, 1.5 if i == 0 else 1.0, device) for i, h in enumerate((H, H_kv, H_kv, H))]
    slopes = torch.tensor([2.0 ** (-1 - h) for h in range(H)], device=device) if kw.get("slopes") else None
    see, scale, cap = visible(T, T, kw.get("causal", 1), kw.get("window", 0), kw.get("cu")), float(torch.tensor(d ** -0.5)), kw.get("cap", 0.0)
    full = attention(*x[:3], see, scale, cap, slopes, x[3])
    out = []
    for n, i in (("dq", 0), ("dk", 1), ("dv", 2)):
        e = draw(full[n].shape, 30 + i, "f32", 1.0, device).double().abs() * full[n].sign()
        e /= e.abs().max()

        def loss(s):
            y = [t.double() + (s * e if j == i else 0.0) for j, t in enumerate(x[:3])]
            return float((attention(*y, see, scale, cap, slopes)["o"] * x[3].double()).sum())
        quot = lambda h: (loss(h) - loss(-h)) / (2 * h)  # noqa: E731
        c = [quot(2.0 ** -k) for k in (3, 4, 5, 6)]
        a = [(4 * c[j + 1] - c[j]) / 3 for j in range(3)]             # error h^4
        b = [(16 * a[j + 1] - a[j]) / 15 for j in range(2)]           # error h^6
        out.append((n, e, b[1], abs(b[1] - b[0])))
    return x, slopes, full, out


def tolerance(full, n, e, dtype):
    """What the kernels' element-wise bounds leave along a direction."""
    coarse, out = (U16, U16) if dtype == "bf16" else (0.0, U32)
    return float(((full["grad_err"](coarse, out)[n] + out * full[n].abs()) * e.abs()).sum())


@pytest.mark.parametrize("kw", DIFF)
@pytest.mark.parametrize("dtype,part", [("f32", 0.01), ("bf16", 0.2)])
def test_the_differences_see_a_wrong_gradient(dtype, part, kw):
    """(On the CPU.) The 64-bit gradients agree with the differences to what those are off themselves, and gradients that are off by one
    part in a hundred (in five with the tensor-core kernels' bounds) do not pass."""
    x, slopes, full, directions = along_the_gradient(dtype, kw, "cpu")
    for n, e, quot, off in directions:
        dot = float((full[n] * e).sum())
        assert off < 1e-6 * abs(quot) and abs(quot - dot) <= off + 1e-11 * abs(quot), (n, quot, dot, off)
        assert part * abs(dot) > 2 * tolerance(full, n, e, dtype) + off, n


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", DIFF)
def test_gradients_against_extrapolated_differences(kw, dtype):
    x, slopes, full, directions = along_the_gradient(dtype, kw, "cuda")
    q, k, v, dO = x
    T, H, d = q.shape[1:]
    p = api.attn_params(1, T, H, k.shape[2], d, dtype=dtype, causal=kw.get("causal", 1), window=kw.get("window", 0), cap=kw.get("cap", 0.0))
    more = dict(slopes=slopes, cu_seqlens=kw.get("cu"))
    r = api.lawcat_attn_fwd(p, q, k, v, **more)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, **more))
    for n, e, quot, off in directions:
        got = float((r[n].double() * e).sum())
        assert abs(quot - got) <= tolerance(full, n, e, dtype) + off, (n, quot, got, off)
