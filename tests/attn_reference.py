"""Softmax attention, its gradients and the 4-bit cache in 64 bits, from the definitions, and how far a kernel may be from them.

Tolerances are worst cases, counted from the roundings that a kernel makes (half a step is eps / 2 of the type: bf16 2^-8,
fp32 2^-24), per element:
  score          a dot product of d terms and a handful of operations behind it: (d + 16) 2^-24 (scale sum|q||k| + slope |i-j|)
                 absolutely; a weight is off by that much relatively, and so is the row's sum (twice), plus n + 16 steps of 2^-24
  o              that times sum_j p_j |v_j|; tensor-core kernels round p to bf16 (2^-8 of the same sum); the result is rounded once
  dv             the same with dO instead of v
  dx             p (dP - D): p's error, (d + 16) 2^-24 sum|dO||v| for dP, and D = dO.o from the stored o, which is rounded once;
                 tensor-core kernels round dx to bf16
  dq, dk         sums of dx k and dx q with those errors, rounded once
"""
import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8


def visible(T, T_k, causal, window, cu=None, prefix=None, B=1):
    """[B, T, T_k] truth values."""
    i = torch.arange(T)[:, None] + T_k - T
    j = torch.arange(T_k)[None, :]
    see = torch.ones(T, T_k, dtype=torch.bool)
    if causal:
        see &= j <= i
    if window:
        see &= (i - j).abs() < window
    see = see.expand(B, T, T_k).clone()
    if cu is not None:
        doc = torch.repeat_interleave(torch.arange(len(cu) - 1), torch.tensor(cu).diff())
        same = doc[:, None] == doc[None, :]
        if prefix is not None:
            first = torch.tensor(cu)[:-1][doc]
            see |= (j - first[:, None] < torch.tensor(prefix)[doc][:, None])[None]
        see &= same[None]
    elif prefix is not None:
        see |= j[None] < torch.tensor(prefix)[:, None, None]
    return see


def attention(q, k, v, see, scale, cap=0.0, slopes=None, dO=None, stored_o=None):
    """64-bit results and the ingredients of the bounds. q [B,T,H,d], k, v [B,T_k,H_kv,d], see [B,T,T_k]."""
    B, T, H, d = q.shape
    T_k, H_kv = k.shape[1], k.shape[2]
    G = H // H_kv
    q, k, v = q.double(), k.double().repeat_interleave(G, 2), v.double().repeat_interleave(G, 2)
    see = see.to(q.device)[:, None]
    u = torch.einsum("bthd,bshd->bhts", q, k) * scale
    th = torch.tanh(u / cap) if cap else torch.zeros_like(u)
    x = cap * th if cap else u
    dist = (torch.arange(T)[:, None] + T_k - T - torch.arange(T_k)[None, :]).abs().double().to(q.device)
    bias = torch.zeros(H, 1, 1, dtype=torch.float64, device=q.device) if slopes is None else slopes.double().reshape(H, 1, 1)
    x = x - bias * dist
    x = x.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, -1) if T_k else torch.full((B, H, T), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(x - lse.clamp_min(-1e300)[..., None]).masked_fill(~see, 0.0)
    r = dict(o=torch.einsum("bhts,bshd->bthd", p, v), lse=lse.transpose(1, 2))
    # what the scores may be off by, per row (the largest over its visible keys)
    # (1 + th^2 ... the tanh itself adds at most a few steps of cap)
    dx_abs = (d + 16) * U32 * (scale * torch.einsum("bthd,bshd->bhts", q.abs(), k.abs()) + bias.abs() * dist + (cap if cap else 0.0))
    row = dx_abs.masked_fill(~see, 0.0).amax(-1, keepdim=True) if T_k else torch.zeros(B, H, T, 1, dtype=torch.float64, device=q.device)
    n = see.sum(-1, keepdim=True).double()
    r["p_err"] = 2 * row + (n + 16) * U32                      # relative error of a weight
    r["lse_err"] = (row[..., 0] + (n[..., 0] + 16) * U32).transpose(1, 2) + 4 * U32 * r["lse"].abs().nan_to_num(0, 0, 0)
    r["o_mag"] = torch.einsum("bhts,bshd->bthd", p, v.abs())
    r["o_sum"] = torch.einsum("bhts,bshd->bthd", p * r["p_err"], v.abs())
    if dO is None:
        return r
    dO = dO.double()
    so = r["o"] if stored_o is None else stored_o
    D = torch.einsum("bthd,bthd->bht", dO, r["o"])[..., None]
    dP = torch.einsum("bthd,bshd->bhts", dO, v)
    dx = p * (dP - D) * (1 - th * th)
    heads = lambda y: y.reshape(B, T_k, H_kv, G, d).sum(3)  # noqa: E731
    r["dq"] = torch.einsum("bhts,bshd->bthd", dx, k) * scale
    r["dk"] = heads(torch.einsum("bhts,bthd->bshd", dx, q)) * scale
    r["dv"] = heads(torch.einsum("bhts,bthd->bshd", p, dO))
    D_err = torch.einsum("bthd,bthd->bht", dO.abs(), so.double().abs())[..., None]
    dP_mag = torch.einsum("bthd,bshd->bhts", dO.abs(), v.abs())

    def grads(eps_p, eps_o):
        e = dx.abs() * (r["p_err"] + eps_p) + p * ((d + 16) * U32 * dP_mag + (eps_o + (d + 16) * U32) * D_err)
        if cap:  # 1 - th^2 is off by 2 |th| times what th is off by
            e = e + p * (dP - D).abs() * 2 * (dx_abs / cap + 4 * U32)
        nq = (T + 16) * U32
        return dict(dq=scale * torch.einsum("bhts,bshd->bthd", e + dx.abs() * r["p_err"], k.abs()),
                    dk=scale * heads(torch.einsum("bhts,bthd->bshd", e + nq * G * dx.abs(), q.abs())),
                    dv=heads(torch.einsum("bhts,bthd->bshd", p * (r["p_err"] + eps_p + nq * G), dO.abs())))
    r["grad_err"] = grads
    return r


def check(got, want, err, out_eps, what, tiny=1e-37):
    """|got - want| <= err + out_eps |want| + tiny, element by element (out_eps: the result's own rounding; tiny: what is lost below
    fp32's least normal number)."""
    got, want = got.double(), want.to(got.device)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fin = torch.isfinite(want)
    assert torch.equal(got[~fin], want[~fin]), f"{what}: {int((got[~fin] != want[~fin]).sum())} values that are not finite differ"
    if not fin.any():
        return
    tol = (err.to(got.device).expand_as(want) + out_eps * want.abs() * 1.0001 + tiny)[fin]
    over = (got - want)[fin].abs() / tol
    assert torch.isfinite(got[fin]).all(), f"{what}: values that are not finite"
    assert float(over.max()) <= 1.0, f"{what}: {float(over.max()):.3g} times the tolerance"


def quantized(x):
    """codes [..., d], scale and minimum [..., groups] of the 4-bit cache, values [..., d]; all in 64 bits."""
    d = x.shape[-1]
    g = x.double().reshape(*x.shape[:-1], -1, min(32, d))
    low = g.amin(-1, keepdim=True).bfloat16().double()
    scale = ((g.amax(-1, keepdim=True) - low) / 15).bfloat16().double()
    code = torch.where(scale > 0, torch.round((g - low) / torch.where(scale > 0, scale, 1.0)).clamp(0, 15), 0.0)
    return code.reshape(x.shape), scale[..., 0], low[..., 0], (low + code * scale).reshape(x.shape)
