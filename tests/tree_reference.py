"""Attention of drafted tokens over a cache in 64 bits, from the definitions, and how far a kernel may be from it.

Tolerances as in attn_reference.py: a score is off by (d + 16) 2^-24 (scale sum|q||k| + slope distance + cap), a weight by twice that relatively
plus n + 16 steps of 2^-24; operands that a kernel rounds add half a step each: weights eps_p, keys eps_k (to the score), values eps_v.
Weights in fp16 are whole multiples of 2^-24 below 2^-14 (min_p = 2^-25, half of that): the weights are relative to a score of the row, so that
their sum is at least 1, and sum_j p_j v_j / sum_j p_j is off by min_p sum_j |v_j| over the keys that are seen. (A weight of 2e-11 beside one
of 1, whose value is 0: the result is 1.1e-11 by the definition and 0 with weights in fp16, which is 6.67 times the bound without this term.)
"""
import math

import torch

from attn_reference import U16, U32

U11 = 2.0 ** -11   # half a step of fp16


def paths_of(parent):
    """Lists of nodes from the root to each node; empty where a node is not there."""
    out = []
    for i, p in enumerate(parent):
        out.append([i] if p == -1 else out[p] + [i] if 0 <= p < i and out[p] else [])
    return out


def sees(parent, pos, C, window):
    """(cached positions, see [N, cached + N], distances [N, cached + N]) of one sequence."""
    W = window or C
    paths = paths_of(parent)
    first = pos - max(0, min(pos, W - 1))
    cached = list(range(first, max(pos, 0)))
    N, n = len(parent), len(cached)
    see, dist = torch.zeros(N, n + N, dtype=torch.bool), torch.zeros(N, n + N, dtype=torch.float64)
    if pos >= 0:
        for i, path in enumerate(paths):
            if not path:
                continue
            depth = len(path) - 1
            dist[i, :n] = pos + depth - torch.tensor(cached, dtype=torch.float64)
            see[i, :n] = dist[i, :n] < W
            for e, j in enumerate(path):
                dist[i, n + j] = depth - e
                see[i, n + j] = depth - e < W
    return cached, see, dist


def tree_attention(q, k, v, see, dist, scale, cap=0.0, slopes=None, eps_p=0.0, eps_k=0.0, eps_v=0.0, min_p=0.0):
    """q [N, H, d], k, v [n, H_kv, d] in any type; o [N, H, d] and its error bound but for the result's own rounding, in 64 bits."""
    N, H, d = q.shape
    G = H // k.shape[1]
    dev = q.device
    k, v = (torch.where(see.any(0).to(dev)[:, None, None], x.double(), 0.0).repeat_interleave(G, 1) for x in (k, v))   # (rows that no node sees)
    q = torch.where(see.any(1).to(dev)[:, None, None], q.double(), 0.0)
    see, dist = see.to(dev)[None], dist.to(dev)[None]
    u = torch.einsum("thd,shd->hts", q, k) * scale
    x = cap * torch.tanh(u / cap) if cap else u
    bias = torch.zeros(H, 1, 1, dtype=torch.float64, device=dev) if slopes is None else slopes.double().reshape(H, 1, 1)
    x = (x - bias * dist).masked_fill(~see, -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-1e300)
    p = torch.exp(x - top).masked_fill(~see, 0.0)
    p = p / p.sum(-1, keepdim=True).clamp_min(1e-300)
    mag = abs(scale) * torch.einsum("thd,shd->hts", q.abs(), k.abs())
    err = (d + 16) * U32 * (mag + bias.abs() * dist + cap) + eps_k * mag
    row = err.masked_fill(~see, 0.0).amax(-1, keepdim=True)
    p_err = 2 * row + (see.sum(-1, keepdim=True) + 16) * U32
    o = torch.einsum("hts,shd->thd", p, v)
    bound = torch.einsum("hts,shd->thd", p * (p_err + eps_p + eps_v), v.abs())
    return o, bound + min_p * torch.einsum("hts,shd->thd", see.double().expand_as(p), v.abs())


__all__ = ["U11", "U16", "U32", "paths_of", "sees", "tree_attention"]
