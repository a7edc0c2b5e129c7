"""Attention of drafted tokens: rows that are computed again by themselves, at every width, with caps, biases and scales, whole and cut segments: a cached value that
is not finite is seen by the least deep nodes alone, and the others' results are what they are without it. In a whole segment all of its rows are computed
again, in fp32 but for the stored rounding; of a cut one those whose piece it lies in (a row that sees nothing else of that piece leaves it out, and keeps
what the tensor cores have), so that the tensor cores' bound holds there. And caps and values at the ends of their ranges."""
import math

import pytest
import torch

from attn_reference import U16, U32, check, quantized
from paper_2509_18467_b200 import api
from test_attn import draw
from test_attn_decode import rows_of
from test_attn_tree import KINDS, some_tree, tree
from test_attn_tree_range import MIN_P, verify
from tree_reference import U11, sees, tree_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("pos,window", [([80, 300], 60), ([2900], 2600), ([1900] * 20, 1500)])
@pytest.mark.parametrize("N,kw", [(11, {}), (11, dict(cap=8.0, slopes=True)), (11, dict(scale=-0.2, cap=20.0)), (37, dict(slopes=True)), (37, dict(cap=5.0))])
def test_rows_that_do_not_see_it(N, kw, pos, window, d, quant, dtype, exact):
    B, H, H_kv = len(pos), 8, 2
    C = max(pos) + 100
    q, k, v = draw((B, N, H, d), N, dtype, 1.5), draw((B, N, H_kv, d), N + 1, dtype), draw((B, N, H_kv, d), N + 2, dtype)
    K, V = draw((B, C, H_kv, d), N + 3, dtype), draw((B, C, H_kv, d), N + 4, dtype)
    parents = [some_tree(N, b) for b in range(B)]
    scale = kw.get("scale")
    sl = torch.tensor([2.0 ** (-3 - h % 8) for h in range(H)], device="cuda") if kw.get("slopes") else None
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, dtype=dtype, exact=exact, window=window, cap=kw.get("cap", 0.0), scale=scale)
    bad = [x - window + 2 for x in pos]                 # window - 2 behind: nodes of depth 0 and 1 see it
    if quant:
        cache = api.quant_cache(p)
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C, dtype=dtype), K, V, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
        for b in range(B):
            cache[3][b, :, bad[b], 0, 1] = math.nan
        f = api.lawcat_attn_tree_quant
    else:
        for b in range(B):
            V[b, bad[b], :, 3] = math.nan
        cache, f = (K, V), api.lawcat_attn_tree
    o = f(p, q, k, v, *cache, torch.tensor(pos, dtype=torch.int32, device="cuda"), parent=torch.tensor(parents, dtype=torch.int32, device="cuda"), slopes=sl)
    for b, x in enumerate(pos):
        cached, see, dist = sees(parents[b], x, C, window)
        slots = torch.tensor(cached, device="cuda") % C
        if quant:
            Kd, Vd = rows_of(cache, b, slots)
            kn, vn = quantized(k[b])[3], quantized(v[b])[3]
        else:
            Kd, Vd, kn, vn = cache[0][b][slots].double(), cache[1][b][slots].double(), k[b].double(), v[b].double()
        Vd[cached.index(bad[b])] = 0.0
        hit = see[:, cached.index(bad[b])]
        assert hit.any() and not hit.all()
        got = o[b].float()
        seen = got[hit.to(o.device)]                    # channels of a group, or the one channel
        assert torch.isnan(seen[..., :min(d, 32)] if quant else seen[..., 3]).all()
        coarse = dtype == "bf16" and not exact and d >= 64 and window > 64
        eps = dict(eps_p=U11, eps_k=U11, eps_v=U11, min_p=MIN_P) if coarse and quant else dict(eps_p=U16) if coarse else {}
        s = float(torch.tensor(d ** -0.5 if scale is None else scale))
        want, err = tree_attention(q[b], torch.cat([Kd, kn]), torch.cat([Vd, vn]), see, dist, s, kw.get("cap", 0.0), sl, **eps)
        ok = (~hit).to(o.device)
        check(o[b][ok], want[ok], err[ok], U16 if dtype == "bf16" else U32, f"o of sequence {b}")


@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("N", [5, 40])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_caps_far_above_the_scores(d, N, quant, dtype, exact):
    """A cap of 1e6 is none: its own size must not be in the scores' rounding."""
    tree(quant, [0, 70, 700], N, 800, d=d, H=8, H_kv=2, dtype=dtype, exact=exact, cap=1e6, ref_cap=0.0, seed=d, parents=lambda b: some_tree(N, b))


@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("N", [5, 40])
@pytest.mark.parametrize("factor", [1e-12, 1e-3, 500.0, 1e5, 1e18])
def test_sizes_of_values(factor, N, quant, dtype, exact):
    """Values of any size, in some cached rows, in all of them, in the nodes' alone."""
    pos, C, H, H_kv, d = [70, 700], 800, 8, 2, 64
    parents = [some_tree(N, b) for b in range(2)]

    def some(k, v, K, V):
        V[:, ::5] *= factor

    def all_cached(k, v, K, V):
        V.mul_(factor)

    def nodes(k, v, K, V):
        v.mul_(factor)

    for i, mend in enumerate((some, all_cached, nodes)):
        if quant and dtype == "bf16" and not exact:
            q, k, v = draw((2, N, H, d), i, dtype, 1.5), draw((2, N, H_kv, d), i + 1, dtype), draw((2, N, H_kv, d), i + 2, dtype)
            K, V = draw((2, C, H_kv, d), i + 3, dtype), draw((2, C, H_kv, d), i + 4, dtype)
            mend(k, v, K, V)
            verify(q, k, v, K, V, pos, parents)
        else:
            tree(quant, pos, N, C, H=H, H_kv=H_kv, d=d, dtype=dtype, exact=exact, seed=i, parents=parents.__getitem__, mend=mend)
