"""Attention of drafted tokens: what stands in shared memory before a call, and what nodes that are not there hold, changes no bit of the others' results."""
import pytest
import torch

from paper_2509_18467_b200 import api
from test_attn import draw
from test_attn_tree import some_tree

pytestmark = pytest.mark.gpu


def caches(quant, B, C, H_kv, d):
    K, V = draw((B, C, H_kv, d), 4, "bf16"), draw((B, C, H_kv, d), 5, "bf16")
    if not quant:
        return api.lawcat_attn_tree, (K, V)
    p = api.attn_params(B, C, H_kv, H_kv, d, T_k=C)
    cache = api.quant_cache(p)
    api.lawcat_cache_quantize(p, K, V, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    return api.lawcat_attn_tree_quant, cache


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [3, 5, 33, 100])
@pytest.mark.parametrize("kw", [dict(), dict(cap=10.0)])
def test_what_shared_memory_held(kw, G, d, quant):
    """The call in front fills the same places with queries of zero, or very large ones."""
    B, N, C, H_kv = 40, 45, 300, 2
    f, cache = caches(quant, B, C, H_kv, d)
    pos = torch.full((B,), 250, dtype=torch.int32, device="cuda")
    up = torch.tensor([some_tree(N, b) for b in range(B)], dtype=torch.int32, device="cuda")
    p, p4 = api.attn_params(B, N, G * H_kv, H_kv, d, T_k=C, **kw), api.attn_params(B, N, 4 * H_kv, H_kv, d, T_k=C, **kw)
    q, k, v = draw((B, N, G * H_kv, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    outs = []
    for size in (0.0, 1e4, 0.0, 300.0):
        f(p4, draw((B, N, 4 * H_kv, d), 7, "bf16", size), k, v, *cache, pos, parent=up)
        outs.append(f(p, q, k, v, *cache, pos, parent=up))
    assert all(torch.equal(o, outs[0]) for o in outs[1:])


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("N,G", [(10, 3), (10, 4), (45, 4), (45, 5)])
@pytest.mark.parametrize("kw", [dict(), dict(cap=10.0)])
def test_what_absent_nodes_hold(kw, N, G, quant):
    B, C, H_kv, d = 12, 300, 2, 64
    f, cache = caches(quant, B, C, H_kv, d)
    pos = torch.full((B,), 250, dtype=torch.int32, device="cuda")
    parents = [some_tree(N, b) for b in range(B)]
    for row in parents:
        row[N // 3], row[N - 2:] = N, [-2, N - 2]       # what hangs from them is not there either
    up = torch.tensor(parents, dtype=torch.int32, device="cuda")
    there = []
    for row in parents:
        ok = []
        for i, p in enumerate(row):
            ok.append(p == -1 or (0 <= p < i and ok[p]))
        there.append(ok)
    gone = ~torch.tensor(there, device="cuda")
    p = api.attn_params(B, N, G * H_kv, H_kv, d, T_k=C, **kw)
    q, k, v = draw((B, N, G * H_kv, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    outs = []
    for held in (0.0, 1e4, -300.0, float("nan"), float("inf")):
        for x in (q, k, v):
            x[gone] = held
        outs.append(f(p, q, k, v, *cache, pos, parent=up))
        assert not outs[-1][gone].any()
    assert all(torch.equal(o, outs[0]) for o in outs[1:])
