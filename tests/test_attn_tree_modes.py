"""Attention of drafted tokens where the lengths on the device decide how its work is shared out: whole segments while they are short, cut ones where
they are long, both in one captured call; and rows that are not finite where long segments are cut."""
import ctypes
import math

import pytest
import torch

from attn_reference import U16
from paper_2509_18467_b200 import api
from test_attn import draw
from test_attn_tree import some_tree, tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("N,H,H_kv,d", [(3, 8, 2, 64), (7, 16, 2, 128), (33, 8, 2, 128), (70, 8, 2, 64)])
@pytest.mark.parametrize("B", [17, 40])
def test_short_and_long(B, N, H, H_kv, d, quant):
    """All sequences as long as one another, then one of them a hundred tiles longer, then none there."""
    C = 7000
    for pos in ([90] * B, [700] * B, [5200] * B, [90] * (B - 1) + [6900], [6900] + [0] * (B - 1), [-1] * B):
        tree(quant, pos, N, C, H=H, H_kv=H_kv, d=d, seed=N + d, parents=lambda b: some_tree(N, b))


@pytest.mark.parametrize("N,quant", [(6, False), (20, False), (6, True), (20, True)])
def test_rows_that_are_not_finite(N, quant):
    """As in test_attn_tree_shares.py, over a window that is long enough for the segments to be cut."""
    B, C, H, H_kv, d, window = 40, 9000, 8, 2, 64, 7000
    q = draw((B, N, H, d), 1, "bf16", 1.5)
    k, v = draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    K, V = draw((B, C, H_kv, d), 4, "bf16"), draw((B, C, H_kv, d), 5, "bf16")
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, window=window)
    at = 8000
    pos = torch.full((B,), at, dtype=torch.int32, device="cuda")

    def run(K, V):
        if not quant:
            return api.lawcat_attn_tree(p, q, k, v, K, V, pos)
        cache = api.quant_cache(p)
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), K, V, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
        return api.lawcat_attn_tree_quant(p, q, k, v, *cache, pos)

    clean = run(K, V)
    for back in (1, 3500, window - 3):     # the last one is seen by nodes 0, 1 and 2 of the chain alone
        bad = V.clone()
        bad[1, at - back, 0] = math.nan
        got = run(K, bad)
        hit = torch.zeros(B, N, H, dtype=torch.bool, device="cuda")
        hit[1, :3 if back > 5000 else N, :H // H_kv] = True
        assert torch.isnan(got[hit]).all()
        rest = got[1, :, :H // H_kv][~hit[1, :, :H // H_kv]]
        want = clean[1, :, :H // H_kv][~hit[1, :, :H // H_kv]]
        assert ((rest.float() - want.float()).abs() <= 2 * U16 * (1 + want.float().abs())).all()
        other = torch.ones(B, N, H, dtype=torch.bool, device="cuda")
        other[1, :, :H // H_kv] = False
        assert torch.equal(got[other], clean[other])


@pytest.mark.parametrize("N", [4, 12, 40])
@pytest.mark.parametrize("quant", [False, True])
def test_replays_at_every_length(quant, N):
    """One captured call, and another that shares its scratch, while sequences grow and shrink."""
    B, C, H, H_kv, d = 36, 6000, 8, 2, 128
    p = api.attn_params(B, N, H, H_kv, d, T_k=C)
    q, k, v = draw((B, N, H, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    pasts = [draw((B, C, H_kv, d), 4 + i, "bf16") for i in range(2)]
    f, cache = api.lawcat_attn_tree, pasts
    if quant:
        cache, f = api.quant_cache(p), api.lawcat_attn_tree_quant
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), *pasts, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(int(api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_TREE)), dtype=torch.uint8, device="cuda")
    f(p, q, k, v, *cache, pos, ws=ws)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = f(p, q, k, v, *cache, pos, ws=ws)
        graphs.append((g, out))
    ws.fill_(255)
    for at in (5, 200, 5900, 40, 3000, 9000, 0, 5999, 64, 1000):
        for skew in (0, 1):
            pos.copy_(torch.tensor([at if skew == 0 or b % 9 else (at * 7 + 13 * b) % 6100 for b in range(B)]))
            for g, out in graphs:
                g.replay()
            want = f(p, q, k, v, *cache, pos)
            for g, out in graphs:
                assert torch.equal(out, want)
