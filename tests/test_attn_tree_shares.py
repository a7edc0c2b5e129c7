"""Attention of drafted tokens whose work is shared out over the SMs: segments cut into pieces that meet in a second kernel, or in the block that has
their first; batches of very different lengths; rows that are not finite in cut segments; scratch that holds anything; waits that run out."""
import math

import pytest
import torch

from attn_reference import U16
from paper_2509_18467_b200 import api
from test_attn import draw
from test_attn_tree import some_tree, tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,H,H_kv", [(5, 8, 4), (11, 16, 4), (40, 16, 4), (70, 8, 2)])
@pytest.mark.parametrize("lengths", ["even", "one long", "ragged"])
def test_pieces(lengths, N, H, H_kv, d, quant):
    """Four segments or fewer per SM's block in straight shares, up to 35 pieces to a segment, or one block with many segments."""
    C = 4000
    pos = dict(even=[1500] * 24, ragged=[(b * 977) % 4100 for b in range(36)])
    pos["one long"] = [3990] + [3] * 47
    tree(quant, pos[lengths], N, C, H=H, H_kv=H_kv, d=d, seed=N + d, parents=lambda b: some_tree(N, b))


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("B", [1, 2, 8, 31, 32, 33, 90])
def test_numbers_of_sequences(B, quant):
    """Shares that end with segments (few sequences), straight ones, and more sequences than a warp has lanes; with biases, caps and windows."""
    pos = [(b * 389 + 700) % 2900 if b % 7 != 3 else -1 for b in range(B)]
    tree(quant, pos, 9, 2500, H=4, H_kv=2, d=64, seed=B, parents=lambda b: some_tree(9, b), slopes=True, cap=15.0, window=2000)


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("B", [3, 40])
def test_rows_that_are_not_finite_in_cut_segments(B, quant):
    """Cached tokens that are not finite, in the first, a middle and the last piece; what does not see them stays as it was."""
    N, C, H, H_kv, d, window = 6, 3000, 8, 2, 64, 1800
    q = draw((B, N, H, d), 1, "bf16", 1.5)
    k, v = draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    K, V = draw((B, C, H_kv, d), 4, "bf16"), draw((B, C, H_kv, d), 5, "bf16")
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, window=window)
    pos = torch.full((B,), 2800, dtype=torch.int32, device="cuda")

    def run(K, V):
        if not quant:
            return api.lawcat_attn_tree(p, q, k, v, K, V, pos)
        cache = api.quant_cache(p)
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), K, V, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
        return api.lawcat_attn_tree_quant(p, q, k, v, *cache, pos)

    clean = run(K, V)
    for back in (1, 900, window - 3):     # the last one is seen by nodes 0, 1 and 2 of the chain alone
        bad = V.clone()
        bad[1, 2800 - back, 0] = math.nan
        got = run(K, bad)
        hit = torch.zeros(B, N, H, dtype=torch.bool, device="cuda")
        hit[1, :3 if back > 1000 else N, :H // H_kv] = True
        assert torch.isnan(got[hit]).all()
        rest = got[1, :, :H // H_kv][~hit[1, :, :H // H_kv]]
        want = clean[1, :, :H // H_kv][~hit[1, :, :H // H_kv]]
        assert ((rest.float() - want.float()).abs() <= 2 * U16 * (1 + want.float().abs())).all()
        other = torch.ones(B, N, H, dtype=torch.bool, device="cuda")
        other[1, :, :H // H_kv] = False
        assert torch.equal(got[other], clean[other])


@pytest.mark.parametrize("quant", [False, True])
def test_scratch_that_holds_anything_and_replays(quant):
    """Straight shares: what a call finds in its scratch, its own numbers of an earlier replay among it, does not matter."""
    B, N, C, H, H_kv, d = 24, 12, 2000, 16, 4, 128
    p = api.attn_params(B, N, H, H_kv, d, T_k=C)
    q, k, v = draw((B, N, H, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    pasts = [draw((B, C, H_kv, d), 4 + i, "bf16") for i in range(2)]
    f, cache = api.lawcat_attn_tree, pasts
    if quant:
        cache, f = api.quant_cache(p), api.lawcat_attn_tree_quant
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), *pasts, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    pos = torch.tensor([(b * 531) % 2400 for b in range(B)], dtype=torch.int32, device="cuda")
    import ctypes
    ws = torch.empty(int(api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_TREE)), dtype=torch.uint8, device="cuda")
    want = f(p, q, k, v, *cache, pos, ws=ws)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = f(p, q, k, v, *cache, pos, ws=ws)
        graphs.append((g, out))
    for fill in (0, 255, 0x7f, None, None):
        if fill is not None:
            ws.fill_(fill)
        for g, out in graphs:
            g.replay()
            assert torch.equal(out, want)
    for i in range(20):                   # other lengths, then the first again
        pos.copy_(torch.tensor([(b * 531 + 97 * i) % 2400 for b in range(B)]))
        for g, out in graphs:
            g.replay()
        assert torch.equal(graphs[0][1], graphs[1][1])
        assert torch.equal(graphs[0][1], f(p, q, k, v, *cache, pos))


@pytest.mark.parametrize("quant,N", [(False, 12), (False, 60), (True, 4), (True, 60)])
def test_a_wait_that_runs_out(quant, N):
    B, C, H, H_kv, d = 24, 8000, 16, 4, 64
    p = api.attn_params(B, N, H, H_kv, d, T_k=C)
    q, k, v = draw((B, N, H, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    pasts = [draw((B, C, H_kv, d), 4 + i, "bf16") for i in range(2)]
    f, cache = api.lawcat_attn_tree, pasts
    if quant:
        cache, f = api.quant_cache(p), api.lawcat_attn_tree_quant
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), *pasts, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    pos = torch.full((B,), 7000, dtype=torch.int32, device="cuda")
    want = f(p, q, k, v, *cache, pos)
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    api.test_set_wait_limit(1)
    try:
        f(p, q, k, v, *cache, pos, dev_status=st)
        torch.cuda.synchronize()
    finally:
        api.test_set_wait_limit(0)
    assert st[0].item() == 5                                  # LAWCAT_ERR_TIMEOUT
    assert torch.equal(f(p, q, k, v, *cache, pos), want)      # the context and the next call are whole
