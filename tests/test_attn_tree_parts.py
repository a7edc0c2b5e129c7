"""Attention of drafted tokens over 4 bits with 65 to 128 rows, whose tiles the unpacking warps share out in parts: no tile may pass a warp that has no
part of it (a barrier's phase bit, seen a use too late, is the wrong one: the waits run out, or a stage in use is written)."""
import pytest
import torch

from paper_2509_18467_b200 import api
from test_attn import draw
from test_attn_tree import some_tree, tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,H,H_kv,d", [(32, 16, 4, 128), (17, 8, 2, 128), (32, 16, 4, 64), (70, 2, 2, 64), (30, 24, 8, 128)])
@pytest.mark.parametrize("lengths", ["long", "cut", "many short", "mixed"])
def test_every_tile_is_followed(lengths, N, H, H_kv, d):
    """Twenty calls give the same bits, none of them runs out of time, and the last ones are right."""
    pos, C = {"long": ([6000 - 90 * b for b in range(24)], 6100), "cut": ([1500] * 37, 1600), "many short": ([b % 3 for b in range(600)], 500),
              "mixed": ([0 if b % 5 else 450 for b in range(600)], 500)}[lengths]
    B = len(pos)
    p = api.attn_params(B, N, H, H_kv, d, T_k=C)
    q, k, v = draw((B, N, H, d), 1, "bf16", 1.5), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    cache = api.quant_cache(p)
    api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), *[torch.randn(B, C, H_kv, d, device="cuda").bfloat16() for _ in range(2)],
                              torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    at = torch.tensor(pos, dtype=torch.int32, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    api.test_set_wait_limit(200_000_000)      # (0.1 s: none of these calls takes a hundredth of that)
    try:
        outs = [api.lawcat_attn_tree_quant(p, q, k, v, *cache, at, dev_status=status) for _ in range(20)]
        torch.cuda.synchronize()
    finally:
        api.test_set_wait_limit(0)
    assert status[0].item() == 0
    assert all(torch.equal(o, outs[0]) for o in outs[1:])
    few = range(0, B, max(1, B // 40))
    tree(True, [pos[b] for b in few], N, C, H=H, H_kv=H_kv, d=d, seed=N, parents=lambda b: some_tree(N, b))
