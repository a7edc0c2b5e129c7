"""Attention of drafted tokens whose rows are computed again (a value is not finite): the other roles of a block wait for that, as long as the rows that are
computed take, not as long as one step of a tile."""
import math

import pytest
import torch

from paper_2509_18467_b200 import api
from test_attn import draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quant,N", [(False, 12), (False, 60), (True, 30), (True, 60)])
@pytest.mark.parametrize("short", [0, 1])
def test_rows_computed_again_are_waited_for(short, quant, N):
    """Two segments to a block, or long ones and short ones in turn; those of some long sequences hold a NaN each, and a wait may take a fraction of the
    time that its rows take (a long segment has 250 tiles, for which a wait is four times as long)."""
    B, C, H, H_kv, d, long = (148, 16384, 16, 4, 64, 16000) if short else (74, 16384, 16, 4, 64, 16000)
    p = api.attn_params(B, N, H, H_kv, d, T_k=C)
    q, k, v = draw((B, N, H, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    K, V = [torch.randn(B, C, H_kv, d, device="cuda").bfloat16() for _ in range(2)]
    at = [100 if short and b % 2 else long for b in range(B)]
    hit = [b for b in range(B) if (b % 6 == 0 if short else b == 1)]
    f, cache = api.lawcat_attn_tree, (K, V)
    if quant:
        f, cache = api.lawcat_attn_tree_quant, api.quant_cache(p)
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), K, V, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    pos = torch.tensor(at, dtype=torch.int32, device="cuda")
    clean = f(p, q, k, v, *cache, pos)
    for b in hit:
        if quant:
            cache[3][b, :, 50] = math.nan
        else:
            cache[1][b, 50] = math.nan
    status = torch.zeros(4, dtype=torch.int32, device="cuda")

    def call():
        t = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        t[0].record()
        o = f(p, q, k, v, *cache, pos, dev_status=status)
        t[1].record()
        torch.cuda.synchronize()
        return o, t[0].elapsed_time(t[1])

    _, ms = call()
    assert status[0].item() == 0
    api.test_set_wait_limit(int(ms * 1.9e6 / (4 if short else 2)))
    try:
        o, _ = call()
    finally:
        api.test_set_wait_limit(0)
    assert status[0].item() == 0
    assert torch.isnan(o[hit]).all()
    others = [b for b in range(B) if b not in hit]
    assert torch.equal(o[others], clean[others])
