"""How many parts a row block's keys are shared out into by the exact attention kernels (as the scratch that they ask for shows)."""
import ctypes

import pytest
import torch

from paper_2509_18467_b200 import api

up = lambda x, a: (x + a - 1) // a  # noqa: E731


@pytest.mark.gpu
@pytest.mark.parametrize("B,T,T_k,H", [(2, 1057, 1057, 4), (1, 100, 1200, 16), (1, 1500, 1500, 4), (1, 554, 554, 4), (1, 700, 1400, 20), (3, 200, 900, 9)])
def test_whole_rounds_of_the_blocks_that_an_SM_holds(B, T, T_k, H):
    """At width 128 a block of the fp32 forward holds 64 rows of queries and a tile of 64 keys and of 64 values, 132 words each, and
    64 x 68 weights: 118784 bytes, so that an SM has room for one. Without a mask (or with all keys in the past) all blocks are alike: of
    the least number of parts that gives each SM two blocks (four where there are blocks for every SM) up to twice as many, the one whose
    rounds over the SMs' places, each a part long, end first by 5 %."""
    p = api.attn_params(B, T, H, H, 128, T_k=T_k, dtype="f32", causal=0)
    rows = B * T * H
    blocks, most, sms = up(T, 64) * B * H, min(up(T_k, 64), 16), torch.cuda.get_device_properties(0).multi_processor_count
    assert 2 * 118784 > 232448 and blocks < 4 * sms
    best = least = min(up((2 if blocks < sms else 4) * sms, blocks), most)
    for n in range(least + 1, min(2 * least, most) + 1):
        if up(blocks * n, sms) * best * 100 < up(blocks * best, sms) * n * 95:
            best = n
    want = up(8 * B * T, 256) * 256 + up(4 * best * rows * 128, 256) * 256 + up(8 * best * rows, 256) * 256
    assert api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_FWD) == want, (least, best)


@pytest.mark.gpu
@pytest.mark.parametrize("H,H_kv,d,heads,resident", [(32, 8, 64, 4, 4), (64, 8, 64, 8, 4), (32, 8, 128, 4, 4), (64, 8, 128, 8, 3), (8, 1, 128, 8, 3)])
@pytest.mark.parametrize("B,C", [(1, 32768), (16, 16384), (64, 16384), (64, 3000)])
def test_parts_of_a_step_over_a_cache_in_4_bits(B, C, H, H_kv, d, heads, resident):
    """Four rounds of the blocks that share an SM (four at most: three where a block takes eight heads of 128), no more than pieces of 512
    slots. (The scratch is that of the step in the storage type, with two blocks an SM or one and sixteen heads a block, where that is larger.)"""
    p = api.attn_params(B, 1, H, H_kv, d, T_k=C)
    sms, G = torch.cuda.get_device_properties(0).multi_processor_count, H // H_kv
    parts = lambda heads, resident: max(1, min(up(4 * resident * sms, B * H_kv * up(G, heads)), up(C, 512)))  # noqa: E731
    n = max(parts(heads, resident), parts(4 if G <= 4 else 8, 2 if d == 64 else 1))
    assert api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_DECODE) == (0 if n == 1 else up(4 * B * H * n * (d + 2), 256) * 256)
