"""Attention calls at the edges of what is documented: the smallest and largest caps and scales."""
import ctypes
import math

import pytest
import torch

from attn_reference import U16, U32, attention, check, visible
from paper_2509_18467_b200 import api, build
from test_attn import KINDS, draw

FP32_MAX = 3.4028234663852886e38


@pytest.mark.parametrize("scale,cap,ok", [
    (0.125, FP32_MAX, False), (0.125, 2.3e38, True), (0.125, 1e-39, False), (0.125, 1e-38, True), (1.3, 1e-38, False), (-1.3, 1e-38, False), (1e-3, 2e-39, False),
    (FP32_MAX, 0.0, False), (-FP32_MAX, 0.0, False), (2.3e38, 0.0, True), (1e20, 1e-20, False), (1e20, 1e-17, True), (0.0, 1e-38, True)])
def test_caps_and_scales_that_fp32_does_not_hold_are_refused(scale, cap, ok):
    build.build()
    p = api.attn_params(1, 8, 4, 2, 64, scale=scale, cap=cap)
    need = [api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), op) for op in (api.OP_ATTN_FWD, api.OP_ATTN_BWD)]
    assert all((n > 0) == ok for n in need)
    if not ok:
        x = ctypes.c_void_p(0x1000)
        assert api.lib().lawcat_attn_fwd(ctypes.byref(p), None, None, 0, x, x, x, None, x, None, x, 1 << 20, None, None) == 1
        assert api.lib().lawcat_attn_decode(ctypes.byref(p), *[x] * 6, None, x, x, 1 << 20, None, None) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("cap", [2.3e38, 1e30, 1e-30, 1e-38])
def test_the_largest_and_smallest_caps(cap, dtype, exact):
    """A cap far above all scores is none; under one far below them every key weighs the same. Query rows of zeros among them."""
    T, H, d = 200, 2, 64
    q, k, v = [draw((1, T, H, d), 5 + i, dtype) for i in range(3)]
    q[:, ::7] = 0.0
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    r = api.lawcat_attn_fwd(api.attn_params(1, T, H, H, d, dtype=dtype, exact=exact, cap=cap), q, k, v)
    scale = 0.125 if cap > 1 else 0.0
    ref = attention(q, k, v, visible(T, T, 1, 0), scale)
    check(r["o"], ref["o"], ref["o_sum"] + coarse * ref["o_mag"], out, "o")
    check(r["lse"], ref["lse"], ref["lse_err"], U32, "lse")
    p = api.attn_params(1, 1, H, H, d, T_k=T, dtype=dtype, exact=exact, cap=cap)
    pos = torch.tensor([T - 1], dtype=torch.int32, device="cuda")
    for t in (T - 1, T - 4):    # (the last row is not one of zeros, the other one is)
        step = [q[:, t].contiguous(), k[:, -1].contiguous(), v[:, -1].contiguous()]
        o = api.lawcat_attn_decode(p, *step, k.clone(), v.clone(), pos)
        ref = attention(q[:, t:t + 1], k, v, visible(1, T, 1, 0), scale)
        check(o[:, None], ref["o"], ref["o_sum"] + coarse * ref["o_mag"], out, f"row {t}")
