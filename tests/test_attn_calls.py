"""Attention calls at the edges of what is documented: the smallest and largest caps and scales, rows that are not finite behind a shared-out
past, many sequences with prefixes, captured calls that share their scratch."""
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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("kw", [dict(), dict(cap=9.0), dict(slopes=True)])
def test_rows_that_are_not_finite_behind_a_past_that_is_shared_out(kw, bad, dtype, exact):
    """77 queries behind 4096 keys, whose keys are shared out over several blocks: what the last 13 tokens hold reaches the earlier queries
    neither by the products nor where a part's rows are computed again."""
    T, T_k, H, H_kv, d, at = 77, 4096, 4, 2, 64, 64
    q, k, v, dO = [draw((1, n, h, d), 40 + i, dtype) for i, (n, h) in enumerate(((T, H), (T_k, H_kv), (T_k, H_kv), (T, H)))]
    sl = torch.tensor([2.0 ** (-3 - h) for h in range(H)], device="cuda") if kw.get("slopes") else None
    p = api.attn_params(1, T, H, H_kv, d, T_k=T_k, dtype=dtype, exact=exact, cap=kw.get("cap", 0.0))
    ref = attention(q, k, v, visible(T, T_k, 1, 0), 0.125, kw.get("cap", 0.0), sl, dO)
    for x, n in ((q, T), (k, T_k), (v, T_k), (dO, T)):
        x[:, n - T + at:, :, 5] = bad
    r = api.lawcat_attn_fwd(p, q, k, v, slopes=sl)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, slopes=sl))
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    err = dict(ref["grad_err"](coarse, out), o=ref["o_sum"] + coarse * ref["o_mag"], lse=ref["lse_err"])
    for n in ("o", "lse", "dq"):
        check(r[n][:, :at], ref[n][:, :at], err[n][:, :at], U32 if n == "lse" else out, n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
def test_more_sequences_with_prefixes_than_one_table(dtype, exact):
    """600 sequences (three launches of the interval table), each with a prefix of its own, more keys than queries."""
    B, T, T_k, H, H_kv, d = 600, 9, 14, 2, 1, 64
    q, k, v, dO = [draw((B, n, h, d), i, dtype) for i, (n, h) in enumerate(((T, H), (T_k, H_kv), (T_k, H_kv), (T, H)))]
    prefix = [(5 * b) % (T_k + 1) for b in range(B)]
    p = api.attn_params(B, T, H, H_kv, d, T_k=T_k, dtype=dtype, exact=exact)
    r = api.lawcat_attn_fwd(p, q, k, v, prefix=prefix)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, prefix=prefix))
    ref = attention(q, k, v, visible(T, T_k, 1, 0, None, prefix, B), 0.125, 0.0, None, dO, r["o"])
    coarse, out = U16 if dtype == "bf16" and not exact else 0.0, U16 if dtype == "bf16" else U32
    err = dict(ref["grad_err"](coarse, out), o=ref["o_sum"] + coarse * ref["o_mag"], lse=ref["lse_err"])
    for n in ("o", "lse", "dq", "dk", "dv"):
        check(r[n], ref[n], err[n], U32 if n == "lse" else out, n)


@pytest.mark.gpu
def test_captured_calls_that_share_their_scratch():
    """Two graphs, each a forward and gradients, and a third with decode steps, over the same scratch, replayed in turn."""
    B, T, T_k, H, H_kv, d = 1, 70, 3000, 4, 2, 64
    ps = [api.attn_params(B, T, H, H_kv, d, T_k=T_k), api.attn_params(B, T, H, H_kv, d, T_k=T_k, dtype="f32", causal=0)]
    pd = api.attn_params(B, 1, H, H_kv, d, T_k=T_k)
    L = api.lib()
    ws = torch.empty(max(L.lawcat_attn_workspace_bytes(ctypes.byref(p), op) for p, ops in ((ps[0], (7, 8)), (ps[1], (7, 8)), (pd, (9,))) for op in ops),
                     dtype=torch.uint8, device="cuda")
    sets = [[draw((B, n, h, d), 10 * s + i, dt) for i, (n, h) in enumerate(((T, H), (T_k, H_kv), (T_k, H_kv), (T, H)))] for s, dt in ((0, "bf16"), (1, "f32"))]
    pos = torch.tensor([T_k - 1], dtype=torch.int32, device="cuda")

    def train(i):
        q, k, v, dO = sets[i]
        r = api.lawcat_attn_fwd(ps[i], q, k, v, ws=ws)
        r.update(api.lawcat_attn_bwd(ps[i], q, k, v, r["o"], r["lse"], dO, ws=ws))
        return r

    def decode():
        q, k, v, _ = sets[0]
        return dict(o=api.lawcat_attn_decode(pd, q[:, 0].contiguous(), k[:, -1].contiguous(), v[:, -1].contiguous(), k, v, pos, ws=ws))
    runs = [lambda: train(0), lambda: train(1), decode]
    want = [f() for f in runs]
    torch.cuda.synchronize()
    graphs = []
    for f in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = f()
        graphs.append((g, out))
    for order in ((0, 1, 2), (2, 1, 0), (1, 1, 0, 2, 2)):
        for i in order:
            graphs[i][0].replay()
        torch.cuda.synchronize()
        for (_, out), w in zip(graphs, want):
            for n in w:
                assert torch.equal(out[n], w[n]), n
