"""Rotary positions and their gradient against 64 bits: layouts, parts of a head, far and negative positions, packed documents, drafted nodes,
scalings for long contexts, results in place; and what is refused.

Tolerance: the angle is off by half a step of a float in [-1, 1) half turns (pi 2^-25) and 2^-32 of a turn, sine and cosine by 2 steps of
their own (2 * 2^-23): less than 2^-21 together; the products, their sum and the scale add 4 * 2^-24; the result is rounded once."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

from attn_reference import U16, U32, check
from paper_2509_18467_b200 import api, build

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
PI = Fraction("3.14159265358979323846264338327950288419716939937510")


def draw(shape, seed, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(DT[dtype]).cuda()


def angles(positions, freq):
    """[..., pairs] angles modulo a turn in 64 bits, from exact products."""
    flat = positions.reshape(-1).tolist()
    exact = [Fraction(f) for f in freq]
    if max(abs(n) for n in flat) < 1 << 20:   # (a product in 64 bits is then off by 2^-33 at most)
        return positions.double()[..., None] * torch.tensor(list(freq), dtype=torch.float64)
    rows = [[float((n * f) % (2 * PI)) for f in exact] for n in flat]
    return torch.tensor(rows, dtype=torch.float64).reshape(*positions.shape, len(exact))


def turned(x, positions, freq, rot, layout, scale, sign):
    """Result and error bound in 64 bits; x [B, T, heads, d], positions [B, T]."""
    a = sign * angles(positions, freq)[:, :, None].to(x.device)
    y, err = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    u, w = x[..., one].double(), x[..., two].double()
    y[..., one], y[..., two] = scale * (u * a.cos() - w * a.sin()), scale * (u * a.sin() + w * a.cos())
    err[..., one] = err[..., two] = abs(scale) * (u.abs() + w.abs()) * (2.0 ** -21 + 4 * U32)
    return y, err


def case(B=2, T=7, H=4, H_kv=2, d=64, rot=None, layout="half", dtype="bf16", scale=1.0, positions=None, start=None, parent=None, at=None, freq=None,
         place=False, seed=0, only_q=False):
    rot = rot or d
    freq = api.rope_frequencies(rot) if freq is None else freq
    p = api.rope_params(B, T, H, H_kv, d, rot=rot, layout=layout, dtype=dtype, scale=scale)
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kw = dict(positions=ints(positions), start=ints(start), parent=ints(parent))
    if at is None:
        at = positions if positions is not None else [[s + t for t in range(T)] for s in (start or [0] * B)]
    at = torch.tensor(at)
    for f, sign in ((api.lawcat_rope_fwd, 1), (api.lawcat_rope_bwd, -1)):
        q, k = draw((B, T, H, d), seed, dtype), None if only_q else draw((B, T, H_kv, d), seed + 1, dtype)
        want = [turned(x, at, freq, rot, layout, float(torch.tensor(scale)), sign) for x in (q, k) if x is not None]
        if place:
            got = f(p, freq, q, k, **kw, **(dict(q_out=q, k_out=k) if sign > 0 else dict(dq=q, dk=k)))
            assert got[0] is q and got[1] is k
        else:
            got = f(p, freq, q, k, **kw)
        for x, (y, err), name in zip(got, want, "qk"):
            check(x, y, err, U16 if dtype == "bf16" else U32, f"{name}, sign {sign}")
            assert torch.equal(x[..., rot:].double(), y[..., rot:])


LAYOUTS = ["half", "interleaved"]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d,rot", [(16, 16), (16, 2), (32, 32), (32, 20), (64, 64), (64, 32), (64, 6), (128, 128), (128, 64), (128, 126), (128, 8), (128, 12)])
def test_widths(d, rot, layout, dtype):
    case(d=d, rot=rot, layout=layout, dtype=dtype, T=19, start=[0, 1000], seed=d + rot)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("B,T,H,H_kv", [(1, 1, 1, 1), (1, 1, 32, 8), (64, 1, 32, 8), (1, 1223, 32, 8), (3, 511, 7, 1), (2, 2049, 5, 5), (1, 3, 128, 128)])
def test_sizes(B, T, H, H_kv, layout):
    case(B=B, T=T, H=H, H_kv=H_kv, layout=layout, d=128, start=[37 * b for b in range(B)], seed=T)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_and_negative_positions(dtype):
    at = [[0, -1, 1, 131071, 131072, -131072, 2 ** 20 + 1, 2 ** 31 - 1, -2 ** 31, 1234567891]]
    case(B=1, T=len(at[0]), d=128, positions=at, dtype=dtype)
    case(B=2, T=3, d=64, start=[2 ** 31 - 3, -2 ** 31], at=[[2 ** 31 - 3 + t for t in range(3)], [-2 ** 31 + t for t in range(3)]], dtype=dtype)


@pytest.mark.gpu
def test_packed_documents():
    at = [[t for n in (5, 1, 0, 300, 17) for t in range(n)]]
    case(B=1, T=len(at[0]), positions=at, rot=32, layout="interleaved")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [6, 300])
def test_drafted_nodes(T):
    """Depths from parents; nodes that are not there stand at the start."""
    parent = [-1, 0, 0, 2, 1, -1] + [i - 1 for i in range(6, T)]
    depth = [0, 1, 1, 2, 2, 0] + list(range(1, T - 5))
    gone = [3, -1, -2, 2, 7, -1] + [-2] * (T - 6)
    gone_depth = [0, 0, 0, 0, 0, 0] + [0] * (T - 6)
    case(B=2, T=T, start=[100, 7], parent=[parent, gone], at=[[100 + e for e in depth], [7 + e for e in gone_depth]])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_in_place(layout, dtype):
    case(B=2, T=133, d=128, rot=64, layout=layout, dtype=dtype, start=[0, 5], place=True)


@pytest.mark.gpu
def test_queries_alone_and_a_scale():
    case(only_q=True, scale=1.3, T=40)
    case(scale=-0.25, T=40, freq=[0.0, 6.283185307179586] + [1e-9 * 3 ** i for i in range(20)], rot=44)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS)
def test_gradient_against_differences(layout):
    """<dL/dq, e> is what L changes by along e; L = <w, rope(q)> is linear, so that a difference of any length is exact but for roundings."""
    p = api.rope_params(1, 50, 3, 3, 32, rot=20, layout=layout, dtype="f32", scale=0.7)
    freq = api.rope_frequencies(20)
    q, w, e = draw((1, 50, 3, 32), 1, "f32"), draw((1, 50, 3, 32), 2, "f32"), draw((1, 50, 3, 32), 3, "f32")
    start = torch.tensor([9], dtype=torch.int32, device="cuda")
    L = lambda x: (w.double() * api.lawcat_rope_fwd(p, freq, x, start=start)[0].double()).sum()  # noqa: E731
    dq, _ = api.lawcat_rope_bwd(p, freq, w, start=start)
    diff, slope = L(q + e) - L(q - e), 2 * (dq.double() * e.double()).sum()
    room = 4 * (2.0 ** -21 + 8 * U32) * float((w.abs() * (q.abs() + e.abs()).amax(-1, keepdim=True)).double().sum()) * 2
    assert abs(float(diff - slope)) <= room


@pytest.mark.gpu
def test_captured_call_keeps_its_frequencies_and_reads_new_positions():
    p = api.rope_params(2, 3, 4, 2, 64)
    q, k = draw((2, 3, 4, 64), 1, "bf16"), draw((2, 3, 2, 64), 2, "bf16")
    start = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    api.lawcat_rope_fwd(p, api.rope_frequencies(64), q, k, start=start)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        freq = api.rope_frequencies(64)
        got = api.lawcat_rope_fwd(p, freq, q, k, start=start)
        for i in range(32):
            freq[i] = 0.0
    start += 1000
    g.replay()
    want = api.lawcat_rope_fwd(p, api.rope_frequencies(64), q, k, start=start)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("scaling,kw", [("plain", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=4.0)),
                                        ("wavelength", dict(factor=8.0, original=4096, low=1.0, high=4.0)),
                                        ("channel", dict(factor=16.0, original=8192, low=1.0, high=32.0)),
                                        ("channel", dict(factor=2.0, original=10, low=1.0, high=32.0))])
@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (20, 100.0)])
def test_frequencies(rot, base, scaling, kw):
    build.build()
    got = list(api.rope_frequencies(rot, base, scaling, **kw))
    factor, original = kw.get("factor", 1.0), kw.get("original", 0.0)
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    for i, f in enumerate(got):
        plain = base ** (-2 * i / rot)
        if scaling in ("plain", "base"):
            keep = 1.0
        elif scaling == "linear":
            keep = 0.0
        elif scaling == "wavelength":
            keep = min(1.0, max(0.0, (original * plain / (2 * math.pi) - 1.0) / 3.0))
        else:
            c = lambda r: rot * math.log(original / (2 * math.pi * r)) / (2 * math.log(base))  # noqa: E731
            a, z = max(0, math.floor(c(32.0))), min(rot - 1, math.ceil(c(1.0)))
            keep = 1 - min(1.0, max(0.0, (i - a) / max(z - a, 0.001)))
        assert f == pytest.approx(plain * (keep + (1 - keep) / factor), rel=1e-12)


def test_refusals():
    build.build()
    x = ctypes.c_void_p(0x1000)
    fwd = api.lib().lawcat_rope_fwd
    ok = dict(B=1, T=8, H=4, H_kv=2, d=64, dtype=1, rot=64, layout=0, scale=1.0)

    def call(freq=0.5, q=x, k=x, positions=None, start=None, parent=None, qo=x, ko=x, **kw):
        p = api.RopeParams(**{**ok, **kw})
        f = (ctypes.c_double * 64)(*[freq] * 64)
        return fwd(ctypes.byref(p), f, q, k, positions, start, parent, qo, ko, None, 0, None, None)

    for kw in (dict(B=-1), dict(T=-1), dict(dtype=2), dict(layout=2), dict(rot=0), dict(rot=3), dict(rot=66), dict(scale=math.inf), dict(scale=math.nan),
               dict(freq=-0.1), dict(freq=7.0), dict(freq=math.nan), dict(positions=x, start=x), dict(positions=x, parent=x), dict(qo=None), dict(ko=None),
               dict(q=ctypes.c_void_p(0x1004)), dict(start=ctypes.c_void_p(0x1004))):
        assert call(**kw) == 1, kw
    for kw in (dict(d=256, rot=64), dict(d=48, rot=48), dict(B=1 << 20, T=1 << 20), dict(H=1 << 20)):
        assert call(**kw) == 2, kw
    assert call(B=0) == 0 and call(T=0) == 0 and call(q=None, k=None) == 0
    assert fwd(ctypes.byref(api.RopeParams(**ok)), None, x, x, None, None, None, x, x, None, 0, None, None) == 1
    f = api.lib().lawcat_rope_frequencies
    out = (ctypes.c_double * 64)()
    for args in ((3, 1e4, 0, 1.0, 0.0, 1.0, 4.0), (0, 1e4, 0, 1.0, 0.0, 1.0, 4.0), (130, 1e4, 0, 1.0, 0.0, 1.0, 4.0), (64, 1.0, 0, 1.0, 0.0, 1.0, 4.0),
                 (64, 1e4, 5, 1.0, 0.0, 1.0, 4.0), (64, 1e4, 1, 0.5, 0.0, 1.0, 4.0), (64, 1e4, 3, 2.0, 0.0, 1.0, 4.0), (64, 1e4, 3, 2.0, 100.0, 4.0, 4.0),
                 (64, 1e4, 4, 2.0, 100.0, 0.0, 4.0), (64, math.inf, 0, 1.0, 0.0, 1.0, 4.0)):
        assert f(*args, out) == 1, args
    with pytest.raises(ValueError, match="angles"):
        api.lawcat_rope_fwd(api.rope_params(1, 2, 2, 2, 64), [0.5] * 31, torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="^k: expected"):
        api.lawcat_rope_fwd(api.rope_params(1, 2, 2, 2, 64), [0.5] * 32, None, torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="^positions: expected"):
        api.lawcat_rope_fwd(api.rope_params(1, 2, 2, 2, 64), [0.5] * 32, None, positions=torch.zeros(1, 2, dtype=torch.int64))
