"""Accepted tokens into a cache, in the storage type and in 4 bits: paths, whole pieces of a prompt, rings that wrap, sequences that are not
there; what is not written stays as it is."""
import ctypes

import pytest
import torch

from paper_2509_18467_b200 import api, build
from test_attn import draw

gpu = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.uint8)


def accept(quant, pos, T, C, path=None, H_kv=2, d=64, dtype="bf16", seed=0, want_pos=True):
    B = len(pos)
    k, v = draw((B, T, H_kv, d), seed, dtype), draw((B, T, H_kv, d), seed + 1, dtype)
    p = api.attn_params(B, T, H_kv, H_kv, d, T_k=C, dtype=dtype)
    at = torch.tensor(pos, dtype=torch.int32, device="cuda")
    if quant:
        cache = [torch.randint(0, 255, t.shape, device="cuda").to(t.dtype) for t in api.quant_cache(p)]
    else:
        cache = [draw((B, C, H_kv, d), seed + 2 + i, dtype) for i in range(2)]
    want = [t.clone() for t in cache]
    ends = []
    for b, x in enumerate(pos):
        rows = list(range(T)) if path is None else path[b]
        n = next((i for i, r in enumerate(rows) if not 0 <= r < T), len(rows))
        rows = rows[:n] if x >= 0 else []
        ends.append(x + len(rows))
        for t, r in list(enumerate(rows))[max(0, len(rows) - C):]:
            slot = (x + t) % C
            if quant:   # (one row by the call that quantizes rows in order)
                one = api.attn_params(1, 1, H_kv, H_kv, d, T_k=C, dtype=dtype)
                row = [y[b:b + 1].clone() for y in want]
                api.lawcat_cache_quantize(one, k[b:b + 1, r:r + 1].contiguous(), v[b:b + 1, r:r + 1].contiguous(),
                                          torch.tensor([slot], dtype=torch.int32, device="cuda"), *row)
                for y, z in zip(want, row):
                    y[b:b + 1] = z
            else:
                want[0][b, slot], want[1][b, slot] = k[b, r], v[b, r]
    up = None if path is None else torch.tensor(path, dtype=torch.int32, device="cuda")
    f = api.lawcat_cache_accept_quant if quant else api.lawcat_cache_accept
    got = f(p, k, v, at, *cache, path=up)
    assert got.tolist() == ends and at.tolist() == list(pos)
    for x, y in zip(cache, want):
        assert torch.equal(bits(x), bits(y))


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("H_kv", [1, 3, 8])
def test_paths(H_kv, d, quant, dtype):
    path = [[0, 2, 5, -1], [6, 6, 1, 0], [-1, 0, 1, 2], [3, 7, 1, 2], [1, -2 ** 31, 0, 0], [4, 2 ** 31 - 1, 0, 0], [0, 1, 2, 3]]
    accept(quant, [0, 19, 5, 20, 33, 2 ** 31 - 9, -1], 7, 20, path, H_kv=H_kv, d=d, dtype=dtype, seed=H_kv + d)


@gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("M,C", [(1, 1), (9, 4), (300, 64), (300, 700), (3, 2)])
def test_paths_longer_than_the_ring(M, C, quant):
    accept(quant, [0, 5, 1000], 4, C, [[(i * 7 + b) % 4 if i < M - b else -1 for i in range(M)] for b in range(3)], seed=M)


@gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("T,C", [(1, 5), (37, 100), (100, 100), (250, 100)])
def test_whole_pieces(T, C, quant):
    accept(quant, [0, 77, -3], T, C, H_kv=4, d=32, seed=T)


@gpu
def test_a_long_piece():
    accept(False, [100, 8000], 5000, 8192, H_kv=8, d=128)


@gpu
@pytest.mark.parametrize("quant", [False, True])
def test_captured_and_replayed(quant):
    p = api.attn_params(2, 5, 2, 2, 64, T_k=30)
    k, v = draw((2, 5, 2, 64), 1, "bf16"), draw((2, 5, 2, 64), 2, "bf16")
    cache = api.quant_cache(p) if quant else [torch.zeros(2, 30, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    pos, nxt = (torch.tensor([3, 4], dtype=torch.int32, device="cuda") for _ in range(2))
    path = torch.tensor([[0, 1, -1], [-1, 0, 0]], dtype=torch.int32, device="cuda")
    f = api.lawcat_cache_accept_quant if quant else api.lawcat_cache_accept
    f(p, k, v, pos, *[t.clone() for t in cache], path=path, pos_out=nxt)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f(p, k, v, pos, *cache, path=path, pos_out=nxt)
    want = [t.clone() for t in cache]
    for row in ([[0, 1, -1], [-1, 0, 0]], [[4, 2, 0], [3, -1, 0]], [[-1, 0, 0], [1, 1, 1]]):
        path.copy_(torch.tensor(row))
        g.replay()
        f(p, k, v, pos, *want, path=path)
        assert all(torch.equal(bits(x), bits(y)) for x, y in zip(cache, want))
        pos.copy_(nxt)


def test_refusals():
    build.build()
    L, x, y, odd = api.lib(), ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_void_p(0x1008)
    call = lambda p, M, ptrs: L.lawcat_cache_accept(ctypes.byref(p), M, *ptrs, None, 0, None, None)  # noqa: E731
    P = lambda **kw: api.attn_params(**{**dict(B=2, T=8, H=4, H_kv=2, d=64, T_k=100), **kw})  # noqa: E731
    good = [x, x, x, x, x, x, y]   # k, v, pos, path, K, V, pos_out
    for kw in (dict(B=-1), dict(T=-1), dict(dtype=7), dict(T_k=0), dict(window=101)):
        assert call(P(**kw), 3, good) == 1, kw
    assert call(P(d=48), 3, good) == 2 and call(P(), -1, good) == 1
    for i in range(7):
        bad = list(good)
        bad[i] = odd
        assert call(P(), 3, bad) == 1, i
        if i not in (3, 6):
            bad[i] = None
            assert call(P(), 3, bad) == 1, i
    assert call(P(), 3, [x, x, x, x, x, x, x]) == 1       # pos_out is pos
    assert call(P(B=0), 3, [None] * 7) == 0 and call(P(T=0), 3, [None, None, x, x, None, None, None]) == 0
    quant = lambda p, ptrs: L.lawcat_cache_accept_quant(ctypes.byref(p), 3, *ptrs, None, 0, None, None)  # noqa: E731
    good = [x] * 8 + [y]
    for i in range(9):
        bad = list(good)
        bad[i] = odd
        assert quant(P(), bad) == 1, i
        if i not in (3, 8):
            bad[i] = None
            assert quant(P(), bad) == 1, i
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    args = dict(k_t=z(2, 8, 2, 64), v_t=z(2, 8, 2, 64), pos=z(2, dt=torch.int32), K=z(2, 100, 2, 64), V=z(2, 100, 2, 64))
    for name, t in (("k_t", z(2, 7, 2, 64)), ("pos", z(3, dt=torch.int32)), ("path", z(3, 4, dt=torch.int32)), ("path", z(2, 4, dt=torch.int64)),
                    ("K", z(2, 99, 2, 64)), ("pos_out", z(2))):
        with pytest.raises(ValueError, match=f"^{name}: expected"):
            api.lawcat_cache_accept(P(), **{**args, name: t})
    with pytest.raises(ValueError, match="^path: no entries"):
        api.lawcat_cache_accept(P(), **{**args, "path": z(2, 0, dt=torch.int32)})
