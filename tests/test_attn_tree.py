"""Attention of drafted tokens over a cache, in the storage type and in 4 bits, against 64 bits (tree_reference.py): trees and chains, rings that
wrap, windows, nodes and sequences that are not there, slots that hold no token, rows that are not finite; and that it gives what the same
tokens one by one give."""
import ctypes
import math
import random

import pytest
import torch

from attn_reference import U16, U32, check, quantized
from paper_2509_18467_b200 import api, build
from test_attn import draw
from test_attn_decode import rows_of
from tree_reference import U11, paths_of, sees, tree_attention

gpu = pytest.mark.gpu
KINDS = [("f32", 0), ("bf16", 1), ("bf16", 0)]


def some_tree(N, seed, depth=8):
    """Parents of N nodes, up to `depth` deep."""
    rng, row, d = random.Random(seed), [], []
    for i in range(N):
        p = -1 if i == 0 or rng.random() < 0.1 else rng.randint(max(0, i - 9), i - 1)
        while p >= 0 and d[p] >= depth - 1:
            p = row[p]
        row.append(p)
        d.append(d[p] + 1 if p >= 0 else 0)
    return row


def tree(quant, pos, N, C=100, H=4, H_kv=2, d=64, dtype="bf16", window=0, cap=0.0, slopes=False, exact=0, seed=0, parents=None, garbage=math.nan,
         mend=None, scale=None, std=1.5, ref_cap=None):
    """One call for sequences at positions `pos`; parents: a list of N per sequence, None for a chain, or a function of the sequence's number.
    Slots without a token and nodes that are not there hold `garbage`. mend(k, v, K, V): changes the inputs (storage type) in place."""
    B = len(pos)
    q, k, v = draw((B, N, H, d), seed, dtype, std), draw((B, N, H_kv, d), seed + 1, dtype), draw((B, N, H_kv, d), seed + 2, dtype)
    pasts = [draw((B, C, H_kv, d), seed + 3 + i, dtype) for i in range(2)]
    sl = torch.tensor([2.0 ** (-3 - h % 8) for h in range(H)], device="cuda") if slopes else None
    chain = parents is None
    parents = [list(range(-1, N - 1))] * B if chain else [parents(b) if callable(parents) else parents for b in range(B)]
    for b in range(B):
        for i, path in enumerate(paths_of(parents[b])):
            if not path or pos[b] < 0:
                for x in (q, k, v):
                    x[b, i] = garbage
    if mend:
        mend(k, v, *pasts)
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, dtype=dtype, window=window, cap=cap, exact=exact, scale=scale)
    if quant:
        cache = api.quant_cache(p)
        pc = api.attn_params(B, C, H, H_kv, d, T_k=C, dtype=dtype)
        api.lawcat_cache_quantize(pc, pasts[0], pasts[1], torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
        for b, x in enumerate(pos):
            for t in cache:
                t[b][:, max(0, x):].fill_(garbage if t.dtype != torch.uint8 else 255)
    else:
        cache = tuple(x.clone() for x in pasts)
        for b, x in enumerate(pos):
            for t in cache:
                t[b][max(0, x):].fill_(garbage)
    before = [t.clone() for t in cache]
    at = torch.tensor(pos, dtype=torch.int32, device="cuda")
    up = None if chain else torch.tensor(parents, dtype=torch.int32, device="cuda")
    f = api.lawcat_attn_tree_quant if quant else api.lawcat_attn_tree
    o = f(p, q, k, v, *cache, at, parent=up, slopes=sl, o_t=torch.full_like(q, 7.0))
    for t, was in zip(cache, before):
        assert torch.equal(t.view(torch.uint8), was.view(torch.uint8))
    coarse = dtype == "bf16" and not exact and d >= 64
    # operands on the tensor cores: weights in the storage type; over 4 bits weights, keys and values in fp16
    eps = dict(eps_p=U11, eps_k=U11, eps_v=U11, min_p=2.0 ** -25) if coarse and quant else dict(eps_p=U16) if coarse else {}
    for b, x in enumerate(pos):
        cached, see, dist = sees(parents[b], x, C, window)
        slots = torch.tensor(cached, dtype=torch.long, device="cuda") % C
        if quant:
            K, V = rows_of(cache, b, slots)
            kn, vn = quantized(k[b])[3], quantized(v[b])[3]
        else:
            K, V, kn, vn = cache[0][b][slots].double(), cache[1][b][slots].double(), k[b].double(), v[b].double()
        keys, values = torch.cat([K, kn]), torch.cat([V, vn])
        s = float(torch.tensor(d ** -0.5 if scale is None else scale))
        want, err = tree_attention(q[b], keys, values, see, dist, s, cap if ref_cap is None else ref_cap, sl, **eps)
        hidden = ~see.any(1).to(o.device)
        assert not o[b][hidden].any(), f"sequence {b}: nodes that are not there"
        check(o[b], want, err, U16 if dtype == "bf16" else U32, f"o of sequence {b} at {x}")
    return o


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("pos,C", [([0], 1), ([0, 1, 62, 63, 64, 65], 100), ([99, 100, 101, 250, -1, 7], 100), ([5, 700, -5, 1299, 1300], 1300), ([12345], 1300)])
def test_positions(pos, C, quant, dtype, exact):
    tree(quant, pos, 5, C, dtype=dtype, exact=exact, seed=len(pos) + C)
    tree(quant, pos, 21, C, dtype=dtype, exact=exact, seed=len(pos) + C, parents=lambda b: some_tree(21, b))


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("N", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 256])
def test_numbers_of_nodes(N, quant, dtype, exact):
    tree(quant, [300, 11], N, 400, H=4, H_kv=2, dtype=dtype, exact=exact, seed=N, parents=lambda b: some_tree(N, N + b, 2 + 20 * b))


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (8, 8), (12, 4), (8, 1), (20, 2), (32, 1)])
def test_heads_and_widths(H, H_kv, d, quant, dtype, exact):
    tree(quant, [40, 333, 600], 11, 400, H=H, H_kv=H_kv, d=d, dtype=dtype, exact=exact, seed=H + d, parents=lambda b: some_tree(11, b))


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("kw", [dict(window=1), dict(window=2), dict(window=64), dict(window=65, slopes=True), dict(window=333, slopes=True), dict(cap=4.0),
                                dict(cap=20.0, slopes=True), dict(slopes=True), dict(scale=-0.1), dict(scale=0.0, slopes=True), dict(scale=0.5, std=4.0)])
def test_windows_caps_and_biases(kw, quant, dtype):
    tree(quant, [0, 1, 63, 64, 500, 1111], 40, 600, dtype=dtype, d=128, H=8, H_kv=2, seed=7, parents=lambda b: some_tree(40, b), **kw)


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("C,N", [(1, 5), (2, 9), (5, 70), (64, 26), (63, 200)])
def test_rings_shorter_than_the_tree(C, N, quant, dtype, exact):
    """A path deeper than the ring: its nodes see the nearest C tokens, the cache's share shrinking to none."""
    tree(quant, [0, C - 1, C, 10 * C + 3], N, C, dtype=dtype, exact=exact, seed=C)
    tree(quant, [0, C - 1, C, 10 * C + 3], N, C, dtype=dtype, exact=exact, seed=C, window=(C + 1) // 2, slopes=True, parents=lambda b: some_tree(N, b, N))


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
def test_nodes_that_are_not_there(quant, dtype, exact):
    """Padding, parents behind their nodes or out of range, and what hangs from such a node."""
    rows = [[-1, 0, 1, -2, -2, -2, -2], [-2] * 7, [0, -1, 1, 9, 3, -5, 2], [-1, 2, 1, 0, 3, 2 ** 31 - 1, -2 ** 31], [-1, 0, 0, 0, 0, 0, 0]]
    tree(quant, [50, 60, 70, 0, 130], 7, 100, dtype=dtype, exact=exact, seed=3, parents=lambda b: rows[b])
    tree(quant, [50, 60, 70, 0, 130], 7, 100, dtype=dtype, exact=exact, seed=3, parents=lambda b: rows[b], garbage=math.inf, H=32, H_kv=8, d=128)


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
def test_long_cache(quant, dtype, exact):
    """Many parts per sequence, lengths from one token on, and positions near the end of 32 bits."""
    tree(quant, [0, 300, 9000, 20000, 2 ** 31 - 1], 19, 9000, H=8, H_kv=2, d=128, seed=5, dtype=dtype, exact=exact, parents=lambda b: some_tree(19, b))


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("C", [90, 3000])
def test_rows_that_are_not_finite(C, quant, dtype, exact):
    """A node whose value is not finite reaches the nodes on whose path it lies and no others; the same for a cached token that has left the
    window of the deeper nodes."""
    N, window = 12, 60
    parent = [-1, 0, 1, 2, 3, -1, 5, 6, 1, 8, -1, 10]
    B, pos = 2, [80 if C == 90 else 2900, 75]
    q = draw((B, N, 8, 64), 1, dtype, 1.5)
    k, v = draw((B, N, 2, 64), 2, dtype), draw((B, N, 2, 64), 3, dtype)
    K, V = draw((B, C, 2, 64), 4, dtype), draw((B, C, 2, 64), 5, dtype)
    p = api.attn_params(B, N, 8, 2, 64, T_k=C, dtype=dtype, exact=exact, window=window)
    at, up = torch.tensor(pos, dtype=torch.int32, device="cuda"), torch.tensor([parent] * B, dtype=torch.int32, device="cuda")

    def run(k, v, K, V):
        if not quant:
            return api.lawcat_attn_tree(p, q, k, v, K, V, at, parent=up)
        cache = api.quant_cache(p)
        pc = api.attn_params(B, C, 8, 2, 64, T_k=C, dtype=dtype)
        api.lawcat_cache_quantize(pc, K, V, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
        return api.lawcat_attn_tree_quant(p, q, k, v, *cache, at, parent=up)

    clean = run(k, v, K, V)
    for bad in (math.nan, math.inf):
        for which in (0, 1):
            x = [k.clone(), v.clone(), K.clone(), V.clone()]
            x[which][0, 5] = bad                              # nodes 5, 6, 7 see it
            x[2 + which][0, (pos[0] - window + 2) % C] = bad  # 58 behind: nodes of depth 0 and 1 see it
            got = run(*x)
            depth = [len(y) - 1 for y in paths_of(parent)]
            hit = torch.tensor([i in (5, 6, 7) or depth[i] <= 1 for i in range(N)], device="cuda")
            assert not torch.isfinite(got[0][hit]).all(-1).any(), (bad, which)
            tol = 2 * (U16 if dtype == "bf16" else 64 * U32) * (1 + clean[0][~hit].float().abs())
            assert ((got[0][~hit].float() - clean[0][~hit].float()).abs() <= tol).all()
            assert torch.equal(got[1], clean[1])


@gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("window", [0, 40])
def test_the_same_tokens_one_by_one(window, dtype, exact, quant):
    """rotate -> verify a tree -> accept a path, against rotate -> decode step by step along that path."""
    B, N, C, H, H_kv, d = 3, 14, 64, 8, 2, 64
    pos0 = [10, 63, 200]
    parents = [some_tree(N, 40 + b, 6) for b in range(B)]
    paths = []
    for b in range(B):
        paths.append(max(paths_of(parents[b]), key=len))
    M = max(map(len, paths))
    path = torch.tensor([x + [-1] * (M - len(x)) for x in paths], dtype=torch.int32, device="cuda")
    q, k, v = draw((B, N, H, d), 1, dtype, 1.5), draw((B, N, H_kv, d), 2, dtype), draw((B, N, H_kv, d), 3, dtype)
    pasts = [draw((B, C, H_kv, d), 4 + i, dtype) for i in range(2)]
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, dtype=dtype, exact=exact, window=window)
    p1 = api.attn_params(B, 1, H, H_kv, d, T_k=C, dtype=dtype, exact=exact, window=window)
    pc = api.attn_params(B, C, H, H_kv, d, T_k=C, dtype=dtype)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def fresh():
        if not quant:
            return [x.clone() for x in pasts]
        c = api.quant_cache(p)
        api.lawcat_cache_quantize(pc, *pasts, ints([0] * B), *c)
        return list(c)

    rope = api.rope_params(B, N, H, H_kv, d, dtype=dtype)
    freq = api.rope_frequencies(d)
    pos, up = ints(pos0), ints(parents)
    cache, steps = fresh(), fresh()
    qr, kr = api.lawcat_rope_fwd(rope, freq, q, k, start=pos, parent=up)
    o = (api.lawcat_attn_tree_quant if quant else api.lawcat_attn_tree)(p, qr, kr, v, *cache, pos, parent=up)
    after = (api.lawcat_cache_accept_quant if quant else api.lawcat_cache_accept)(p, kr, v, pos, *cache, path=path)
    assert after.tolist() == [x + len(y) for x, y in zip(pos0, paths)]
    rope1 = api.rope_params(B, 1, H, H_kv, d, dtype=dtype)
    rows = torch.arange(B, device="cuda")
    for t in range(M):
        live = [t < len(x) for x in paths]
        node = torch.tensor([x[min(t, len(x) - 1)] for x in paths], device="cuda")
        here = ints([x + t if y else -1 for x, y in zip(pos0, live)])
        q1, k1 = api.lawcat_rope_fwd(rope1, freq, q[rows, node][:, None].contiguous(), k[rows, node][:, None].contiguous(), start=ints([x + t for x in pos0]))
        o1 = (api.lawcat_attn_decode_quant if quant else api.lawcat_attn_decode)(p1, q1[:, 0], k1[:, 0], v[rows, node], *steps, here)
        for b in range(B):
            if live[b]:
                x, y = o[b, node[b]].float(), o1[b].float()
                # (both are off by roundings of weights, relative to the largest value at most, and one of the result)
                tol = 4 * (U16 if dtype == "bf16" else 64 * U32) * float(v.float().abs().max())
                assert float((x - y).abs().max()) <= tol
    for x, y in zip(cache, steps):   # the same bits in the cache
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("dtype,exact", KINDS)
def test_captured_and_replayed(dtype, exact, quant):
    """A captured verification reads the positions, parents and cache that it finds; two of them share one scratch."""
    B, N, C, H, H_kv, d = 2, 9, 1500, 8, 2, 128
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, dtype=dtype, exact=exact)
    q, k, v = draw((B, N, H, d), 1, dtype), draw((B, N, H_kv, d), 2, dtype), draw((B, N, H_kv, d), 3, dtype)
    pasts = [draw((B, C, H_kv, d), 4 + i, dtype) for i in range(2)]
    if quant:
        cache = api.quant_cache(p)
        pc = api.attn_params(B, C, H, H_kv, d, T_k=C, dtype=dtype)
        api.lawcat_cache_quantize(pc, *pasts, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
        f = api.lawcat_attn_tree_quant
    else:
        cache, f = pasts, api.lawcat_attn_tree
    pos = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    up = torch.tensor([some_tree(N, b) for b in range(B)], dtype=torch.int32, device="cuda")
    ws = torch.empty(max(16, int(api.lib().lawcat_attn_workspace_bytes(ctypes.byref(p), api.OP_ATTN_TREE))), dtype=torch.uint8, device="cuda")
    f(p, q, k, v, *cache, pos, parent=up, ws=ws)
    torch.cuda.synchronize()
    g, h = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = f(p, q, k, v, *cache, pos, parent=up, ws=ws)
    with torch.cuda.graph(h):
        chain = f(p, q, k, v, *cache, pos, ws=ws)
    for at in ([0, 1], [1499, 1500], [2900, 700], [-1, 64]):
        pos.copy_(torch.tensor(at))
        up.copy_(torch.tensor([some_tree(N, at[0] + b + 3) for b in range(B)]))
        ws.fill_(255)   # (NaN everywhere)
        g.replay()
        h.replay()
        assert torch.equal(got, f(p, q, k, v, *cache, pos, parent=up))
        assert torch.equal(chain, f(p, q, k, v, *cache, pos))


@gpu
@pytest.mark.parametrize("quant", [False, True])
def test_two_streams_at_once(quant):
    B, N, C, H, H_kv, d = 2, 20, 5000, 8, 2, 64
    p = api.attn_params(B, N, H, H_kv, d, T_k=C)
    q, k, v = draw((B, N, H, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    pasts = [draw((B, C, H_kv, d), 4 + i, "bf16") for i in range(2)]
    f, cache = api.lawcat_attn_tree, pasts
    if quant:
        cache, f = api.quant_cache(p), api.lawcat_attn_tree_quant
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), *pasts, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    pos = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([4000, 17], [1, 6000])]
    want = [f(p, q, k, v, *cache, x) for x in pos]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pos]
    for _ in range(20):
        got = [f(p, q, k, v, *cache, x, stream=s) for x, s in zip(pos, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@gpu
def test_offsets_beyond_32_bits():
    """A cache of more than 2^31 elements: the last sequence's slots lie behind them."""
    B, C, H, H_kv, d, N = 17, 262144, 4, 4, 128, 3
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, window=50)
    K = torch.zeros(B, C, H_kv, d, dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    x = 5 * C + C - 1
    pos = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    pos[-1] = x
    q, k, v = draw((B, N, H, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    cached, see, dist = sees([-1, 0, 0], x, C, 50)
    slots = torch.tensor(cached, device="cuda") % C
    K[-1, slots], V[-1, slots] = draw((49, H_kv, d), 4, "bf16"), draw((49, H_kv, d), 5, "bf16")
    up = torch.tensor([[-1, 0, 0]] * B, dtype=torch.int32, device="cuda")
    o = api.lawcat_attn_tree(p, q, k, v, K, V, pos, parent=up)
    assert not o[:-1].any()
    want, err = tree_attention(q[-1], torch.cat([K[-1, slots], k[-1]]), torch.cat([V[-1, slots], v[-1]]), see, dist, float(torch.tensor(d ** -0.5)), eps_p=U16)
    check(o[-1], want, err, U16, "o")
    api.lawcat_cache_accept(p, k, v, pos, K, V)
    assert torch.equal(K[-1, [C - 1, 0, 1]], k[-1]) and torch.equal(V[-1, [C - 1, 0, 1]], v[-1])
    assert not K[:-1].any()


def test_refusals():
    build.build()
    L, x, odd = api.lib(), ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)
    ok = dict(B=2, T=8, H=4, H_kv=2, d=64, T_k=100)
    call = lambda p, ptrs, ws=x, nb=1 << 30: L.lawcat_attn_tree(ctypes.byref(p), *ptrs, ws, nb, None, None)  # noqa: E731
    good = [x] * 6 + [None, None, x]
    P = lambda **kw: api.attn_params(**{**ok, **kw})  # noqa: E731
    for kw in (dict(B=-1), dict(T=-1), dict(H_kv=3), dict(dtype=2), dict(window=-1), dict(window=101), dict(T_k=0), dict(scale=math.inf), dict(cap=-1.0)):
        assert call(P(**kw), good) == 1, kw
        assert L.lawcat_attn_workspace_bytes(ctypes.byref(P(**kw)), api.OP_ATTN_TREE) == 0
    for kw in (dict(d=48), dict(T=257), dict(B=1 << 20, T=256, H=32, H_kv=2)):
        assert call(P(**kw), good) == 2, kw
    for i in range(9):
        bad = list(good)
        bad[i] = odd
        assert call(P(), bad) == 1, i
        if i not in (6, 7):
            bad[i] = None
            assert call(P(), bad) == 1, i
    assert call(P(T_k=100000), good, None, 0) == 4 and call(P(T_k=100000), good, x, 64) == 4
    assert call(P(B=0), [None] * 9) == 0 and call(P(T=0), [None] * 9) == 0
    quant = lambda p, ptrs: L.lawcat_attn_tree_quant(ctypes.byref(p), *ptrs, x, 1 << 30, None, None)  # noqa: E731
    good = [x] * 8 + [None, None, x]
    for i in range(11):
        bad = list(good)
        bad[i] = odd
        assert quant(P(), bad) == 1, i
        if i not in (8, 9):
            bad[i] = None
            assert quant(P(), bad) == 1, i
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    p = P()
    args = dict(q_t=z(2, 8, 4, 64), k_t=z(2, 8, 2, 64), v_t=z(2, 8, 2, 64), K=z(2, 100, 2, 64), V=z(2, 100, 2, 64), pos=z(2, dt=torch.int32))
    for name, t in (("q_t", z(2, 7, 4, 64)), ("k_t", z(2, 8, 4, 64)), ("V", z(2, 100, 2, 64, dt=torch.float32)), ("pos", z(2, dt=torch.int64)),
                    ("parent", z(2, 9, dt=torch.int32)), ("slopes", z(4)), ("o_t", z(2, 8, 2, 64))):
        with pytest.raises(ValueError, match=f"^{name}: expected"):
            api.lawcat_attn_tree(p, **{**args, name: t})
