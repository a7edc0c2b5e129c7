"""Rotary positions, attention of drafted tokens and accepting where calls meet: tensors on another device, work queued on the stream of the call,
many query heads to a key-value head, pasts that nobody has written, and a training step (rotate, attention, its gradient, that of the rotation)."""
import pytest
import torch

from attn_reference import U16, U32, attention, check, visible
from paper_2509_18467_b200 import api, build
from test_attn import draw
from test_attn_devices import Elsewhere
from test_attn_tree import KINDS, some_tree, tree
from test_rope import turned

gpu = pytest.mark.gpu
B, T, C, H, H_kv, d = 2, 8, 16, 4, 2, 64


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def tensors(make):
    f32, i32, u8 = (dict(dtype=x) for x in (torch.float32, torch.int32, torch.uint8))
    q, k = (B, T, H, d), (B, T, H_kv, d)
    return dict(q=make(*q), k=make(*k), q_out=make(*q), k_out=make(*k), dq_out=make(*q), dk_out=make(*k), dq=make(*q), dk=make(*k),
                positions=make(B, T, **i32), start=make(B, **i32), parent=make(B, T, **i32), path=make(B, 3, **i32), pos_out=make(B, **i32),
                q_t=make(*q), k_t=make(*k), v_t=make(*k), o_t=make(*q), slopes=make(H, **f32), K=make(B, C, H_kv, d), V=make(B, C, H_kv, d),
                pos=make(B, **i32), ws=make(1 << 16, **u8), dev_status=make(1, **i32),
                kq=make(B, H_kv, C, d // 2, **u8), kp=make(B, H_kv, C, d // 32, 2), vq=make(B, H_kv, C, d // 2, **u8), vp=make(B, H_kv, C, d // 32, 2))


STORED, PACKED = ["K", "V"], ["kq", "kp", "vq", "vp"]
TREE = ["q_t", "k_t", "v_t", "pos", "parent", "slopes", "o_t", "ws", "dev_status"]
ACCEPT = ["k_t", "v_t", "pos", "path", "pos_out", "dev_status"]
CALLS = dict(lawcat_rope_fwd=["q", "k", "start", "parent", "q_out", "k_out"], lawcat_rope_bwd=["dq_out", "dk_out", "positions", "dq", "dk"],
             lawcat_attn_tree=TREE + STORED, lawcat_attn_tree_quant=TREE + PACKED, lawcat_cache_accept=ACCEPT + STORED,
             lawcat_cache_accept_quant=ACCEPT + PACKED)


@pytest.mark.parametrize("name,arg", [(n, a) for n, args in CALLS.items() for a in args])
def test_a_tensor_on_another_device_is_refused(name, arg):
    if torch.cuda.is_available() and torch.cuda.current_device() == 1:
        pytest.skip("the second GPU is the current one")
    here, there = tensors(lambda *s, **kw: torch.zeros(*s, **{"dtype": torch.bfloat16, **kw})), tensors(Elsewhere)
    kw = {n: here[n] for n in CALLS[name]}
    kw[arg] = there[arg]
    if "rope" in name:
        args = (api.rope_params(B, T, H, H_kv, d), api.rope_frequencies(d))
    else:
        args = (api.attn_params(B, T, H, H_kv, d, T_k=C),)
    with pytest.raises(ValueError, match=f"^{arg}: on device cuda:1"):
        getattr(api, name)(*args, **kw)


def test_frequencies_in_another_type():
    """Any sequence of numbers does; an array of floats is converted, not read as one of doubles."""
    import ctypes
    freq = api.rope_frequencies(d)
    seen = []
    fake = lambda name, p, op, args, *more: seen.append([ctypes.c_double.from_address(args[0] + 8 * i).value for i in range(d // 2)])  # noqa: E731
    q = torch.zeros(B, T, H, d, dtype=torch.bfloat16)
    with pytest.MonkeyPatch.context() as m:
        m.setattr(api, "_attn_call", fake)
        for x in (freq, list(freq), (ctypes.c_float * (d // 2))(*freq), torch.tensor(list(freq), dtype=torch.float64)):
            api.lawcat_rope_fwd(api.rope_params(B, T, H, H_kv, d), x, q)
    assert seen[0] == seen[1] == seen[3] == list(freq)
    assert all(abs(x - y) <= 2.0 ** -24 * y for x, y in zip(seen[2], freq))


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("G", [96, 128, 129, 200])
def test_many_heads_to_one(G, quant, dtype, exact):
    """(129 and more to a key-value head: the CUDA cores' kernel; with few nodes, so that the rows are about as many as elsewhere)"""
    # in bf16 the tensor cores' bounds hold for the CUDA cores too
    tree(quant, [0, 70, 333], 5, C=150, H=2 * G, H_kv=2, d=64, dtype=dtype, exact=exact, seed=G, parents=lambda b: some_tree(5, G + b))


@gpu
@pytest.mark.parametrize("quant", [False, True])
def test_calls_wait_for_their_stream(quant):
    """Everything of a step is written on a side stream, behind a long kernel, just ahead of the calls that read it; the answers are those of
    the same calls one at a time."""
    N, cap, heads, kv, width = 12, 700, 8, 2, 128
    p = api.attn_params(3, N, heads, kv, width, T_k=cap)
    rope, freq = api.rope_params(3, N, heads, kv, width), api.rope_frequencies(width)
    f, g = (api.lawcat_attn_tree_quant, api.lawcat_cache_accept_quant) if quant else (api.lawcat_attn_tree, api.lawcat_cache_accept)
    source = [draw((3, N, heads, width), 1, "bf16"), draw((3, N, kv, width), 2, "bf16"), draw((3, N, kv, width), 3, "bf16")]
    pos = torch.tensor([5, 650, 1400], dtype=torch.int32, device="cuda")
    up = torch.tensor([some_tree(N, 70 + b) for b in range(3)], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 1, -1], [0, -1, -1], [0, 2, 3]], dtype=torch.int32, device="cuda")
    if quant:
        past = list(api.quant_cache(p))
        rows = [draw((3, cap, kv, width), 4 + i, "bf16") for i in range(2)]
        api.lawcat_cache_quantize(api.attn_params(3, cap, heads, kv, width, T_k=cap), *rows, torch.zeros(3, dtype=torch.int32, device="cuda"), *past)
    else:
        past = [draw((3, cap, kv, width), 4 + i, "bf16") for i in range(2)]

    def step(q, k, v, cache, at, parent, way, stream, sync):
        done = torch.cuda.synchronize if sync else lambda: None
        qr, kr = api.lawcat_rope_fwd(rope, freq, q, k, start=at, parent=parent, stream=stream)
        done()
        o = f(p, qr, kr, v, *cache, at, parent=parent, stream=stream)
        done()
        end = g(p, kr, v, at, *cache, path=way, stream=stream)
        done()
        return [qr, kr, o, end, *cache]

    want = step(*source, [x.clone() for x in past], pos, up, path, None, True)
    blank = [torch.zeros_like(x) for x in (*source, pos, up, path, *past)]
    spin = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for again in range(3):
        for x in blank:
            x.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(10):
                spin @ spin
            for x, y in zip(blank, (*source, pos, up, path, *past)):
                x.copy_(y)
            got = step(*blank[:3], blank[6:], *blank[3:6], side if again else None, False)
        side.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@gpu
@pytest.mark.parametrize("dtype,exact", KINDS)
@pytest.mark.parametrize("packed", [False, True])
def test_a_training_step(packed, dtype, exact):
    """The gradients through attention and rotation. The rotation of a gradient that is off by e_u, e_w is off by less than e_u + e_w more."""
    batch, n, heads, kv, width, rot = 2, 150, 6, 2, 64, 48
    cu = [0, 37, 90, n] if packed else None
    freq = api.rope_frequencies(rot)
    p = api.attn_params(batch, n, heads, kv, width, dtype=dtype, causal=1, exact=exact)
    r = api.rope_params(batch, n, heads, kv, width, rot=rot, dtype=dtype)
    q, k, v, dO = (draw((batch, n, h, width), i, dtype) for i, h in enumerate((heads, kv, kv, heads)))
    row = list(range(n)) if cu is None else [t - max(x for x in cu[:-1] if x <= t) for t in range(n)]
    at = torch.tensor([row] * batch, dtype=torch.int32, device="cuda")
    if packed:
        p = api.attn_params(1, n, heads, kv, width, dtype=dtype, causal=1, exact=exact)
        r = api.rope_params(1, n, heads, kv, width, rot=rot, dtype=dtype)
        q, k, v, dO, at = (x[:1].contiguous() for x in (q, k, v, dO, at))
    qr, kr = api.lawcat_rope_fwd(r, freq, q, k, positions=at)
    out = U16 if dtype == "bf16" else U32
    for x, y in ((q, qr), (k, kr)):
        want, err = turned(x, at.cpu(), freq, rot, "half", 1.0, 1)
        check(y, want, err, out, "turned")
    a = api.lawcat_attn_fwd(p, qr, kr, v, cu_seqlens=cu)
    g = api.lawcat_attn_bwd(p, qr, kr, v, a["o"], a["lse"], dO, cu_seqlens=cu)
    dq, dk = api.lawcat_rope_bwd(r, freq, g["dq"], g["dk"], positions=at)
    ref = attention(qr, kr, v, visible(n, n, 1, 0, cu, None, p.B), float(torch.tensor(width ** -0.5)), 0.0, None, dO, a["o"])
    errs = ref["grad_err"](U16 if dtype == "bf16" and not exact else 0.0, out)
    for got, name in ((dq, "dq"), (dk, "dk")):
        want, err = turned(ref[name], at.cpu(), freq, rot, "half", 1.0, -1)
        e = errs[name] + out * 1.0001 * ref[name].abs()          # what is off before the rotation
        both = e.clone()
        both[..., :rot // 2] = both[..., rot // 2:rot] = e[..., :rot // 2] + e[..., rot // 2:rot]
        check(got, want, err + both * (1 + 2.0 ** -20) + out * both, out, name)
