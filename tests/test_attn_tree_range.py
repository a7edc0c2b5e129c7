"""Attention of drafted tokens over a 4-bit cache whose keys and values lie outside what the tensor cores' fp16 operands hold, against 64 bits.

Keys and values are held times 16 in fp16. A group of 32 channels (minimum m, scale s) that holds values beyond 65504 / 16 does not fit: rows that
see such a slot are computed in fp32, and so are their bounds here (no operand is rounded). The others round keys, values and weights by 2^-11 each.

Below, 16 s and 16 m are whole multiples of 2^-24 as bf16 numbers from 2^-21 on, so that fp16 holds them and, but for 2^-11 of it, the value. Of a
smaller one it holds the nearest such multiple: half a step for each of 15 scales, the minimum and the value, 17 2^-29 in all (ABS). For keys that is
a score's error of |scale| sum|q| 17 2^-29, and rows with |scale| sum|q| above 2^14 are computed in fp32; so are those whose outputs lie
below 2^-15 and that see values of the kind.

Weights are 2^7 times what they are relative to a score of the row, and whole multiples of 2^-24 below 2^-14: off by 2^-32 at most (MIN_P).
"""
import pytest
import torch

from attn_reference import U16, check, quantized
from paper_2509_18467_b200 import api
from test_attn import draw
from test_attn_decode import rows_of
from test_attn_tree import some_tree
from tree_reference import U11, sees, tree_attention

pytestmark = pytest.mark.gpu

FITS = 65504.0 / 16
MIN_P = 2.0 ** -32
# lengths that are whole segments, that are cut into pieces which the first one's block joins, and that a second kernel joins
LENGTHS = {"whole": ([300, 11, 0], 400), "cut": ([1500] * 24, 1600), "few": ([3000], 4000)}


def groups(x):
    """Scale and minimum of each group of the rows x [n, H_kv, d] as the cache holds them."""
    _, scale, low, _ = quantized(x)
    return scale, low


def cached_groups(cache, which, b, slots):
    pr = cache[which][b][:, slots].double().transpose(0, 1)
    return pr[..., 0], pr[..., 1]


def too_wide(scale, low):
    """[n, H_kv]: rows with a group that fp16 does not hold."""
    return ((low.abs() > FITS) | ((low + 15 * scale).abs() > FITS)).any(-1)


ABS = 17 * 2.0 ** -29


def too_small(scale, low):
    """[n, H_kv]: rows with a group whose scale or minimum fp16 may not hold."""
    return (((scale != 0) & (scale < 2.0 ** -21)) | ((low != 0) & (low.abs() < 2.0 ** -21))).any(-1)


def verify(q, k, v, K, V, pos, parents, cap=0.0, scale=None, slopes=None):
    """One call over the quantized K, V [B, C, H_kv, d]; every row within its bound."""
    B, N, H, d = q.shape
    C, H_kv = K.shape[1], K.shape[2]
    p = api.attn_params(B, N, H, H_kv, d, T_k=C, cap=cap, scale=scale)
    cache = api.quant_cache(p)
    api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), K, V, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
    at = torch.tensor(pos, dtype=torch.int32, device="cuda")
    up = torch.tensor(parents, dtype=torch.int32, device="cuda")
    o = api.lawcat_attn_tree_quant(p, q, k, v, *cache, at, parent=up, slopes=slopes)
    s = float(torch.tensor(d ** -0.5 if scale is None else scale))
    for b, x in enumerate(pos):
        cached, see, dist = sees(parents[b], x, C, 0)
        slots = torch.tensor(cached, dtype=torch.long, device="cuda") % C
        Kd, Vd = rows_of(cache, b, slots)
        keys, values = torch.cat([Kd, quantized(k[b])[3]]), torch.cat([Vd, quantized(v[b])[3]])
        seen = lambda x: (see.to("cuda")[:, :, None] & x[None]).any(1).repeat_interleave(H // H_kv, 1)[..., None]  # noqa: E731  [n, H_kv] -> [N, H, 1]
        wide = seen(torch.cat([too_wide(*cached_groups(cache, 1, b, slots)), too_wide(*groups(k[b]))]))
        fine_values = seen(torch.cat([too_small(*cached_groups(cache, 3, b, slots)), too_small(*groups(v[b]))]))
        reach = abs(s) * torch.where(see.any(1).to("cuda")[:, None, None], q[b].double(), 0.0).abs().sum(-1, keepdim=True)
        want, fine = tree_attention(q[b], keys, values, see, dist, s, cap, slopes)
        _, coarse = tree_attention(q[b], keys, values, see, dist, s, cap, slopes, eps_p=U11, eps_k=U11, eps_v=U11, min_p=MIN_P)
        size, _ = tree_attention(q[b], keys, values.abs(), see, dist, s, cap, slopes)
        coarse = coarse + 2 * ABS * reach * size + torch.where(fine_values & (want.abs().amax(-1, keepdim=True) > 0.98 * 2.0 ** -15), ABS, 0.0)
        check(o[b], want, torch.where(wide | (reach > 1.01 * 2.0 ** 14), fine, coarse), U16, f"o of sequence {b} at {x}")
    return o


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("N,d", [(5, 64), (5, 128), (40, 64), (40, 128)])
@pytest.mark.parametrize("where", ["some", "all", "nodes"])
@pytest.mark.parametrize("size", [4000.0, 5000.0, 60000.0])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_one_large_channel_of_the_keys(cap, size, where, N, d, lengths):
    """A channel of some cached keys, of all of them, or of the nodes' alone is +-size, and the queries' +-0.001: ordinary scores."""
    pos, C = LENGTHS[lengths]
    B, H, H_kv, c = len(pos), 8, 2, 5
    q, k, v = draw((B, N, H, d), N, "bf16", 1.5), draw((B, N, H_kv, d), N + 1, "bf16"), draw((B, N, H_kv, d), N + 2, "bf16")
    K, V = draw((B, C, H_kv, d), N + 3, "bf16"), draw((B, C, H_kv, d), N + 4, "bf16")
    sign = 1.0 - 2.0 * ((torch.arange(N)[:, None] + torch.arange(H)) % 2)
    q[..., c] = (1e-3 * sign).to(q)
    large = torch.tensor([size, -size]).to(K)
    if where == "some":
        K[:, ::7, :, c] = large
    elif where == "all":
        K[..., c] = large
    else:
        k[..., c] = large
    verify(q, k, v, K, V, pos, [some_tree(N, b) for b in range(B)], cap)


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("N,d", [(5, 64), (5, 128), (21, 128), (40, 64), (40, 128)])
@pytest.mark.parametrize("std", [1e-4, 3e-5, 1e-5, 4e-6, 1e-6, 1e-9, "some"])
def test_small_values(std, N, d, lengths):
    """All values small, or ("some") a group of each cached row and all of every third."""
    pos, C = LENGTHS[lengths]
    B, H, H_kv = len(pos), 8, 2
    q, k, v = draw((B, N, H, d), N, "bf16", 1.5), draw((B, N, H_kv, d), N + 1, "bf16"), draw((B, N, H_kv, d), N + 2, "bf16")
    K, V = draw((B, C, H_kv, d), N + 3, "bf16"), draw((B, C, H_kv, d), N + 4, "bf16")
    if std == "some":
        V[..., 32:] *= 1e-6
        V[:, ::3] *= 1e-5
    else:
        v *= std
        V *= std
    verify(q, k, v, K, V, pos, [some_tree(N, b) for b in range(B)])


@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("N,d", [(5, 64), (5, 128), (21, 128), (40, 64), (40, 128)])
@pytest.mark.parametrize("small,large", [(1e-5, 1e5), (1e-4, 1e4), (1e-7, 1e7), (1e-5, 300.0), (1e-4, 1e3)])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_small_keys_under_large_queries(cap, small, large, N, d, lengths):
    pos, C = LENGTHS[lengths]
    B, H, H_kv = len(pos), 8, 2
    q, k, v = draw((B, N, H, d), N, "bf16", large), draw((B, N, H_kv, d), N + 1, "bf16", small), draw((B, N, H_kv, d), N + 2, "bf16")
    K, V = draw((B, C, H_kv, d), N + 3, "bf16", small), draw((B, C, H_kv, d), N + 4, "bf16")
    verify(q, k, v, K, V, pos, [some_tree(N, b) for b in range(B)], cap)


@pytest.mark.parametrize("N", [3, 12, 20, 40])
@pytest.mark.parametrize("where", ["newest", "middle", "oldest"])
@pytest.mark.parametrize("B,d", [(1, 128), (24, 64)])
def test_a_sink(B, d, where, N):
    """One token holds all but 2^-12 of the weight and has next to no value; the others' weights are e^-18 of its own each."""
    n, C, H, H_kv = 16380, 16384, 8, 2
    full = lambda x, *s: torch.full(s, x, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, k, v = full(1.5, B, N, H, d), full(0.0, B, N, H_kv, d), full(0.5, B, N, H_kv, d)
    K, V = full(0.0, B, C, H_kv, d), full(0.5, B, C, H_kv, d)
    at = dict(newest=n - 1, middle=n // 2, oldest=0)[where]
    K[:, at], V[:, at] = 1.5, 1e-3
    verify(q, k, v, K, V, [n] * B, [some_tree(N, b) for b in range(B)], scale=18.0 / (2.25 * d))


@pytest.mark.parametrize("N", [5, 40])
def test_values_of_zero_take_no_longer(N):
    """A cache whose values are all zero (a warm-up, a head that is off): nothing is computed twice."""
    B, C, H, H_kv, d = 8, 8192, 8, 2, 128
    p = api.attn_params(B, N, H, H_kv, d, T_k=C)
    q, k, v = draw((B, N, H, d), 1, "bf16"), draw((B, N, H_kv, d), 2, "bf16"), draw((B, N, H_kv, d), 3, "bf16")
    K, V = draw((B, C, H_kv, d), 4, "bf16"), draw((B, C, H_kv, d), 5, "bf16")
    pos = torch.full((B,), 8000, dtype=torch.int32, device="cuda")
    times = []
    for f in (1.0, 0.0):
        cache = api.quant_cache(p)
        api.lawcat_cache_quantize(api.attn_params(B, C, H, H_kv, d, T_k=C), K, V * f, torch.zeros(B, dtype=torch.int32, device="cuda"), *cache)
        once = []
        for _ in range(5):
            t = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            t[0].record()
            o = api.lawcat_attn_tree_quant(p, q, k, v * f, *cache, pos)
            t[1].record()
            torch.cuda.synchronize()
            once.append(t[0].elapsed_time(t[1]))
        times.append(min(once))
        assert f or not o.any()
    assert times[1] < 5 * times[0] + 0.1       # (computed again it takes some hundred times as long)
