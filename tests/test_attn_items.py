"""Softmax attention where one block takes many items in turn: short and empty items behind one another, whose gradients leave while
the next ones' are being written down."""
import pytest
import torch

from attn_reference import U16, U32, attention, check, visible
from paper_2509_18467_b200 import api
from test_attn import draw


def gradients(p, q, k, v, dO):
    r = api.lawcat_attn_fwd(p, q, k, v)
    r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO))
    return r


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,T,T_k,H,H_kv,window", [
    (64, 1024, 128, 8, 2, 0),    # 128 queries with keys, then seven tiles of queries that see none: a block's later items are empty
    (40, 700, 65, 16, 16, 0),    # the same with a ragged end, one head per group
    (600, 64, 64, 4, 2, 0),      # one tile of keys per item
    (24, 1024, 1024, 8, 8, 3),   # two or three tiles of keys per item
])
def test_gradients_of_short_and_empty_items(B, T, T_k, H, H_kv, window, d):
    """Rows without a key have gradients of zero, the others are right, and the same call gives the same bits each time."""
    q, k, v, dO = [draw((B, n, h, d), i, "bf16") for i, (n, h) in enumerate(((T, H), (T_k, H_kv), (T_k, H_kv), (T, H)))]
    p = api.attn_params(B, T, H, H_kv, d, T_k=T_k, window=window)
    first = gradients(p, q, k, v, dO)
    none = max(0, T - T_k)
    for _ in range(8):
        r = gradients(p, q, k, v, dO)
        assert not r["dq"][:, :none].any()
        for n in first:
            assert torch.equal(r[n], first[n]), n
    for b in range(0, B, max(1, B // 6)):
        s = slice(b, b + 1)
        ref = attention(q[s], k[s], v[s], visible(T, T_k, 1, window), float(torch.tensor(d ** -0.5)), 0.0, None, dO[s], first["o"][s])
        err = dict(ref["grad_err"](U16, U16), o=ref["o_sum"] + U16 * ref["o_mag"], lse=ref["lse_err"])
        for n in ("o", "lse", "dq", "dk", "dv"):
            check(first[n][s], ref[n], err[n], U32 if n == "lse" else U16, f"{n} of sequence {b}")
