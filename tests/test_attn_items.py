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


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_the_bound_on_waits_is_not_one_on_an_item(d):
    """Under a bound of 400000 clock cycles, a hundred times what a step takes and a small part of an item of 2200 tiles: a block whose
    roles all go on is not one that has lost something, however long its item. (Which roles wait for an item's end depends on its
    length alone: with the bound's usual value the same goes for items of some million tiles.)"""
    T, H = 140001, 2
    q, k, v, dO = [draw((1, T, h, d), i, "bf16") for i, h in enumerate((H, 1, 1, H))]
    p = api.attn_params(1, T, H, 1, d)
    want = gradients(p, q, k, v, dO)
    torch.cuda.synchronize()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.test_set_wait_limit(400000)
    try:
        r = api.lawcat_attn_fwd(p, q, k, v, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0, "forward"
        r.update(api.lawcat_attn_bwd(p, q, k, v, r["o"], r["lse"], dO, dev_status=status))
        torch.cuda.synchronize()
        assert int(status.item()) == 0, "gradients"
    finally:
        api.test_set_wait_limit(0)
    for n in want:
        assert torch.equal(r[n], want[n]), n
