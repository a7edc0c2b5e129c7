"""Attention calls with a tensor on another device than the current one are refused by name before anything is launched: the launch would
go to the current device with the other one's addresses. (No GPU: the tensors have a device and sizes, no memory.)"""
import pytest
import torch

from paper_2509_18467_b200 import api, build


class Elsewhere(torch.Tensor):
    """A tensor that says it lies on the second GPU."""
    @staticmethod
    def __new__(cls, *sizes, dtype=torch.bfloat16):
        return torch.Tensor._make_wrapper_subclass(cls, sizes, dtype=dtype, device="cuda:1")

    @classmethod
    def __torch_dispatch__(cls, f, types, args=(), kw=None):
        raise NotImplementedError(str(f))


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()
    if torch.cuda.is_available() and torch.cuda.current_device() == 1:
        pytest.skip("the second GPU is the current one")


B, T, C, H, H_kv, d = 2, 8, 16, 4, 2, 64


def tensors(make):
    f32, i32, u8 = (dict(dtype=x) for x in (torch.float32, torch.int32, torch.uint8))
    return dict(q=make(B, T, H, d), k=make(B, T, H_kv, d), v=make(B, T, H_kv, d), o=make(B, T, H, d), lse=make(B, T, H, **f32), dO=make(B, T, H, d),
                slopes=make(H, **f32), q_t=make(B, H, d), k_t=make(B, H_kv, d), v_t=make(B, H_kv, d), K=make(B, C, H_kv, d), V=make(B, C, H_kv, d),
                pos=make(B, **i32), o_t=make(B, H, d), ws=make(1 << 16, **u8), dev_status=make(1, **i32),
                kq=make(B, H_kv, C, d // 2, **u8), kp=make(B, H_kv, C, d // 32, 2),
                vq=make(B, H_kv, C, d // 2, **u8), vp=make(B, H_kv, C, d // 32, 2))


STEP = ["q_t", "k_t", "v_t", "pos", "slopes", "o_t", "ws", "dev_status"]
CACHE = ["k", "v", "pos", "kq", "kp", "vq", "vp", "dev_status"]
CALLS = dict(lawcat_attn_fwd=["q", "k", "v", "slopes", "o", "ws", "dev_status"], lawcat_attn_bwd=["q", "k", "v", "o", "lse", "dO", "slopes", "ws", "dev_status"],
             lawcat_attn_decode=STEP + ["K", "V"], lawcat_attn_decode_quant=STEP + ["kq", "kp", "vq", "vp"],
             lawcat_cache_quantize=CACHE, lawcat_cache_dequantize=CACHE)


@pytest.mark.parametrize("name,arg", [(n, a) for n, args in CALLS.items() for a in args])
def test_a_tensor_on_another_device_is_refused(name, arg):
    step = "decode" in name
    p = api.attn_params(B, 1 if step else T, H, H_kv, d, T_k=C if step or "cache" in name else T)
    here, there = tensors(lambda *s, **kw: torch.zeros(*s, **{"dtype": torch.bfloat16, **kw})), tensors(Elsewhere)
    kw = {n: here[n] for n in CALLS[name]}
    kw[arg] = there[arg]
    with pytest.raises(ValueError, match=f"^{arg}: on device cuda:1"):
        getattr(api, name)(p, **kw)
