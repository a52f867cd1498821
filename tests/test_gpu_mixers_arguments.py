"""Calls of the mixers whose arguments have to be refused, or taken by their value; and tensors written by a call while autograd holds
them for a backward pass."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, T, HQ, HKV, D = 2, 40, 4, 2, 64


def inputs(io=torch.float32, seed=0):
    gen = torch.Generator(DEV).manual_seed(seed)
    rnd = lambda *s, dt=io: torch.randn(*s, generator=gen, device=DEV).to(dt)
    return dict(q=rnd(B, T, HQ, D), k=rnd(B, T, HKV, D), v=rnd(B, T, HKV, D), dout=rnd(B, T, HQ, D),
                state=rnd(B, HKV, D, D, dt=torch.float32), ld=torch.tensor([-0.02, -0.3], device=DEV))


def token(x, t=0):
    return [x[n][:, t].contiguous() for n in "qkv"]


@pytest.mark.parametrize("scale", [0.0, -0.0, 0, 1e-50, 1e-40, 1e50, float("inf"), float("nan"), -1.0, torch.tensor(0.0)], ids=str)
def test_scales_that_are_refused(scale):
    """None selects 1 / sqrt(d), 0 does not: nothing but positive numbers that fp32 holds, with reciprocals that it holds."""
    import paper_2605_09877_amd as kvm
    x = inputs()
    qkv, ck = [x[n] for n in "qkv"], kvm.window_cache(B, HKV, D, window=8, dtype=torch.float32, device=DEV)
    pos, lse = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, T, HQ, device=DEV)
    for call in (lambda: kvm.window_prefill(*qkv, window=8, scale=scale), lambda: kvm.kvm_window_attention(*qkv, window=8, scale=scale),
                 lambda: kvm.window_backward(*qkv, x["q"], lse, x["dout"], window=8, scale=scale),
                 lambda: kvm.window_decode(*ck, *token(x), pos, window=8, scale=scale),
                 lambda: kvm.linear_prefill(*qkv, x["ld"], scale=scale), lambda: kvm.kvm_linear_attention(*qkv, x["ld"], scale=scale),
                 lambda: kvm.linear_backward(*qkv, x["ld"], x["dout"], scale=scale),
                 lambda: kvm.linear_decode(x["state"], *token(x), x["ld"], scale=scale)):
        with pytest.raises(ValueError, match="scale"):
            call()
