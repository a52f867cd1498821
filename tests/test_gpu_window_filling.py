"""Window prompts whose workgroups fill the device in rows longer than those that take P as two operands: the kernel behind large
bf16 prompts (132 sequences of four KV heads: 1584 workgroups of 128 queries; 70 of eight heads on two: 1400 of 32 queries of
four heads; the waves share key tiles below 512 and 256).  The bounds are those of test_gpu_window."""
import numpy as np
import pytest
import torch

from oracle import mixers_oracle as mo
from test_gpu_window import DEV, DT, f64, make, noise, out_bound, run_case, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io,d,B,Hq,Hkv", [("bf16", 128, 132, 4, 4), ("bf16", 64, 132, 4, 4), ("bf16", 128, 70, 8, 2), ("bf16", 64, 70, 8, 2),
                                           ("bf16", 64, 70, 6, 2), ("f32", 64, 132, 4, 4), ("f32", 128, 70, 8, 2)])
@pytest.mark.parametrize("T,W,S", [(300, 100, 3), (261, 62, 5), (300, 299, 0)])
def test_long_rows(io, d, B, Hq, Hkv, T, W, S):
    """Lengths of all kinds, four of the sequences compared: out with and without lse, lse, all gradients."""
    import paper_2605_09877_amd as kvm
    x = make(io, B, T, T, Hq, Hkv, d, seed=2)
    lens = [(37 * b) % (T + 1) for b in range(B)]
    lens[0], lens[B // 3], lens[B // 2], lens[B - 1] = T, 257, 129, 0
    kw = dict(window=W, n_sink=S, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    leaves = [x[n].clone().requires_grad_() for n in "qkv"]
    o = kvm.kvm_window_attention(*leaves, **kw)
    grads = torch.autograd.grad(o, leaves, x["dout"])
    _, lse = kvm.window_prefill(x["q"], x["k"], x["v"], want_lse=True, **kw)
    plain = kvm.window_prefill(x["q"], x["k"], x["v"], **kw)
    for b in (0, B // 3, B // 2, B - 1):
        one = {n: t[b:b + 1] for n, t in x.items()}
        y = {n: f64(t) for n, t in one.items()}
        ref, rlse = mo.window(y["q"], y["k"], y["v"], W, S, [lens[b]])
        tol = out_bound(io, one, ref, W, S, [lens[b]], None)
        within(o[b:b + 1], ref, tol, f"out {b}")
        within(plain[b:b + 1], ref, tol, f"out without lse {b}")
        got, live = f64(lse[b:b + 1]), np.isfinite(rlse)
        assert np.array_equal(live, np.isfinite(got)) and np.all(got[~live] == -np.inf)
        e = (2.0 ** -8 if io == "bf16" else 0) + noise(one, None, T) * (2 + np.abs(rlse[live]).max(initial=0))
        assert np.all(np.abs(got[live] - rlse[live]) <= e), f"lse {b}"
        rg = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], W, S, [lens[b]])
        mg = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], W, S, [lens[b]], absolute=True)
        e = noise(one, None, T * (Hq // Hkv)) + (2 * 2.0 ** -8 + 2.0 ** -14 if io == "bf16" else 0)
        for got, r, m, name in zip(grads, rg, mg, ("dq", "dk", "dv")):
            within(got[b:b + 1], r, e * m + (2.0 ** -8 * np.abs(r) if io == "bf16" else 0), f"{name} {b}")
    for b, n in enumerate(lens):
        for t in (o, plain, *grads):
            assert torch.count_nonzero(t[b, n:]) == 0


@pytest.mark.parametrize("io,d,step", [("bf16", 128, 0.02), ("bf16", 128, 0.5), ("bf16", 64, 0.5), ("bf16", 64, -0.3), ("f32", 64, 0.1)])
def test_maxima_that_rise_or_fall_along_the_keys(io, d, step):
    """A logit of about step for every key: the reference of the exponentials moves often, seldom, or never again."""
    import paper_2605_09877_amd as kvm
    B, T, W, S = 132, 300, 250, 2
    x = make(io, 1, T, T, 4, 4, d, seed=3)
    x["q"] = (1 + 0.1 * x["q"].float()).to(DT[io])
    x["k"] = (step * d ** -0.5 * torch.arange(T, device=DEV).view(1, T, 1, 1) + 0.05 * x["k"].float()).to(DT[io])
    y = {n: f64(t) for n, t in x.items()}
    ref = mo.window(y["q"], y["k"], y["v"], W, S)[0]
    tol = out_bound(io, x, ref, W, S, None, None)
    many = [x[m].repeat(B, 1, 1, 1) for m in "qkv"]
    for out in (kvm.window_prefill(*many, window=W, n_sink=S), kvm.window_prefill(*many, window=W, n_sink=S, want_lse=True)[0]):
        within(out[:1], ref, tol, "out")
        assert torch.equal(out, out[:1].expand_as(out))


@pytest.mark.parametrize("io,d", [("bf16", 64), ("bf16", 128), ("f32", 128)])
@pytest.mark.parametrize("B,T,Hq,Hkv", [(64, 120, 1, 1), (100, 160, 1, 1), (66, 33, 4, 1)])
def test_many_short_rows(io, d, B, T, Hq, Hkv):
    """Either side of the rule for 64 units and more: waves that share key tiles, and that do not (520 workgroups, a group's heads)."""
    run_case(io, B, T, Hq, Hkv, d, window=50, n_sink=2, lens=[(23 * b) % (T + 1) for b in range(B - 1)] + [T])
