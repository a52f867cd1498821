"""Slow decays over many steps: the factor that one step multiplies a state by is not a float, and its rounding, the same in every step,
must not add up.

Every entry of the state is multiplied once a step and rounded once a step, by 2^-24 of it at most; over n steps, whose roundings are
independent of each other and of the other entries' (the increments are random), the mean of the relative error over the state's 4096
entries has a standard deviation of (n / 3 / 4096)^(1/2) 2^-24.  A factor off by r 2^-24 shifts that mean by n r 2^-24."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 64


def decay(tokens):
    """A log decay of about -1e-5 whose power over so many tokens lies between two floats: at least 0.4 of 2^-24 from the nearest."""
    a = np.float32(-1e-5)
    while True:
        f = math.exp(float(a) * tokens)
        off = (f - float(np.float32(f))) * 2.0 ** 24
        if abs(off) >= 0.4:
            return float(a), off
        a = np.nextafter(a, np.float32(-1))


def shift(got, ref):
    """The mean relative error, weighted by the entries' squares."""
    return float(((got.double() - ref) * ref).sum() / (ref * ref).sum())


@pytest.mark.parametrize("io,chunk", [(torch.float32, 32), (torch.bfloat16, 64)])
def test_prompts_of_many_segments(io, chunk):
    """One head of 64 channels: 1024 segments of two chunks.  k and v stop after the first segment, so that the end state is
    a power of the decay times what that left; the other segments add nothing."""
    import paper_2605_09877_amd as kvm
    seg = 2 * chunk
    T = 1024 * seg
    a, off = decay(seg)
    gen = torch.Generator(DEV).manual_seed(1)
    q, k, v = (torch.zeros(1, T, 1, D, dtype=io, device=DEV) for _ in range(3))
    for t in (k, v):
        t[:, :seg] = torch.randn(1, seg, 1, D, generator=gen, device=DEV).to(io)
    q[:, -1] = torch.randn(1, 1, D, generator=gen, device=DEV).to(io)
    out, end = kvm.linear_prefill(q, k, v, torch.tensor([a], device=DEV))
    w = torch.exp(a * torch.arange(T - 1, T - 1 - seg, -1, dtype=torch.float64, device=DEV))
    ref = (k[0, :seg, 0].double() * w[:, None]).T.contiguous() @ v[0, :seg, 0].double()
    # 1023 steps that add nothing: no increments make the roundings independent of each other here, but those of the entries are.
    # One entry's add up to 1023 2^-24 at most; the mean of 4096 has a deviation of that / 3^(1/2) / 64.  The first
    # segment's own sums: 8 roundings of powers and operands, common to all entries at worst.
    tol = (5 * 1023 / 3 ** 0.5 / 64 + 8) * 2.0 ** -24
    assert 1023 * abs(off) * 2.0 ** -24 > 3 * tol
    assert abs(shift(end[0, 0], ref)) <= tol
    want = (q[0, -1, 0].double() @ ref) / D ** 0.5
    mag = (q[0, -1, 0].double().abs() @ ref.abs()) / D ** 0.5
    e = 2.0 ** -8 + 2.0 ** -7 if io is torch.bfloat16 else (2 * D + 2 * 1024) * 2.0 ** -24
    assert torch.all((out[0, -1, 0].double() - want).abs() <= e * mag)


@pytest.mark.parametrize("B", [1, 600])   # (both arrangements of units)
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
def test_single_tokens(io, B):
    import paper_2605_09877_amd as kvm
    a, off = decay(1)
    n = 2000
    gen = torch.Generator(DEV).manual_seed(2)
    state = torch.randn(1, 1, D, D, generator=gen, device=DEV).repeat(B, 1, 1, 1)
    k, v = ((torch.randn(n, 1, 1, D, generator=gen, device=DEV) / 16).to(io) for _ in range(2))
    q = torch.zeros(B, 1, D, dtype=io, device=DEV)
    ref, lam, ld = state[0, 0].double(), math.exp(a), torch.tensor([a], device=DEV)
    out = torch.empty_like(q)
    for t in range(n):
        kt, vt = k[t].expand(B, 1, D).contiguous(), v[t].expand(B, 1, D).contiguous()
        kvm.linear_decode(state, q, kt, vt, ld, out=out)
        ref = lam * ref + k[t, 0, 0].double()[:, None] * v[t, 0, 0].double()[None]
    assert torch.equal(state, state[:1].expand_as(state))
    tol = 5 * (n / 3 / D ** 2) ** 0.5 * 2.0 ** -24 + 4 * 2.0 ** -24
    assert n / 2 * abs(off) * 2.0 ** -24 > 3 * tol
    assert abs(shift(state[0, 0], ref)) <= tol


def test_a_token_of_a_state_that_grows_beyond_fp32():
    """A log decay above 0 whose power is no float: infinities of the state's signs, as the product with one is."""
    import paper_2605_09877_amd as kvm
    state = torch.tensor([1.0, -2.0], device=DEV).repeat(D * D // 2).view(1, 1, D, D).contiguous()
    want = state * float("inf")
    zero = torch.zeros(1, 1, D, device=DEV)
    for a in (100.0, 1000.0):
        got = state.clone()
        kvm.linear_decode(got, zero, zero, zero, torch.tensor([a], device=DEV))
        assert torch.equal(got, want)
