"""Linear attention with decay against the token-by-token recurrence in fp64: prompts, gradients, single tokens.

Bounds, element by element.  Every result is a sum of products with positive weights (powers of the decay), so the same sum
over absolute values bounds what roundings can do to it.  bf16: the result is rounded once (2^-8 of it), the products of
pairs inside a chunk once (2^-8 of the sum of absolute values), and the state's operands have 16 bits (2^-16 of it, twice).
fp32 sums, in either type: each of the at most 2 d + 2 T terms and steps that a value goes through adds 2^-24 of it."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import mixers_oracle as mo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return None if t is None else t.detach().to("cpu", torch.float64).numpy()


def make(io, B, T, Hq, Hkv, d, seed=0, carried=True, slow=8.0):
    gen = torch.Generator(DEV).manual_seed(1000 * seed + 7 * T + d)
    rnd = lambda *s, dt=DT[io]: torch.randn(*s, generator=gen, device=DEV).to(dt)
    x = dict(q=rnd(B, T, Hq, d), k=rnd(B, T, Hkv, d), v=rnd(B, T, Hkv, d), dout=rnd(B, T, Hq, d))
    x["state"] = rnd(B, Hkv, d, d, dt=torch.float32) if carried else None
    x["dstate"] = rnd(B, Hkv, d, d, dt=torch.float32) if carried else None
    x["log_decay"] = torch.log1p(-(2.0 ** -torch.linspace(1, slow, Hkv, dtype=torch.float64))).float().to(DEV)
    return x


def bound(io, ref, mag, d, T):
    steps = (2 * d + 2 * T + 64) * 2.0 ** -24
    return (2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -15 + steps) * mag if io == "bf16" else steps * mag) + 1e-30


def check(io, got, ref, mag, d, T, name):
    got = f64(got)
    assert got.shape == ref.shape, name
    bad = np.abs(got - ref) - bound(io, ref, mag, d, T)
    assert np.all(np.isfinite(got)) and bad.max() <= 0, (name, bad.max(), np.unravel_index(bad.argmax(), bad.shape))


def magnitudes(x, lens, scale):
    a = {n: None if t is None else np.abs(f64(t)) for n, t in x.items() if n != "log_decay"}
    ld = f64(x["log_decay"])
    out, st = mo.linear(a["q"], a["k"], a["v"], ld, a["state"], lens, scale)
    grads = mo.linear_backward(a["q"], a["k"], a["v"], ld, a["dout"], a["state"], a["dstate"], lens, scale)
    return (out, st, *grads)


def run_case(io, B, T, Hq, Hkv, d, lens=None, carried=True, scale=None, seed=0, slow=8.0):
    import paper_2605_09877_amd as kvm
    x = make(io, B, T, Hq, Hkv, d, seed, carried, slow)
    ld = f64(x["log_decay"])
    y = {n: f64(t) for n, t in x.items()}
    ref = (*mo.linear(y["q"], y["k"], y["v"], ld, y["state"], lens, scale),
           *mo.linear_backward(y["q"], y["k"], y["v"], ld, y["dout"], y["state"], y["dstate"], lens, scale))
    mag = magnitudes(x, lens, scale)
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    leaves = [x[n].clone().requires_grad_() for n in ("q", "k", "v")]
    start = x["state"].clone().requires_grad_() if carried else None
    out, st = kvm.kvm_linear_attention(*leaves, x["log_decay"], state=start, lens=dl, scale=scale)
    if carried:
        grads = torch.autograd.grad((out, st), (*leaves, start), (x["dout"], x["dstate"]))
    else:
        grads = torch.autograd.grad(out, leaves, x["dout"])
    # (the state's gradient passes no products inside a chunk, and is fp32 like the state)
    for i, (got, name) in enumerate(zip((out, st, *grads), ("out", "state", "dq", "dk", "dv", "dstate"))):
        check("f32" if name in ("state", "dstate") else io, got, ref[i], mag[i], d, T, name)
    # rows behind a sequence are zero to the bit
    if lens is not None:
        for b, n in enumerate(lens):
            for t in (out, *grads[:3]):
                assert torch.count_nonzero(t[b, max(n, 0):]) == 0
    return x, out, st


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 130, 200])
def test_lengths_about_the_chunk(io, d, T):
    run_case(io, 1, T, 2, 1, d)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (6, 2), (8, 1), (5, 5)])
def test_shared_and_odd_heads(io, Hq, Hkv):
    run_case(io, 2, 97, Hq, Hkv, 64, carried=False)


@pytest.mark.parametrize("io,d", [("bf16", 128), ("f32", 64), ("bf16", 64), ("f32", 128)])
def test_padded_batch_with_empty_sequences(io, d):
    run_case(io, 5, 150, 4, 2, d, lens=[0, 150, 1, 64, 129])


@pytest.mark.parametrize("io,d", [("bf16", 128), ("f32", 64)])
def test_long_enough_to_be_cut_into_segments(io, d):
    """Segments of at least 8 chunks, ends inside the first, on a border and in the last."""
    T = 64 * 8 * 3 + 17 if io == "bf16" else 32 * 8 * 4 + 5
    edge = 64 * 13 if io == "bf16" else 32 * 9
    run_case(io, 4, T, 2, 1, d, lens=[T, edge, 3, T - 18], slow=12.0)


def test_scale_and_strong_and_no_decay():
    run_case("f32", 1, 100, 2, 2, 64, scale=0.37)
    import paper_2605_09877_amd as kvm
    x = make("f32", 1, 100, 2, 2, 64)
    for a in (0.0, -1e-3, -3.0, -60.0):   # the last: nothing but the own token is left
        ld = torch.full((2,), a, device=DEV)
        out, st = kvm.linear_prefill(x["q"], x["k"], x["v"], ld, state=x["state"])
        ref = mo.linear(f64(x["q"]), f64(x["k"]), f64(x["v"]), f64(ld), f64(x["state"]))
        mag = mo.linear(*[np.abs(f64(x[n])) for n in "qkv"], f64(ld), np.abs(f64(x["state"])))
        check("f32", out, ref[0], mag[0], 64, 100, "out")
        check("f32", st, ref[1], mag[1], 64, 100, "state")


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_views_of_a_fused_projection(io):
    """q, k and v as slices of one buffer, out into a slice of another; nothing around it is written."""
    import paper_2605_09877_amd as kvm
    B, T, Hq, Hkv, d = 2, 75, 4, 2, 64
    x = make(io, B, T, Hq, Hkv, d)
    fused = torch.cat([x["q"], x["k"], x["v"]], dim=2)
    wide = torch.full((B, T, Hq + 3, d), 7.0, device=DEV, dtype=DT[io])
    want, wst = kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"], state=x["state"])
    got, st = kvm.linear_prefill(fused[:, :, :Hq], fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:], x["log_decay"],
                                 state=x["state"], out=wide[:, :, 1:1 + Hq])
    assert torch.equal(got, want) and torch.equal(st, wst)
    assert bool((wide[:, :, 0] == 7).all()) and bool((wide[:, :, 1 + Hq:] == 7).all())


@pytest.mark.parametrize("io,d,G", [("bf16", 128, 1), ("bf16", 64, 4), ("f32", 128, 11), ("f32", 64, 2)])
@pytest.mark.parametrize("B", [1, 3, 600])
def test_tokens_one_by_one(io, d, G, B):
    """Decode steps against the recurrence (600 sequences: the arrangement of many units), idle sequences left alone."""
    import paper_2605_09877_amd as kvm
    Hkv, steps = 1, 3
    x = make(io, B, steps, Hkv * G, Hkv, d)
    n = min(B, 5)
    active = torch.ones(B, dtype=torch.int32, device=DEV)
    if B > 1:
        active[1] = 0
    state = x["state"].clone()
    y = {m: f64(None if t is None or m == "log_decay" else t[:n]) for m, t in x.items()}
    y["log_decay"] = f64(x["log_decay"])
    lens = [steps if a else 0 for a in active[:n].tolist()]
    ref, rst = mo.linear(y["q"], y["k"], y["v"], y["log_decay"], y["state"], lens)
    mag, mst = mo.linear(*[np.abs(y[m]) for m in "qkv"], y["log_decay"], np.abs(y["state"]), lens)
    for t in range(steps):
        out = kvm.linear_decode(state, x["q"][:, t].contiguous(), x["k"][:, t].contiguous(), x["v"][:, t].contiguous(),
                                x["log_decay"], active=active)
        check(io, out[:n], ref[:, t], mag[:, t], d, steps, "out")
    check("f32", state[:n], rst, mst, d, steps, "state")
    if B > 1:
        assert torch.equal(state[1], x["state"][1]) and torch.count_nonzero(out[1]) == 0


def test_prompt_in_pieces_then_tokens_is_one_prompt():
    import paper_2605_09877_amd as kvm
    B, T, Hq, Hkv, d = 2, 200, 4, 2, 64
    x = make("f32", B, T, Hq, Hkv, d)
    want, wst = kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"])
    outs, st = [], None
    for t0, t1 in ((0, 37), (37, 38), (38, 190)):
        o, st = kvm.linear_prefill(*[x[n][:, t0:t1] for n in "qkv"], x["log_decay"], state=st, state_out=st)
        outs.append(o)
    for t in range(190, T):
        outs.append(kvm.linear_decode(st, *[x[n][:, t].contiguous() for n in "qkv"], x["log_decay"])[:, None])
    mag, mst = mo.linear(*[np.abs(f64(x[n])) for n in "qkv"], f64(x["log_decay"]))
    check("f32", torch.cat(outs, dim=1), f64(want), 2 * mag, d, T, "out")
    check("f32", st, f64(wst), 2 * mst, d, T, "state")


@pytest.mark.parametrize("io,d", [("bf16", 128), ("f32", 64)])
def test_padding_may_hold_anything(io, d):
    """NaN and infinities behind a sequence's end reach nothing."""
    import paper_2605_09877_amd as kvm
    x = make(io, 3, 140, 2, 1, d)
    lens = torch.tensor([0, 70, 139], dtype=torch.int32, device=DEV)
    args = dict(state=x["state"], lens=lens)
    want = kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"], **args)
    gwant = kvm.linear_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], dstate_out=x["dstate"], want_dstate=True, **args)
    for b, n in enumerate(lens.tolist()):
        for i, name in enumerate(("q", "k", "v", "dout")):
            x[name][b, n:] = float("nan") if i % 2 else float("inf")
    got = kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"], **args)
    ggot = kvm.linear_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], dstate_out=x["dstate"], want_dstate=True, **args)
    for a, b in zip((*want, *gwant), (*got, *ggot)):
        assert torch.equal(a, b)


def test_same_call_same_bits_and_other_streams():
    import paper_2605_09877_amd as kvm
    x = make("bf16", 2, 700, 4, 2, 128)
    want = kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"], state=x["state"])
    gwant = kvm.linear_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], state=x["state"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"], state=x["state"])
        ggot = kvm.linear_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], state=x["state"])
    side.synchronize()
    for a, b in zip((*want, *gwant[:3]), (*got, *ggot[:3])):
        assert torch.equal(a, b)


def test_captured_prompt_gradient_and_token():
    import paper_2605_09877_amd as kvm
    x = make("bf16", 1, 1100, 4, 2, 128)
    tok = [x[n][:, 5].contiguous() for n in "qkv"]

    def work(st):
        out, end = kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"], state=x["state"])
        g = kvm.linear_backward(x["q"], x["k"], x["v"], x["log_decay"], x["dout"], state=x["state"], want_dstate=True)
        st.copy_(x["state"])
        return (out, end, *g, kvm.linear_decode(st, *tok, x["log_decay"]), st)

    want = [t.clone() for t in work(torch.empty_like(x["state"]))]
    torch.cuda.synchronize()
    st = torch.empty_like(x["state"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(st)
    for _ in range(3):
        for t in got:
            t.zero_()
        kvm.linear_prefill(x["k"].repeat(1, 1, 2, 1), x["k"], x["v"], x["log_decay"])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)


def test_gradient_is_the_slope():
    """Directional differences of the loss in fp32: central, in a direction of every input at once.  The loss is linear in q and
    in dout, and its third-order term is e^2 of the direction's, so what is left is the rounding of two losses."""
    import paper_2605_09877_amd as kvm
    x = make("f32", 2, 90, 4, 2, 64)
    gen = torch.Generator(DEV).manual_seed(5)
    ins = [x["q"], x["k"], x["v"], x["state"]]
    dirs = [torch.randn(t.shape, generator=gen, device=DEV) for t in ins]
    eps = 2.0 ** -9

    def loss(sign):
        q, k, v, s = [t + sign * eps * u for t, u in zip(ins, dirs)]
        out, st = kvm.linear_prefill(q, k, v, x["log_decay"], state=s)
        return (out.double() * x["dout"].double()).sum() + (st.double() * x["dstate"].double()).sum()

    leaves = [t.clone().requires_grad_() for t in ins]
    out, st = kvm.kvm_linear_attention(*leaves[:3], x["log_decay"], state=leaves[3])
    grads = torch.autograd.grad((out, st), leaves, (x["dout"], x["dstate"]))
    slope = sum((g.double() * u.double()).sum() for g, u in zip(grads, dirs))
    diff = (loss(1) - loss(-1)) / (2 * eps)
    size = sum((g.double() * u.double()).abs().sum() for g, u in zip(grads, dirs))
    assert abs(slope - diff) <= 1e-3 * size


def test_refusals_by_the_binding():
    import paper_2605_09877_amd as kvm
    x = make("bf16", 2, 8, 4, 2, 64)
    ok = (x["q"], x["k"], x["v"], x["log_decay"])
    for bad in (dict(lens=torch.tensor([8, 8], device=DEV)), dict(state=x["state"].bfloat16()), dict(state=x["state"][:1]),
                dict(out=torch.empty_like(x["q"]).transpose(1, 2)), dict(scale=-1.0)):
        with pytest.raises((ValueError, kvm.KVMError)):
            kvm.linear_prefill(*ok, **bad)
    with pytest.raises(ValueError):
        kvm.linear_prefill(x["q"], x["k"].float(), x["v"], x["log_decay"])
    with pytest.raises(ValueError):
        kvm.linear_prefill(x["q"].half(), x["k"].half(), x["v"].half(), x["log_decay"])
    with pytest.raises(ValueError):
        kvm.linear_prefill(x["q"][:, :, :3], x["k"], x["v"], x["log_decay"])
    with pytest.raises(ValueError):
        kvm.linear_prefill(x["q"][:, :0], x["k"][:, :0], x["v"][:, :0], x["log_decay"])
    with pytest.raises(ValueError):
        kvm.kvm_linear_attention(x["q"], x["k"], x["v"], x["log_decay"].clone().requires_grad_())
    with pytest.raises(kvm.KVMError):   # rows that start off a 16-byte border
        wide = torch.zeros(2, 8, 4, 70, dtype=torch.bfloat16, device=DEV)
        kvm.linear_prefill(wide[..., 1:65], x["k"], x["v"], x["log_decay"])


def test_gradients_of_gradients_are_refused_and_a_graph_can_be_used_twice():
    import paper_2605_09877_amd as kvm
    x = make("f32", 1, 40, 2, 1, 64)
    leaves = [x[n].clone().requires_grad_() for n in "qkv"]
    out = kvm.kvm_linear_attention(*leaves, x["log_decay"])[0]
    first = torch.autograd.grad(out, leaves, x["dout"], retain_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(out, leaves, x["dout"], retain_graph=True, create_graph=True)
    for a, b in zip(first, torch.autograd.grad(out, leaves, x["dout"])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("io,d,B,Hq,Hkv", [("bf16", 128, 140, 8, 4), ("bf16", 64, 140, 4, 2), ("f32", 128, 140, 4, 4)])
def test_many_sequences(io, d, B, Hq, Hkv):
    """Units enough to fill the device without cutting sequences or sharing heads; a few of the sequences compared."""
    import paper_2605_09877_amd as kvm
    T = 330
    x = make(io, B, T, Hq, Hkv, d, slow=10.0)
    lens = [(11 * b) % (T + 1) for b in range(B)]
    lens[0], lens[B // 2], lens[B - 1] = T, 129, 64
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    leaves = [x[n].clone().requires_grad_() for n in ("q", "k", "v", "state")]
    out, st = kvm.kvm_linear_attention(*leaves[:3], x["log_decay"], state=leaves[3], lens=dl)
    grads = torch.autograd.grad((out, st), leaves, (x["dout"], x["dstate"]))
    ld = f64(x["log_decay"])
    for b in (0, B // 2, B - 1):
        one = {n: t if n == "log_decay" else t[b:b + 1] for n, t in x.items()}
        y = {n: f64(t) for n, t in one.items()}
        ref = (*mo.linear(y["q"], y["k"], y["v"], ld, y["state"], [lens[b]]),
               *mo.linear_backward(y["q"], y["k"], y["v"], ld, y["dout"], y["state"], y["dstate"], [lens[b]]))
        mag = magnitudes(one, [lens[b]], None)
        for i, (got, name) in enumerate(zip((out, st, *grads), ("out", "state", "dq", "dk", "dv", "dstate"))):
            check("f32" if name in ("state", "dstate") else io, got[b:b + 1], ref[i], mag[i], d, T, f"{name} {b}")


@pytest.mark.parametrize("io,G", [("bf16", 6), ("f32", 4), ("bf16", 7)])
def test_heads_shared_among_workgroups_and_single_chunk_segments(io, G):
    """One unit, many query heads: as many workgroups as divide the group walk its state, each cut chunk by chunk."""
    run_case(io, 1, 64 * 9 + 5 if io == "bf16" else 32 * 7 + 3, G, 1, 128, slow=9.0)


def test_backward_with_and_without_what_the_prompt_kept():
    import paper_2605_09877_amd as kvm
    x = make("bf16", 1, 1500, 2, 1, 128)
    keep = []
    kvm.linear_prefill(x["q"], x["k"], x["v"], x["log_decay"], state=x["state"], keep=keep)
    held = keep[0].clone()
    args = (x["q"], x["k"], x["v"], x["log_decay"], x["dout"])
    a = kvm.linear_backward(*args, state=x["state"], kept=keep[0], want_dstate=True)
    b = kvm.linear_backward(*args, state=x["state"], want_dstate=True)
    assert torch.equal(keep[0], held)   # read alone
    # (without it the states that dq starts from are made of 16 bits of every decayed value, not of 24)
    for p, q in zip(a[1:], b[1:]):
        assert torch.equal(p, q)
    mag = magnitudes({n: t for n, t in x.items() if n != "dstate"} | {"dstate": None}, None, None)[2]
    assert np.all(np.abs(f64(a[0]) - f64(b[0])) <= 2.0 ** -7 * np.abs(f64(a[0])) + 2.0 ** -14 * mag)
    with pytest.raises(ValueError):
        kvm.linear_backward(*args, kept=keep[0][:-256])


@pytest.mark.parametrize("io,B,T,Hq,Hkv,d", [
    ("bf16", 1, 130, 8, 1, 128), ("bf16", 2, 4000, 8, 2, 128), ("bf16", 40, 1030, 4, 4, 64), ("f32", 1, 300, 6, 2, 64)])
def test_state_given_back_in_place(io, B, T, Hq, Hkv, d):
    """state_out is the state the call starts from: its readers are not the workgroups that write it."""
    import paper_2605_09877_amd as kvm
    x = make(io, B, T, Hq, Hkv, d, slow=8.0)
    lens = torch.tensor([T - (b * 37) % T for b in range(B)], dtype=torch.int32, device=DEV)
    if B > 1:
        lens[1] = 0
    a = (x["q"], x["k"], x["v"], x["log_decay"])
    out, end = kvm.linear_prefill(*a, state=x["state"], lens=lens)
    st = x["state"].clone()
    out2, end2 = kvm.linear_prefill(*a, state=st, lens=lens, state_out=st)
    assert end2 is st and torch.equal(out, out2) and torch.equal(end, st)


def test_scale_by_value():
    import paper_2605_09877_amd as kvm
    x = make("f32", 1, 40, 1, 1, 64)
    a = (x["q"], x["k"], x["v"], x["log_decay"])
    scale = torch.tensor(0.5)
    half = kvm.linear_prefill(*a, scale=scale)[0]
    scale.fill_(0.25)
    assert torch.equal(half, 2 * kvm.linear_prefill(*a, scale=scale)[0])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_a_decay_that_keeps_nothing(io):
    """log_decay = -infinity for one head: out_t = scale (q_t . k_t) v_t there, and nothing of the start state."""
    import paper_2605_09877_amd as kvm
    B, T, d = 1, 700, 64
    x = make(io, B, T, 2, 2, d)
    ld = torch.tensor([-float("inf"), -0.1], device=DEV)
    leaves = [x[n].clone().requires_grad_() for n in ("q", "k", "v", "state")]
    out, st = kvm.kvm_linear_attention(*leaves[:3], ld, state=leaves[3])
    grads = torch.autograd.grad((out, st), leaves, (x["dout"], x["dstate"]))
    y = {n: f64(t) for n, t in x.items()}
    ref = (*mo.linear(y["q"], y["k"], y["v"], f64(ld), y["state"]),
           *mo.linear_backward(y["q"], y["k"], y["v"], f64(ld), y["dout"], y["state"], y["dstate"]))
    mag = magnitudes(dict(x, log_decay=ld), None, None)
    for i, (got, name) in enumerate(zip((out, st, *grads), ("out", "state", "dq", "dk", "dv", "dstate"))):
        check("f32" if name in ("state", "dstate") else io, got, ref[i], mag[i], d, T, name)
    token = x["state"].clone()
    o = kvm.linear_decode(token, *(x[n][:, 0].contiguous() for n in "qkv"), ld)
    check(io, o, ref[0][:, 0], mag[0][:, 0], d, 1, "token")
    assert torch.count_nonzero(grads[3][:, 0]) == 0
