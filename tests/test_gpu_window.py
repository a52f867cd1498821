"""Sliding-window attention with sinks against the pair-by-pair definition in fp64: prompts, gradients, the ring cache.

Bounds, element by element, from sums over absolute values (mag).  bf16: the result is rounded once (2^-8 of it) and P or dS once
(2^-8 of the sum; in the forward pass numerator and denominator see the same rounded P, which moves the quotient by 2^-8 of
sum p |v - out| at most); D = dout . out is taken over 16 bits of out.  fp32 sums, in either type: each of the n keys and d
channels that a value goes through adds 2^-24, and an error of a logit, d + 16 roundings of at most `top`, the largest sum |q k| scale,
is a relative error of P."""
import numpy as np
import pytest
import torch

from oracle import mixers_oracle as mo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return None if t is None else t.detach().to("cpu", torch.float64).numpy()


def make(io, B, Tq, Tk, Hq, Hkv, d, seed=0):
    gen = torch.Generator(DEV).manual_seed(1000 * seed + 7 * Tk + d)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(DT[io])
    return dict(q=rnd(B, Tq, Hq, d), k=rnd(B, Tk, Hkv, d), v=rnd(B, Tk, Hkv, d), dout=rnd(B, Tq, Hq, d))


def noise(x, scale, n):
    d = x["q"].shape[-1]
    scale = d ** -0.5 if scale is None else scale
    top = scale * float(x["q"].float().norm(dim=-1).max()) * float(x["k"].float().norm(dim=-1).max())
    return (2 * n + 2 * d + 64 + 4 * (d + 16) * (top + 1)) * 2.0 ** -24


def within(got, ref, tol, name):
    got = f64(got)
    assert got.shape == ref.shape and np.all(np.isfinite(got)), name
    bad = np.abs(got - ref) - tol - 1e-30
    assert bad.max() <= 0, (name, bad.max(), np.unravel_index(bad.argmax(), bad.shape))


def out_bound(io, x, ref, window, n_sink, lens, scale):
    mag = mo.window(f64(x["q"]), f64(x["k"]), np.abs(f64(x["v"])), window, n_sink, lens, scale)[0]
    e = noise(x, scale, min(x["k"].shape[1], window + n_sink)) * mag
    return e + (2.0 ** -8 * (2 * np.abs(ref) + mag) if io == "bf16" else 0)


def run_case(io, B, T, Hq, Hkv, d, window, n_sink=0, lens=None, scale=None, Tq=None, seed=0):
    import paper_2605_09877_amd as kvm
    Tq = T if Tq is None else Tq
    x = make(io, B, Tq, T, Hq, Hkv, d, seed)
    y = {n: f64(t) for n, t in x.items()}
    dl = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    kw = dict(window=window, n_sink=n_sink, lens=dl, scale=scale)
    ref, rlse = mo.window(y["q"], y["k"], y["v"], window, n_sink, lens, scale)
    out, lse = kvm.window_prefill(x["q"], x["k"], x["v"], want_lse=True, **kw)
    within(out, ref, out_bound(io, x, ref, window, n_sink, lens, scale), "out")
    lse = f64(lse)
    live = np.isfinite(rlse)
    assert np.array_equal(live, np.isfinite(lse)) and np.all(lse[~live] == -np.inf)
    # (bf16: the sum is over P as rounded, 2^-8 of it at most)
    tol = (2.0 ** -8 if io == "bf16" else 0) + noise(x, scale, T) * (2 + np.abs(rlse[live]).max(initial=0))
    assert np.all(np.abs(lse[live] - rlse[live]) <= tol)
    leaves = [x[n].clone().requires_grad_() for n in "qkv"]
    o = kvm.kvm_window_attention(*leaves, **kw)
    assert torch.equal(o, out)
    grads = torch.autograd.grad(o, leaves, x["dout"])
    rgrads = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], window, n_sink, lens, scale)
    mags = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], window, n_sink, lens, scale, absolute=True)
    # (the row sum that lse holds is over rounded P: one more 2^-8 of P in bf16)
    e = noise(x, scale, T * (Hq // Hkv)) + (2 * 2.0 ** -8 + 2.0 ** -14 if io == "bf16" else 0)
    for got, r, m, name in zip(grads, rgrads, mags, ("dq", "dk", "dv")):
        within(got, r, e * m + (2.0 ** -8 * np.abs(r) if io == "bf16" else 0), name)
    if lens is not None:
        for b, n in enumerate(lens):
            n = max(n, 0)
            assert torch.count_nonzero(grads[1][b, n:]) == 0 and torch.count_nonzero(grads[2][b, n:]) == 0
            nq = max(n - (T - Tq), 0)
            assert torch.count_nonzero(out[b, nq:]) == 0 and torch.count_nonzero(grads[0][b, nq:]) == 0


@pytest.mark.parametrize("io,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 65, 127, 128, 129, 200])
def test_lengths_about_the_tiles(io, d, T):
    run_case(io, 1, T, 2, 1, d, window=50, n_sink=3)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (2, 128), (31, 64), (32, 0), (33, 33), (64, 5), (65, 65), (299, 4), (300, 4),
                                           (5000, 100)])
def test_windows_and_sinks(io, window, n_sink):
    run_case(io, 1, 300, 2, 2, 64, window, n_sink)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (4, 1), (8, 2), (6, 2), (5, 5)])   # (groups of four: waves take heads)
def test_shared_and_odd_heads(io, Hq, Hkv):
    run_case(io, 2, 150, Hq, Hkv, 64, 40, 2)


@pytest.mark.parametrize("io,d,Hq", [("bf16", 128, 4), ("f32", 64, 2), ("bf16", 64, 3), ("f32", 128, 4)])
def test_padded_batch_with_empty_sequences(io, d, Hq):
    run_case(io, 5, 170, Hq, 1, d, 37, 5, lens=[0, 170, 1, 3, 131])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("Tq,lens", [(1, None), (30, None), (100, [160, 61, 60, 0, 100])])
def test_queries_behind_earlier_keys(io, Tq, lens):
    run_case(io, 1 if lens is None else 5, 160, 4, 2, 64, 45, 4, lens=lens, Tq=Tq)


def test_scale_and_many_units():
    run_case("f32", 1, 70, 2, 1, 64, 20, 1, scale=0.5)
    run_case("bf16", 9, 140, 3, 3, 64, 64, 1)   # 27 units, three to an XCD and three left over


@pytest.mark.parametrize("io,G", [("bf16", 4), ("f32", 2)])
def test_views_of_a_fused_projection(io, G):
    import paper_2605_09877_amd as kvm
    B, T, Hkv, d = 2, 140, 2, 64
    Hq = G * Hkv
    x = make(io, B, T, T, Hq, Hkv, d)
    fused = torch.cat([x["q"], x["k"], x["v"]], dim=2)
    wide = torch.full((B, T, Hq + 3, d), 7.0, device=DEV, dtype=DT[io])
    want = kvm.window_prefill(x["q"], x["k"], x["v"], window=40, n_sink=3)
    kvm.window_prefill(fused[:, :, :Hq], fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:], window=40, n_sink=3, out=wide[:, :, 1:1 + Hq])
    assert torch.equal(wide[:, :, 1:1 + Hq], want)
    assert bool((wide[:, :, 0] == 7).all()) and bool((wide[:, :, 1 + Hq:] == 7).all())


@pytest.mark.parametrize("io,d,Hq", [("bf16", 128, 4), ("f32", 64, 2), ("bf16", 64, 1)])
def test_padding_may_hold_anything(io, d, Hq):
    import paper_2605_09877_amd as kvm
    x = make(io, 3, 140, 140, Hq, 1, d)
    lens = torch.tensor([0, 70, 139], dtype=torch.int32, device=DEV)
    kw = dict(window=50, n_sink=4, lens=lens)

    def both():
        leaves = [x[n].clone().requires_grad_() for n in "qkv"]
        o = kvm.kvm_window_attention(*leaves, **kw)
        return (o, *torch.autograd.grad(o, leaves, x["dout"]))

    want = both()
    for b, n in enumerate(lens.tolist()):
        for i, name in enumerate(("q", "k", "v", "dout")):
            x[name][b, n:] = float("nan") if i % 2 else float("inf")
    for a, b in zip(want, both()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("io,d,Hq", [("bf16", 128, 4), ("bf16", 64, 2), ("f32", 64, 1), ("f32", 128, 2)])
def test_values_that_are_not_finite_reach_who_sees_them(io, d, Hq):
    """NaN and infinities in k and v of single tokens: queries that do not see them have their finite results, those that do what
    the definition gives (a NaN key or value: NaN; an infinite value: that infinity; a key of -infinity: no weight, where q is positive)."""
    import paper_2605_09877_amd as kvm
    T, W, S = 260, 60, 2
    x = make(io, 1, T, T, Hq, 1, d)
    want = kvm.window_prefill(x["q"], x["k"], x["v"], window=W, n_sink=S)
    x["v"][0, 100, 0, 3] = float("nan")
    x["v"][0, 150, 0, 5] = float("inf")
    x["k"][0, 200, 0, 7] = float("nan")
    got = kvm.window_prefill(x["q"], x["k"], x["v"], window=W, n_sink=S)
    sees = lambda t, j: j <= t < j + W
    for t in range(T):
        if sees(t, 200):
            assert torch.isnan(got[0, t]).all()
            continue
        w = want[0, t].clone()
        if sees(t, 100):
            assert torch.isnan(got[0, t, :, 3]).all()
            w[:, 3] = got[0, t, :, 3] = 0
        if sees(t, 150):
            assert torch.isinf(got[0, t, :, 5]).all()
            w[:, 5] = got[0, t, :, 5] = 0
        # (a query done again, key by key in fp32, has another order of sums and no rounded P)
        tol = 2.0 ** -6 if io == "bf16" else 1e-4
        assert (got[0, t].float() - w.float()).abs().max() <= tol * (1 + w.float().abs().max()), t
    x = make(io, 1, 40, 40, Hq, 1, d)
    x["q"].abs_()
    x["k"][0, :, 0, 0] = float("-inf")
    assert torch.count_nonzero(kvm.window_prefill(x["q"] + 1, x["k"], x["v"], window=W, n_sink=S)) == 0


def ring(x, t, window, n_sink):
    """What the cache has to hold behind position t: {row: position}."""
    return {p if p < n_sink else n_sink + (p - n_sink) % window: p for p in range(t + 1)}


@pytest.mark.parametrize("io,d,G", [("bf16", 128, 4), ("bf16", 64, 1), ("f32", 64, 3), ("f32", 128, 5), ("bf16", 128, 9)])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (7, 3), (100, 4), (64, 0), (600, 128)])
def test_prompt_then_tokens(io, d, G, window, n_sink):
    """Sequences of different lengths (one empty) filled, then decoded until every ring has wrapped, an idle one among them."""
    import paper_2605_09877_amd as kvm
    lens, steps = [150, 0, 2, 99], 12
    B, T = len(lens), 150 + steps
    x = make(io, B, T, T, G, 1, d)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ck, cv = kvm.window_cache(B, 1, d, window=window, n_sink=n_sink, dtype=DT[io], device=DEV)
    ck.fill_(float("nan"))
    cv.fill_(float("nan"))
    kvm.window_fill(ck, cv, x["k"][:, :150], x["v"][:, :150], window=window, n_sink=n_sink, lens=dl)
    y = {n: f64(t) for n, t in x.items()}
    for step in range(steps):
        pos = [n + step for n in lens]
        if step == 5:
            pos[2] = -1
        take = lambda n: torch.stack([x[n][b, max(p, 0)] for b, p in enumerate(pos)])
        out = kvm.window_decode(ck, cv, take("q"), take("k"), take("v"), torch.tensor(pos, dtype=torch.int32, device=DEV),
                                window=window, n_sink=n_sink)
        for b, p in enumerate(pos):
            if p < 0:
                assert torch.count_nonzero(out[b]) == 0
                lens[b] -= 1   # (the token comes a step later)
                continue
            one = {n: t[b:b + 1, :p + 1] for n, t in y.items()}
            q1 = one["q"][:, -1:]
            ref, _ = mo.window(q1, one["k"], one["v"], window, n_sink)
            mag, _ = mo.window(q1, one["k"], np.abs(one["v"]), window, n_sink)
            tol = noise(x, None, min(p + 1, window + n_sink)) * mag + (2.0 ** -8 * np.abs(ref) if io == "bf16" else 0)
            within(out[b:b + 1, None], ref, tol, f"step {step} sequence {b}")
    for b, p in enumerate(pos):
        for row, at in ring(x, p, window, n_sink).items():
            assert torch.equal(ck[b, 0, row], x["k"][b, at, 0]) and torch.equal(cv[b, 0, row], x["v"][b, at, 0])


def test_fill_leaves_rows_without_tokens_and_far_positions_decode():
    import paper_2605_09877_amd as kvm
    ck, cv = kvm.window_cache(2, 3, 64, window=20, n_sink=2, device=DEV)
    ck.fill_(5)
    cv.fill_(6)
    x = make("bf16", 2, 9, 9, 3, 3, 64)
    kvm.window_fill(ck, cv, x["k"], x["v"], window=20, n_sink=2, lens=torch.tensor([9, 0], dtype=torch.int32, device=DEV))
    assert torch.equal(ck[0, :, :9], x["k"][0].transpose(0, 1)) and bool((ck[0, :, 9:] == 5).all()) and bool((ck[1] == 5).all())
    assert torch.equal(cv[0, :, :9], x["v"][0].transpose(0, 1)) and bool((cv[1] == 6).all())
    # a position near the end of int32: its row, and every row seen
    far = 2 ** 31 - 2
    ck, cv = (torch.randn(1, 1, 22, 64, device=DEV) for _ in range(2))
    q, k, v = (torch.randn(1, 1, 64, device=DEV) for _ in range(3))
    row = 2 + (far - 2) % 20
    want_k, want_v = ck.clone(), cv.clone()
    want_k[0, 0, row], want_v[0, 0, row] = k[0, 0], v[0, 0]
    out = kvm.window_decode(ck, cv, q, k, v, torch.tensor([far], dtype=torch.int32, device=DEV), window=20, n_sink=2)
    assert torch.equal(ck, want_k) and torch.equal(cv, want_v)
    p = torch.softmax((want_k[0, 0].double() @ q[0, 0].double()) / 8, 0)
    assert (out[0, 0].double() - p @ want_v[0, 0].double()).abs().max() <= 1e-5


@pytest.mark.parametrize("B,Hkv,G,window", [(1, 8, 4, 4096), (40, 8, 2, 700), (300, 4, 1, 90), (1, 1, 1, 20000)])
def test_decode_arrangements(B, Hkv, G, window):
    """Few sequences with long caches (ranges joined by a second launch) to many with short ones (one workgroup each)."""
    import paper_2605_09877_amd as kvm
    gen = torch.Generator(DEV).manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()
    rows, d = window + 4, 128
    ck, cv = rnd(B, Hkv, rows, d), rnd(B, Hkv, rows, d)
    q, k, v = rnd(B, Hkv * G, d), rnd(B, Hkv, d), rnd(B, Hkv, d)
    pos = torch.randint(0, 2 * rows, (B,), generator=gen, device=DEV, dtype=torch.int32)
    pos[0] = rows // 2
    wk, wv = ck.clone(), cv.clone()
    place = torch.where(pos < 4, pos, 4 + (pos - 4) % window).long()
    b = torch.arange(B, device=DEV)
    wk[b, :, place], wv[b, :, place] = k, v
    out = kvm.window_decode(ck, cv, q, k, v, pos, window=window, n_sink=4)
    assert torch.equal(ck, wk) and torch.equal(cv, wv)
    filled = torch.arange(rows, device=DEV) <= pos[:, None]
    for i in range(0, B, max(1, B // 8)):
        t = (q[i].double().reshape(Hkv, G, d) @ wk[i].double().mT.contiguous()) * d ** -0.5
        p = torch.softmax(t.masked_fill(~filled[i], float("-inf")), -1)
        ref, mag = (p @ wv[i].double()).reshape(-1, d), (p @ wv[i].double().abs()).reshape(-1, d)
        top = float(t.abs().max())
        tol = 2.0 ** -8 * ref.abs() + (2 * rows + 2 * d + 4 * (d + 16) * (top * 16 + 1)) * 2.0 ** -24 * mag + 1e-30
        assert bool(((out[i].double() - ref).abs() <= tol).all())


def test_same_call_same_bits_other_streams_and_captured():
    import paper_2605_09877_amd as kvm
    x = make("bf16", 2, 700, 700, 4, 1, 128)
    ck, cv = kvm.window_cache(2, 1, 128, window=300, n_sink=4, device=DEV)
    tok = [x[n][:, -1].contiguous() for n in "qkv"]
    pos = torch.tensor([699, 300], dtype=torch.int32, device=DEV)
    kw = dict(window=300, n_sink=4)

    def work():
        rest = torch.empty_like(x["q"])
        out, lse = kvm.window_prefill(x["q"], x["k"], x["v"], want_lse=True, out_rest=rest, **kw)
        g = kvm.window_backward(x["q"], x["k"], x["v"], out, lse, x["dout"], out_rest=rest, **kw)
        kvm.window_fill(ck, cv, x["k"][:, :699], x["v"][:, :699], **kw)
        return (out, *g, kvm.window_decode(ck, cv, *tok, pos, **kw))

    want = [t.clone() for t in work()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = work()
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for _ in range(3):
        for t in got:
            t.zero_()
        kvm.window_prefill(x["q"], x["v"], x["k"], window=77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)


def test_gradient_is_the_slope():
    """Central differences of the loss in a direction of all inputs: the third-order term is of the order of e^2 (2^-14) of the
    size of the gradient's terms, the rounding of two fp32 losses far below."""
    import paper_2605_09877_amd as kvm
    x = make("f32", 2, 90, 90, 4, 2, 64)
    gen = torch.Generator(DEV).manual_seed(5)
    ins = [x[n] for n in "qkv"]
    dirs = [torch.randn(t.shape, generator=gen, device=DEV) for t in ins]
    eps, kw = 2.0 ** -7, dict(window=30, n_sink=3)

    def loss(sign):
        out = kvm.window_prefill(*[t + sign * eps * u for t, u in zip(ins, dirs)], **kw)
        return (out.double() * x["dout"].double()).sum()

    leaves = [t.clone().requires_grad_() for t in ins]
    grads = torch.autograd.grad(kvm.kvm_window_attention(*leaves, **kw), leaves, x["dout"])
    slope = sum((g.double() * u.double()).sum() for g, u in zip(grads, dirs))
    diff = (loss(1) - loss(-1)) / (2 * eps)
    size = sum((g.double() * u.double()).abs().sum() for g, u in zip(grads, dirs))
    assert abs(slope - diff) <= 1e-3 * size


def test_refusals_by_the_binding():
    import paper_2605_09877_amd as kvm
    x = make("bf16", 2, 8, 8, 4, 2, 64)
    ok = (x["q"], x["k"], x["v"])
    for bad in (dict(window=0), dict(window=1 << 30), dict(window=4, n_sink=129), dict(window=4, n_sink=-1),
                dict(window=4, lens=torch.tensor([8, 8], device=DEV)), dict(window=4, scale=-1.0), dict(window=4, scale=float("nan")),
                dict(window=4, out=torch.empty_like(x["q"]).transpose(1, 2)), dict(window=4, out_rest=torch.empty_like(x["k"]))):
        with pytest.raises((ValueError, kvm.KVMError)):
            kvm.window_prefill(*ok, **bad)
    for q, k, v in ((x["q"], x["k"].float(), x["v"]), (x["q"].half(), x["k"].half(), x["v"].half()), (x["q"][:, :, :3], x["k"], x["v"]),
                    (x["q"], x["k"][:, :7], x["v"][:, :7]), (x["q"][:, :0], x["k"], x["v"])):
        with pytest.raises(ValueError):
            kvm.window_prefill(q, k, v, window=4)
    ck, cv = kvm.window_cache(2, 2, 64, window=4, device=DEV)
    with pytest.raises(ValueError):
        kvm.window_decode(ck, cv, x["q"][:, 0], x["k"][:, 0].contiguous(), x["v"][:, 0].contiguous(),
                          torch.zeros(2, dtype=torch.int32, device=DEV), window=4)
    with pytest.raises(ValueError):
        kvm.window_decode(ck, cv, *[x[n][:, 0].contiguous() for n in "qkv"], torch.zeros(2, device=DEV), window=4)
    with pytest.raises(ValueError):
        kvm.window_fill(ck, cv, x["k"], x["v"], window=5)


def test_gradients_of_gradients_are_refused_and_a_graph_can_be_used_twice():
    import paper_2605_09877_amd as kvm
    x = make("f32", 1, 40, 40, 2, 1, 64)
    leaves = [x[n].clone().requires_grad_() for n in "qkv"]
    out = kvm.kvm_window_attention(*leaves, window=9)
    first = torch.autograd.grad(out, leaves, x["dout"], retain_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(out, leaves, x["dout"], retain_graph=True, create_graph=True)
    for a, b in zip(first, torch.autograd.grad(out, leaves, x["dout"])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("io,d,B,Hq,Hkv,T", [
    ("bf16", 128, 132, 4, 4, 150), ("bf16", 64, 70, 8, 2, 140), ("bf16", 128, 70, 8, 2, 140),   # a head or four to a workgroup
    ("f32", 64, 132, 4, 4, 150), ("f32", 128, 132, 4, 4, 140), ("f32", 128, 70, 8, 2, 140)])
def test_many_sequences(io, d, B, Hq, Hkv, T):
    """Calls that fill the device: workgroups whose waves share tiles of keys (prompt, dq) and take a key tile's queries whole (dk, dv).
    Lengths of all kinds, a few of the sequences compared."""
    import paper_2605_09877_amd as kvm
    x = make(io, B, T, T, Hq, Hkv, d)
    lens = [(7 * b) % (T + 1) for b in range(B)]
    lens[0], lens[B // 2], lens[B - 1] = T, 129, 33
    W, S = 45, 3
    kw = dict(window=W, n_sink=S, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    leaves = [x[n].clone().requires_grad_() for n in "qkv"]
    o = kvm.kvm_window_attention(*leaves, **kw)
    grads = torch.autograd.grad(o, leaves, x["dout"])
    for b in (0, B // 2, B - 1):
        one = {n: t[b:b + 1] for n, t in x.items()}
        y = {n: f64(t) for n, t in one.items()}
        ref = mo.window(y["q"], y["k"], y["v"], W, S, [lens[b]])[0]
        within(o[b:b + 1], ref, out_bound(io, one, ref, W, S, [lens[b]], None), f"out {b}")
        rg = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], W, S, [lens[b]])
        mg = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], W, S, [lens[b]], absolute=True)
        e = noise(one, None, T * (Hq // Hkv)) + (2 * 2.0 ** -8 + 2.0 ** -14 if io == "bf16" else 0)
        for got, r, m, name in zip(grads, rg, mg, ("dq", "dk", "dv")):
            within(got[b:b + 1], r, e * m + (2.0 ** -8 * np.abs(r) if io == "bf16" else 0), f"{name} {b}")
    for b, n in enumerate(lens):
        for t in (o, *grads):
            assert torch.count_nonzero(t[b, n:]) == 0


def test_more_units_than_a_grids_second_dimension():
    """70000 sequences of a few tokens: gradients with sinks, the cache filled and asked."""
    import paper_2605_09877_amd as kvm
    B, T, W, S, d = 70000, 4, 2, 1, 64
    x = make("bf16", 8, T, T, 1, 1, d)
    many = {n: t.repeat(B // 8, 1, 1, 1) for n, t in x.items()}
    leaves = [many[n].clone().requires_grad_() for n in "qkv"]
    o = kvm.kvm_window_attention(*leaves, window=W, n_sink=S)
    grads = torch.autograd.grad(o, leaves, many["dout"])
    ck, cv = kvm.window_cache(B, 1, d, window=W, n_sink=S, device=DEV)
    kvm.window_fill(ck, cv, many["k"], many["v"], window=W, n_sink=S)
    for t in (o, *grads, ck, cv):   # the same eight sequences again and again
        t = t.unflatten(0, (B // 8, 8))
        assert torch.equal(t, t[:1].expand_as(t))
    y = {n: f64(t) for n, t in x.items()}
    ref = mo.window(y["q"], y["k"], y["v"], W, S)[0]
    within(o[:8], ref, out_bound("bf16", x, ref, W, S, None, None), "out")
    rg = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], W, S)
    mg = mo.window_backward(y["q"], y["k"], y["v"], y["dout"], W, S, absolute=True)
    for got, r, m, name in zip(grads, rg, mg, ("dq", "dk", "dv")):
        within(got[:8], r, (noise(x, None, T) + 2 * 2.0 ** -8 + 2.0 ** -14) * m + 2.0 ** -8 * np.abs(r), name)
    assert torch.equal(ck[:8, 0], x["k"][:, [0, 3, 2], 0]) and torch.equal(cv[-8:, 0], x["v"][:, [0, 3, 2], 0])
    pos = torch.full((B,), T, dtype=torch.int32, device=DEV)   # sees positions 0, 3 and 4
    t = kvm.window_decode(ck, cv, *(many[n][:, i].contiguous() for i, n in enumerate("qkv")), pos, window=W, n_sink=S)
    order = dict(k=np.concatenate([y["k"][:, [0, 3]], y["k"][:, 1:2]], 1), v=np.concatenate([y["v"][:, [0, 3]], y["v"][:, 2:3]], 1))
    ref = mo.window(y["q"][:, :1], order["k"], order["v"], 3)[0]
    t8 = t.unflatten(0, (B // 8, 8))
    assert torch.equal(t8, t8[:1].expand_as(t8))
    one = dict(q=x["q"][:, :1], k=torch.as_tensor(order["k"]), v=torch.as_tensor(order["v"]))
    within(t[:8, None], ref, out_bound("bf16", one, ref, 3, 0, None, None), "token")


@pytest.mark.parametrize("io,d,step", [("bf16", 128, 0.02), ("bf16", 64, 0.5), ("f32", 64, 0.1), ("f32", 128, -0.3)])
def test_maxima_that_rise_or_fall_along_the_keys(io, d, step):
    """A logit of about step for every key: the reference of the exponentials moves often, seldom, or never again; in calls of many
    sequences and of one."""
    import paper_2605_09877_amd as kvm
    B, T, W, S = 132, 200, 150, 2
    x = make(io, 1, T, T, 4, 4, d, seed=3)
    x["q"] = (1 + 0.1 * x["q"].float()).to(DT[io])
    x["k"] = (step * d ** -0.5 * torch.arange(T, device=DEV).view(1, T, 1, 1) + 0.05 * x["k"].float()).to(DT[io])
    y = {n: f64(t) for n, t in x.items()}
    ref = mo.window(y["q"], y["k"], y["v"], W, S)[0]
    tol = out_bound(io, x, ref, W, S, None, None)
    for n in (1, B):
        out, lse = kvm.window_prefill(*(x[m].repeat(n, 1, 1, 1) for m in "qkv"), window=W, n_sink=S, want_lse=True)
        within(out[:1], ref, tol, f"out of {n}")
        assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))


@pytest.mark.parametrize("B,T,W,S", [(8, 24, 300, 0), (4, 100, 64, 3), (2, 700, 9, 0), (1, 900, 300, 5)])
def test_gradients_are_within_two_roundings(B, T, W, S):
    """The norm of the error of dq and dk, bf16: dS is rounded once and the result once, each with an error of 2^-8 / 3^(1/2) of its value
    at the most (a mean square over a step's whole width), independent of the other; another 5 % for what is left of P's rounding."""
    import paper_2605_09877_amd as kvm
    x = make("bf16", B, T, T, 4, 2, 64, seed=9)
    leaves = [x[n].clone().requires_grad_() for n in "qkv"]
    grads = torch.autograd.grad(kvm.kvm_window_attention(*leaves, window=W, n_sink=S), leaves, x["dout"])
    ref = mo.window_backward(*(f64(x[n]) for n in ("q", "k", "v", "dout")), W, S)
    for got, r, name in zip(grads, ref, ("dq", "dk", "dv")):
        error = np.linalg.norm(f64(got) - r) / np.linalg.norm(r)
        assert error <= 1.05 * 2 ** 0.5 * 2.0 ** -8 / 3 ** 0.5, (name, error)
