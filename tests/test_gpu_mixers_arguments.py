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


def test_windows_and_sinks_are_taken_by_value():
    """A size given as a tensor is read in every call, whatever it held in an earlier one."""
    import paper_2605_09877_amd as kvm
    x = inputs()
    qkv = [x[n] for n in "qkv"]
    window, n_sink = torch.tensor(8), torch.tensor(1)
    for w, s in ((8, 1), (20, 1), (20, 3), (5, 0)):
        window.fill_(w)
        n_sink.fill_(s)
        assert torch.equal(kvm.window_prefill(*qkv, window=window, n_sink=n_sink), kvm.window_prefill(*qkv, window=w, n_sink=s))
        caches = [kvm.window_cache(B, HKV, D, window=a, n_sink=b, dtype=torch.float32, device=DEV) for a, b in ((window, n_sink), (w, s))]
        assert caches[0][0].shape == caches[1][0].shape == (B, HKV, w + s, D)
        outs = []
        for c, (a, b) in zip(caches, ((window, n_sink), (w, s))):
            kvm.window_fill(*c, x["k"], x["v"], window=a, n_sink=b)
            outs.append(kvm.window_decode(*c, *token(x), torch.full((B,), T, dtype=torch.int32, device=DEV), window=a, n_sink=b))
        assert torch.equal(*outs)
    assert torch.equal(kvm.window_prefill(*qkv, window=8.0), kvm.window_prefill(*qkv, window=8))
    for bad in (dict(window=7.5), dict(window=8, n_sink=0.5), dict(window=float("nan")), dict(window="8"), dict(window=None)):
        with pytest.raises((ValueError, TypeError)):
            kvm.window_prefill(*qkv, **bad)


def test_the_backward_pass_has_the_forward_passs_sizes():
    """Sizes and scales given as tensors that change before the backward pass."""
    import paper_2605_09877_amd as kvm
    x = inputs()
    leaves = [x[n].requires_grad_() for n in "qkv"]
    for call in (lambda w, s, c: kvm.kvm_window_attention(*leaves, window=w, n_sink=s, scale=c),
                 lambda w, s, c: kvm.kvm_linear_attention(*leaves, x["ld"], scale=c)[0]):
        want = torch.autograd.grad(call(8, 2, 0.5), leaves, x["dout"])
        w, s, c = torch.tensor(8), torch.tensor(2), torch.tensor(0.5)
        out = call(w, s, c)
        w.fill_(30), s.fill_(0), c.fill_(0.125)
        for a, b in zip(want, torch.autograd.grad(out, leaves, x["dout"])):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T0", [40, 1500])   # (one segment and several)
def test_a_state_advanced_before_the_backward_pass_is_noticed(T0):
    """The backward pass reads the state that the call started from: advanced in place since, it is refused and not used."""
    import paper_2605_09877_amd as kvm
    gen = torch.Generator(DEV).manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    q, k, v = (rnd(B, T0, h, D).requires_grad_() for h in (HQ, HKV, HKV))
    x = inputs()
    for advance in (lambda s: kvm.linear_decode(s, *token(x), x["ld"]),
                    lambda s: kvm.linear_prefill(x["q"], x["k"], x["v"], x["ld"], state=s, state_out=s)):
        state = x["state"].clone()
        out, end = kvm.kvm_linear_attention(q, k, v, x["ld"], state=state)
        want = torch.autograd.grad(out, (q, k, v), torch.ones_like(out), retain_graph=True)
        advance(end.detach())   # (the end state is not read again)
        again = torch.autograd.grad(out, (q, k, v), torch.ones_like(out), retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(want, again))
        advance(state)
        with pytest.raises(RuntimeError, match="inplace operation"):
            torch.autograd.grad(out, (q, k, v), torch.ones_like(out))


def test_what_a_call_writes_counts_as_written():
    """Every tensor of the caller's that a call writes has another version afterwards; what it only reads has not."""
    import paper_2605_09877_amd as kvm
    x = inputs(torch.bfloat16)
    qkv = [x[n] for n in "qkv"]
    out, rest, one, end = torch.empty_like(x["q"]), torch.empty_like(x["q"]), torch.empty_like(x["q"][:, 0]).contiguous(), x["state"].clone()
    ck, cv = kvm.window_cache(B, HKV, D, window=8, device=DEV)
    pos = torch.full((B,), T, dtype=torch.int32, device=DEV)
    tok = token(x)
    for call, writes in ((lambda: kvm.window_prefill(*qkv, window=8, out=out, out_rest=rest), (out, rest)),
                         (lambda: kvm.window_fill(ck, cv, x["k"], x["v"], window=8), (ck, cv)),
                         (lambda: kvm.window_decode(ck, cv, *tok, pos, window=8, out=one), (ck, cv, one)),
                         (lambda: kvm.linear_prefill(*qkv, x["ld"], state=x["state"], out=out, state_out=end), (out, end)),
                         (lambda: kvm.linear_decode(end, *tok, x["ld"], out=one), (end, one))):
        every = [*qkv, *tok, x["ld"], x["state"], pos, ck, cv, out, rest, one, end]
        before = [t._version for t in every]
        call()
        for t, n in zip(every, before):
            assert (t._version > n) == any(t is w for w in writes)


def test_tokens_in_inference_mode():
    """States and caches made there have no version: the calls are the same."""
    import paper_2605_09877_amd as kvm
    x = inputs(torch.bfloat16)
    tok, pos = token(x), torch.zeros(B, dtype=torch.int32, device=DEV)

    def work():
        state = x["state"].clone()
        ck, cv = kvm.window_cache(B, HKV, D, window=8, device=DEV)
        kvm.window_fill(ck, cv, x["k"], x["v"], window=8)
        return kvm.linear_decode(state, *tok, x["ld"]), state, kvm.window_decode(ck, cv, *tok, pos + T, window=8), ck, cv

    want = work()
    with torch.inference_mode():
        for a, b in zip(want, work()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("Hq,Hkv,T", [(4, 1, 1), (1, 1, 1), (4, 4, 3)])
def test_many_sequences_of_few_tokens(Hq, Hkv, T):
    """2^18 sequences: no more workgroups are asked for than there are tiles of positions."""
    import paper_2605_09877_amd as kvm
    n = 1 << 18
    gen = torch.Generator(DEV).manual_seed(0)
    one = [torch.randn(8, T, h, D, generator=gen, device=DEV).bfloat16() for h in (Hq, Hkv, Hkv)]
    q, k, v = (t.repeat(n // 8, 1, 1, 1).requires_grad_() for t in one)
    out = kvm.kvm_window_attention(q, k, v, window=2)
    grads = torch.autograd.grad(out, (q, k, v), out.detach())
    for t in (out, *grads):   # the same eight sequences again and again
        t = t.detach().unflatten(0, (n // 8, 8))
        assert torch.equal(t, t[:1].expand_as(t))
    few = [t.clone().requires_grad_() for t in one]
    want = kvm.kvm_window_attention(*few, window=2)
    # Eight sequences are another arrangement: P, dS and each result rounded once on either side, 2^-8 each, and where dP - D
    # cancels (a token that sees itself alone) 128 roundings of 2^-24 of sums of up to 200, times scale |k| <= 1/2.
    for got, ref in zip((out, *grads), (want, *torch.autograd.grad(want, few, want.detach()))):
        assert torch.all((got[:8].float() - ref.float()).abs() <= 2.0 ** -5 * ref.float().abs().max() + 2.0 ** -9)
    assert torch.equal(out[:8, 0], v[:8, 0].repeat_interleave(Hq // Hkv, 1))   # the first token sees itself alone


@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (2, 0, 1), (1, 2, 0), (1, 0, 2)], ids=str)
def test_outputs_in_any_order_of_axes(order):
    """[B, T, H] of out laid out in any order, with rows left out between; entries that share memory are refused."""
    import paper_2605_09877_amd as kvm
    x = inputs()
    qkv = [x[n] for n in "qkv"]
    shape = (B, 2 * T, HQ)
    buf = torch.zeros(*(shape[i] for i in order), D, device=DEV).permute(*(order.index(i) for i in range(3)), 3)
    out = buf[:, ::2]
    for call in (lambda **kw: kvm.window_prefill(*qkv, window=8, **kw), lambda **kw: kvm.linear_prefill(*qkv, x["ld"], **kw)[0]):
        want = call()
        buf.zero_()
        assert torch.equal(call(out=out), want) and torch.count_nonzero(buf[:, 1::2]) == 0
        for bad in (torch.empty(1, T, HQ, D, device=DEV).expand(B, -1, -1, -1), torch.empty(B, T, 1, D, device=DEV).expand(-1, -1, HQ, -1),
                    torch.empty(B * T * HQ * D, device=DEV).as_strided((B, T, HQ, D), (T * D, D, D, 1))):
            with pytest.raises(kvm.KVMError):
                call(out=bad)
    only = torch.empty(1, T, HQ, D, device=DEV).as_strided((1, T, HQ, D), (0, HQ * D, D, 1))   # (an axis of one entry)
    assert torch.equal(kvm.window_prefill(*(t[:1] for t in qkv), window=8, out=only), kvm.window_prefill(*(t[:1] for t in qkv), window=8))


def test_out_rest_of_an_axis_of_one_entry():
    """Its stride, which may be anything, need not be out's; those of the other axes have to be."""
    import paper_2605_09877_amd as kvm
    x = inputs(torch.bfloat16)
    qkv = [x[n][:1] for n in "qkv"]
    wide = torch.zeros(3, T, HQ, D, dtype=torch.bfloat16, device=DEV)
    out, rest = wide[1:2], torch.zeros(1, T, HQ, D, dtype=torch.bfloat16, device=DEV).as_strided((1, T, HQ, D), (D, HQ * D, D, 1))
    want = torch.empty_like(qkv[0])
    kvm.window_prefill(*qkv, window=8, out_rest=want)
    assert kvm.window_prefill(*qkv, window=8, out=out, out_rest=rest) is out and torch.equal(rest, want) and torch.count_nonzero(rest)
    for bad in (wide[:1, :, :1].expand(-1, -1, HQ, -1), wide[:1].transpose(1, 2), wide[:1, ::2], torch.zeros(1, T, 2 * HQ, D, device=DEV)[:, :, ::2]):
        with pytest.raises(ValueError, match="out_rest"):
            kvm.window_prefill(*qkv, window=8, out=out, out_rest=bad)


@pytest.mark.parametrize("T0", [40, 700])   # (P of the window as two operands and as one)
def test_calls_whose_gradients_are_not_wanted(T0):
    """The bits of a call whose gradients are, from views of a fused projection too; no memory but the results' and the workspace's."""
    import paper_2605_09877_amd as kvm
    gen = torch.Generator(DEV).manual_seed(0)
    fused = torch.randn(4, T0, HQ + 2 * HKV, D, generator=gen, device=DEV).bfloat16()
    ld = torch.tensor([-0.02, -0.3], device=DEV)
    views = lambda t: t.split((HQ, HKV, HKV), 2)
    size = 4 * T0 * HQ * D * 2
    for call, results in ((lambda q, k, v: (kvm.kvm_window_attention(q, k, v, window=90, n_sink=3),), size + size // D * 2),
                          (lambda q, k, v: kvm.kvm_linear_attention(q, k, v, ld), size + 4 * HKV * D * D * 4)):
        want = call(*views(fused.clone().requires_grad_()))
        assert all(t.requires_grad for t in want)
        with torch.no_grad():
            for q in (fused, fused.clone().requires_grad_()):
                torch.cuda.synchronize()
                torch.cuda.reset_peak_memory_stats()
                before = torch.cuda.memory_stats()["requested_bytes.all.current"]
                got = call(*views(q))   # (bytes as asked for: the allocator's blocks may be up to 1 MiB larger)
                used = torch.cuda.memory_stats()["requested_bytes.all.peak"] - before
                assert all(torch.equal(a, b) and not b.requires_grad for a, b in zip(want, got))
                workspace = 12 * 4 * HKV * D * D * 4 if len(got) == 2 and T0 > 40 else 256   # (start states of up to 12 segments)
                assert used <= results + workspace
        assert not call(*views(fused))[0].requires_grad


def test_any_layout_with_and_without_gradients():
    """q, k and v that the forward calls do not take as they lie: broadcast heads and sequences, channels apart, rows off 16-byte borders."""
    import paper_2605_09877_amd as kvm
    x = inputs(torch.bfloat16)
    off = torch.zeros(B * T * HKV * D + 8, dtype=torch.bfloat16, device=DEV)[1:1 + B * T * HKV * D].view(B, T, HKV, D)
    wide = torch.zeros(B, T, HKV, D + 3, dtype=torch.bfloat16, device=DEV)[..., 3:]
    apart = torch.zeros(B, T, D, HKV, dtype=torch.bfloat16, device=DEV).transpose(2, 3)
    for t in (wide, apart):
        t.copy_(x["k"])
    for q, k, v in ((x["q"], x["k"][:, :, :1].expand(-1, -1, HKV, -1), x["v"]), (x["q"], x["k"][:1].expand(B, -1, -1, -1), x["v"][:1].expand(B, -1, -1, -1)),
                    (x["q"], wide, x["v"]), (x["q"], apart, wide), (x["q"].transpose(0, 1).contiguous().transpose(0, 1), x["k"], x["v"]),
                    (x["q"][:1, :1], x["k"][:1, :1, :1], apart[:1, :1, 1:])):
        dense = [t.contiguous() for t in (q, k, v)]
        for call in (lambda *a: kvm.kvm_window_attention(*a, window=9), lambda *a: kvm.kvm_linear_attention(*a, x["ld"][:a[1].shape[2]])[0]):
            want = call(*dense)
            assert torch.equal(call(q, k, v), want)
            assert torch.equal(call(q, k.detach().requires_grad_(), v), want)
    for call in (lambda k: kvm.kvm_window_attention(x["q"], k, x["v"], window=9), lambda k: kvm.kvm_linear_attention(x["q"], k, x["v"], x["ld"])):
        with pytest.raises(kvm.KVMError):   # (dense, and off a 16-byte border: refused with gradients and without)
            call(off)
        with pytest.raises(kvm.KVMError):
            call(off.detach().requires_grad_())


def test_forward_mode_is_refused():
    """Tangents are not dropped where no gradient is wanted otherwise."""
    import paper_2605_09877_amd as kvm
    from torch.autograd import forward_ad
    x = inputs()
    for grad in (True, False):
        with torch.set_grad_enabled(grad), forward_ad.dual_level():
            dual = forward_ad.make_dual(x["k"], x["k"])
            for call in (lambda k: kvm.kvm_window_attention(x["q"], k, x["v"], window=8), lambda k: kvm.kvm_linear_attention(x["q"], k, x["v"], x["ld"])):
                call(x["k"])
                with pytest.raises(RuntimeError, match="jvp"):
                    call(dual)
