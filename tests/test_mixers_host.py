"""The mixers beside the layer without a GPU: what their C entry points refuse before any launch, the sizes they ask for, and the
oracle's implementations pinned by differences, by hand, and by forms that share no code with them."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import mixers_oracle as mo
from paper_2605_09877_amd import binding as kb

P = 0x10000000   # aligned, never dereferenced: every call below returns an error first
BIG = 1 << 62


def lin(**kw):
    return kb.kvm_linear_config(*(dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=128, io_dtype=kb.KVM_BF16, scale=0.0) | kw).values())


def win(**kw):
    return kb.kvm_window_config(*(dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, io_dtype=kb.KVM_F32, n_sink=4, window=100,
                                       scale=0.0) | kw).values())


HEADS = [dict(batch=0), dict(batch=-1), dict(n_q_heads=3), dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_kv_heads=-2), dict(head_dim=96),
         dict(head_dim=32), dict(head_dim=256), dict(io_dtype=7), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf),
         dict(batch=1 << 22)]


class LinearCalls:
    """The three calls with arguments that are right but for `over` (by name)."""

    def __init__(self, lib, cfg):
        self.lib, self.cfg = lib, cfg

    def prefill(self, **over):
        a = dict(q=P, k=P, v=P, ld=P, s0=P, lens=None, out=P, s1=P, T=70, strides=None, ws=P, n=BIG, stream=None) | over
        return self.lib.kvm_linear_prefill(self.cfg, *a.values())

    def backward(self, **over):
        a = dict(q=P, k=P, v=P, ld=P, s0=P, lens=None, dout=P, ds1=P, dq=P, dk=P, dv=P, ds0=P, T=70, kept=None, ws=P, n=BIG, stream=None) | over
        return self.lib.kvm_linear_backward(self.cfg, *a.values())

    def decode(self, **over):
        a = dict(state=P, q=P, k=P, v=P, ld=P, active=None, out=P, stream=None) | over
        return self.lib.kvm_linear_decode(self.cfg, *a.values())


class WindowCalls:
    def __init__(self, lib, cfg):
        self.lib, self.cfg = lib, cfg

    def prefill(self, **over):
        a = dict(q=P, k=P, v=P, lens=None, out=P, rest=None, lse=None, Tq=70, Tk=70, strides=None, stream=None) | over
        return self.lib.kvm_window_prefill(self.cfg, *a.values())

    def backward(self, **over):
        a = dict(q=P, k=P, v=P, lens=None, out=P, rest=None, lse=P, dout=P, dq=P, dk=P, dv=P, Tq=70, Tk=70, ws=P, n=BIG, stream=None) | over
        return self.lib.kvm_window_backward(self.cfg, *a.values())

    def fill(self, **over):
        a = dict(ck=P, cv=P, k=P, v=P, lens=None, T=70, strides=None, stream=None) | over
        return self.lib.kvm_window_fill(self.cfg, *a.values())

    def decode(self, **over):
        a = dict(ck=P, cv=P, q=P, k=P, v=P, pos=P, out=P, ws=P, n=BIG, stream=None) | over
        return self.lib.kvm_window_decode(self.cfg, *a.values())


@pytest.mark.parametrize("bad", HEADS, ids=str)
def test_linear_configurations_refused(bad):
    lib = kb.load_library()
    c = LinearCalls(lib, lin(**bad))
    assert lib.kvm_linear_workspace_bytes(c.cfg, 70) == 0
    assert {c.prefill(), c.backward(), c.decode()} == {kb.KVM_ERR_ARG}


@pytest.mark.parametrize("bad", HEADS + [dict(window=0), dict(window=-1), dict(window=1 << 30), dict(n_sink=-1), dict(n_sink=129)], ids=str)
def test_window_configurations_refused(bad):
    lib = kb.load_library()
    c = WindowCalls(lib, win(**bad))
    assert lib.kvm_window_backward_workspace_bytes(c.cfg, 70, 70) == lib.kvm_window_decode_workspace_bytes(c.cfg) == 0
    assert {c.prefill(), c.backward(), c.fill(), c.decode()} == {kb.KVM_ERR_ARG}


def strides(**kw):
    """[B, 70, 4 or 2, d = 128 at most] dense but for kw."""
    s = kb.kvm_strides()
    for n in "qkvo":
        setattr(s, n + "_b", 70 * 4 * 128)
        setattr(s, n + "_t", 4 * 128)
        setattr(s, n + "_h", 128)
    s.lse_b, s.lse_t, s.lse_h = 280, 4, 1
    for n, v in kw.items():
        setattr(s, n, v)
    return C.byref(s)


BAD_STRIDES = [dict(q_t=516 + 1), dict(k_h=12), dict(v_b=-512), dict(o_t=64 - 8), dict(k_t=(1 << 23) + 512), dict(v_h=0)]


def test_linear_arguments_refused():
    lib = kb.load_library()
    c = LinearCalls(lib, lin())
    for name in ("q", "k", "v", "ld", "out", "ws"):
        assert c.prefill(**{name: None}) == kb.KVM_ERR_ARG, name
    for name in ("q", "k", "v", "s0", "out", "s1", "ws"):
        assert c.prefill(**{name: P + 8}) == kb.KVM_ERR_ARG, name
    for T in (0, -1, 1 << 29, 1 << 31, BIG):
        assert c.prefill(T=T) == c.backward(T=T) == kb.KVM_ERR_ARG and lib.kvm_linear_workspace_bytes(c.cfg, T) == 0
    for bad in BAD_STRIDES:
        assert c.prefill(strides=strides(**bad)) == kb.KVM_ERR_ARG, bad
    for name in ("q", "k", "v", "ld", "dout", "dq", "dk", "dv", "ws"):
        assert c.backward(**{name: None}) == kb.KVM_ERR_ARG, name
    for name in ("q", "k", "v", "s0", "dout", "ds1", "dq", "dk", "dv", "ds0", "kept", "ws"):
        assert c.backward(**{name: P + 4}) == kb.KVM_ERR_ARG, name
    need = lib.kvm_linear_workspace_bytes(c.cfg, 70)
    assert c.prefill(n=need - 1) == c.backward(n=need - 1) == kb.KVM_ERR_CAPACITY
    for name in ("state", "q", "k", "v", "ld", "out"):
        assert c.decode(**{name: None}) == kb.KVM_ERR_ARG, name
    for name in ("state", "q", "k", "v", "out"):
        assert c.decode(**{name: P + 8}) == kb.KVM_ERR_ARG, name
    wide = LinearCalls(lib, lin(n_q_heads=1 << 17, n_kv_heads=1 << 17, batch=1))   # rows longer than 2^23 elements
    assert wide.backward() == wide.prefill() == kb.KVM_ERR_ARG
    assert LinearCalls(lib, lin(n_q_heads=1, n_kv_heads=1, batch=1 << 23)).backward() == kb.KVM_ERR_ARG   # 512 threads for each state


def test_window_arguments_refused():
    lib = kb.load_library()
    c = WindowCalls(lib, win())
    for name in ("q", "k", "v", "out"):
        assert c.prefill(**{name: None}) == c.prefill(**{name: P + 8}) == kb.KVM_ERR_ARG, name
    assert c.prefill(rest=P + 2) == kb.KVM_ERR_ARG
    for Tq, Tk in ((0, 70), (-1, 70), (71, 70), (1, 1 << 30), (BIG, BIG), (0, 0)):
        assert c.prefill(Tq=Tq, Tk=Tk) == c.backward(Tq=Tq, Tk=Tk) == kb.KVM_ERR_ARG
        assert lib.kvm_window_backward_workspace_bytes(c.cfg, Tq, Tk) == 0
    for bad in BAD_STRIDES + [dict(q_h=2), dict(k_t=60)]:
        assert c.prefill(strides=strides(**bad)) == kb.KVM_ERR_ARG, bad
    for bad in (dict(lse_b=-1), dict(lse_t=0), dict(lse_h=-1)):
        assert c.prefill(lse=P, strides=strides(**bad)) == kb.KVM_ERR_ARG, bad
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv", "ws"):
        assert c.backward(**{name: None}) == c.backward(**{name: P + 8}) == kb.KVM_ERR_ARG, name
    assert c.backward(lse=None) == c.backward(rest=P + 2) == kb.KVM_ERR_ARG
    need = lib.kvm_window_backward_workspace_bytes(c.cfg, 70, 70)
    assert c.backward(n=need - 1) == kb.KVM_ERR_CAPACITY
    for name in ("ck", "cv", "k", "v"):
        assert c.fill(**{name: None}) == c.fill(**{name: P + 8}) == kb.KVM_ERR_ARG, name
    for T in (0, -5, 1 << 30):
        assert c.fill(T=T) == kb.KVM_ERR_ARG
    for bad in (dict(k_t=2), dict(v_b=-512), dict(k_h=129)):
        assert c.fill(strides=strides(**bad)) == kb.KVM_ERR_ARG, bad
    for name in ("ck", "cv", "q", "k", "v", "out", "ws"):
        assert c.decode(**{name: None}) == c.decode(**{name: P + 8}) == kb.KVM_ERR_ARG, name
    assert c.decode(pos=None) == kb.KVM_ERR_ARG
    assert c.decode(n=lib.kvm_window_decode_workspace_bytes(c.cfg) - 1) == kb.KVM_ERR_CAPACITY
    huge = WindowCalls(lib, win(window=(1 << 30) - 1, batch=1))   # more rows than a launch has threads for
    assert huge.fill() == kb.KVM_ERR_ARG
    many = WindowCalls(lib, win(batch=(1 << 24) - 1, n_q_heads=1, n_kv_heads=1))
    assert many.prefill(Tq=1000, Tk=1000) == many.backward(Tq=1000, Tk=1000) == kb.KVM_ERR_ARG


def test_workspaces_hold_what_is_cut():
    lib = kb.load_library()
    state = 4 * 128 * 128 * 2 * 2
    assert lib.kvm_linear_workspace_bytes(lin(), 1) == 256                      # not cut: nothing in it
    assert lib.kvm_linear_workspace_bytes(lin(), 4096) >= 2 * state             # start states of two segments at least
    for T in (1, 64, 447, 513, 4096, 1 << 20, (1 << 29) - 1):
        n = lib.kvm_linear_workspace_bytes(lin(), T)
        assert n == 256 or (n % state == 0 and 2 <= n // state <= -(-T // 64))
    for c in (win(), win(n_q_heads=64, n_kv_heads=8, batch=64, io_dtype=kb.KVM_BF16)):
        H = c.batch * c.n_q_heads
        for Tq, Tk in ((1, 1), (70, 70), (70, 700), (5000, 5000)):   # D = dout . out, and the sinks' shares
            assert lib.kvm_window_backward_workspace_bytes(c, Tq, Tk) >= 4 * H * Tq + (8 * c.batch * c.n_kv_heads * 4 * 64 if Tk > 100 else 0)
        assert lib.kvm_window_decode_workspace_bytes(c) > 0


# ---- the oracle


def problem(seed, B=2, Tq=9, Tk=9, Hq=4, Hkv=2, d=3):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((B, Tq, Hq, d)), rng.standard_normal((B, Tk, Hkv, d)), rng.standard_normal((B, Tk, Hkv, d)),
            rng.standard_normal((B, Tq, Hq, d)))


def test_linear_oracle_by_hand():
    one = lambda *x: np.array(x, np.float64).reshape(1, -1, 1, 1)
    out, end = mo.linear(one(2, 1, 3), one(1, 2, 1), one(5, 7, 1), [math.log(0.5)], np.full((1, 1, 1, 1), 4.0), scale=1.0)
    # S = 2 + 5 = 7; 3.5 + 14 = 17.5; 8.75 + 1 = 9.75
    assert np.allclose(out.ravel(), [14, 17.5, 29.25], rtol=1e-14) and np.isclose(end.item(), 9.75, rtol=1e-14)


@pytest.mark.parametrize("lens", [None, [9, 4], [0, 1], [-3, 99]])
def test_linear_oracle_is_the_masked_product_and_its_gradient_autograds(lens):
    q, k, v, dout = problem(1)
    B, T, Hq, d = q.shape
    rng = np.random.default_rng(2)
    ld, s0, ds = np.array([-0.3, -0.02]), rng.standard_normal((B, 2, d, d)), rng.standard_normal((B, 2, d, d))
    tq, tk, tv, ts = (torch.tensor(x, requires_grad=True) for x in (q, k, v, s0))
    n = [T] * B if lens is None else [min(max(x, 0), T) for x in lens]
    out, end = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(s0.shape, dtype=torch.float64)
    for b in range(B):
        i = torch.arange(n[b], dtype=torch.float64)
        for h in range(Hq):
            a = ld[h // 2]
            w = torch.exp(a * (i[:, None] - i[None])) * (i[:, None] >= i[None])
            x, y, z = tq[b, :n[b], h], tk[b, :n[b], h // 2], tv[b, :n[b], h // 2]
            o = ((x @ y.T) * w) @ z + torch.exp(a * (i + 1))[:, None] * (x @ ts[b, h // 2])
            out[b, :n[b], h] = o / math.sqrt(d)
        for h in range(2):
            y, z = tk[b, :n[b], h], tv[b, :n[b], h]
            end[b, h] = math.exp(ld[h] * n[b]) * ts[b, h] + (torch.exp(ld[h] * (n[b] - 1 - i))[:, None] * y).T @ z
    got = mo.linear(q, k, v, ld, s0, lens)
    assert np.allclose(got[0], out.detach(), rtol=1e-12, atol=1e-12) and np.allclose(got[1], end.detach(), rtol=1e-12, atol=1e-12)
    grads = torch.autograd.grad((out, end), (tq, tk, tv, ts), (torch.tensor(dout), torch.tensor(ds)))
    for g, r in zip(mo.linear_backward(q, k, v, ld, dout, s0, ds, lens), grads):
        assert np.allclose(g, r, rtol=1e-12, atol=1e-12)


def test_window_sees_by_hand():
    assert mo.window_sees(5, 9, 2, 1) == [0, 4, 5]
    assert mo.window_sees(5, 9, 6, 0) == [0, 1, 2, 3, 4, 5]
    assert mo.window_sees(0, 9, 1, 8) == [0]            # a sink that is still to come is not seen
    assert mo.window_sees(3, 9, 1, 2) == [0, 1, 3]


@pytest.mark.parametrize("window,n_sink,Tq,lens", [(3, 0, 9, None), (2, 2, 9, [9, 4]), (1, 1, 5, [0, 7]), (50, 3, 9, None), (4, 20, 1, None)])
def test_window_oracle_is_the_masked_softmax_and_its_gradient_autograds(window, n_sink, Tq, lens):
    q, k, v, dout = problem(3, Tq=Tq)
    B, _, Hq, d = q.shape
    Tk = 9
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    t, j = np.arange(Tq)[:, None] + Tk - Tq, np.arange(Tk)[None]
    out, lse = torch.zeros(q.shape, dtype=torch.float64), np.full((B, Tq, Hq), -np.inf)
    for b in range(B):
        n = Tk if lens is None else lens[b]
        mask = torch.tensor((j <= t) & ((j > t - window) | (j < n_sink)) & (j < n) & (t < n))
        rows = mask.any(1)
        if not rows.any():
            continue
        for h in range(Hq):
            s = (tq[b, :, h] @ tk[b, :, h // 2].T / math.sqrt(d)).masked_fill(~mask, -torch.inf)[rows]
            out[b, rows, h] = torch.softmax(s, 1) @ tv[b, :, h // 2]
            lse[b, rows.numpy(), h] = torch.logsumexp(s, 1).detach()
    got = mo.window(q, k, v, window, n_sink, lens)
    assert np.allclose(got[0], out.detach(), rtol=1e-12, atol=1e-12)
    assert np.array_equal(np.isfinite(lse), np.isfinite(got[1])) and np.allclose(got[1][np.isfinite(lse)], lse[np.isfinite(lse)], rtol=1e-12)
    grads = torch.autograd.grad(out, (tq, tk, tv), torch.tensor(dout))
    mine = mo.window_backward(q, k, v, dout, window, n_sink, lens)
    bound = mo.window_backward(q, k, v, dout, window, n_sink, lens, absolute=True)
    for g, r, m in zip(mine, grads, bound):
        assert np.allclose(g, r, rtol=1e-12, atol=1e-12) and np.all(m >= np.abs(g) * (1 - 1e-12))


def test_oracle_gradients_are_slopes():
    """Central differences of <dout, out> along random directions: the step's square and 2^-52 / step, relative."""
    q, k, v, dout = problem(5)
    rng = np.random.default_rng(6)
    ld, s0 = np.array([-0.3, -0.02]), rng.standard_normal((2, 2, 3, 3))
    cases = [(lambda a: mo.linear(a[0], a[1], a[2], ld, a[3])[0], [q, k, v, s0], mo.linear_backward(q, k, v, ld, dout, s0)),
             (lambda a: mo.window(*a, 3, 1)[0], [q, k, v], mo.window_backward(q, k, v, dout, 3, 1))]
    for f, args, grads in cases:
        for i, g in enumerate(grads):
            way = rng.standard_normal(args[i].shape)
            step = lambda h: [x + h * way if j == i else x for j, x in enumerate(args)]
            h = 1e-5
            slope = ((f(step(h)) - f(step(-h))) * dout).sum() / (2 * h)
            assert abs(slope - (g * way).sum()) <= 1e-7 * (1 + np.abs(g * way).sum())


def test_strides_of_axes_of_one_entry():
    """Such an axis is never stepped along: its stride, which may be anything, is not looked at."""
    q = torch.empty(64).as_strided((1, 1, 1, 64), (3, 5, 7, 1))
    k = torch.empty(2, 9, 1, 64).as_strided((2, 9, 1, 64), (9 * 64, 64, 1, 1))
    s = kb._row_strides(q, k, k, q)
    assert (s.q_b, s.q_t, s.q_h) == (64, 64, 64) and (s.k_b, s.k_t, s.k_h) == (576, 64, 64) and (s.o_b, s.o_t, s.o_h) == (64, 64, 64)
    wide = torch.empty(2, 9, 3, 128)[:, :, :, :64]
    assert (kb._row_strides(wide, k, k, wide).q_t, kb._row_strides(wide, k, k, wide).q_h) == (384, 128)


def test_tensors_of_the_host_are_refused():
    q, k, pos = torch.zeros(1, 4, 2, 64), torch.zeros(1, 4, 2, 64), torch.zeros(1, dtype=torch.int32)
    cache, state, ld = torch.zeros(1, 2, 5, 64), torch.zeros(1, 2, 64, 64), torch.zeros(2)
    for call in (lambda: kb.window_prefill(q, k, k, window=3), lambda: kb.window_fill(cache, cache, k, k, window=5),
                 lambda: kb.window_decode(cache, cache, q[:, 0], k[:, 0], k[:, 0], pos, window=5),
                 lambda: kb.window_backward(q, k, k, q, torch.zeros(1, 4, 2), q, window=3), lambda: kb.linear_prefill(q, k, k, ld),
                 lambda: kb.linear_backward(q, k, k, ld, q), lambda: kb.linear_decode(state, q[:, 0], k[:, 0], k[:, 0], ld)):
        with pytest.raises(ValueError, match="GPU"):
            call()
