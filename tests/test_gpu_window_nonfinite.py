"""Prompts of window attention with a value that is not finite in q, k or v: which results it reaches, whatever its key's place in the
query's order of keys.  Calls of one sequence (the waves of a workgroup share key tiles) and of 132 (they do not: 792 workgroups
at least, or 1320 where each has the four heads of a group).

What the definition gives is worked out by the numpy oracle with the affected queries left out; the bounds of the others are those of
test_gpu_window: a query done again key by key has fewer roundings than they allow."""
import numpy as np
import pytest
import torch

from oracle import mixers_oracle as mo
from test_gpu_window import f64, make, noise, out_bound, within

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
KINDS = [("bf16", 128, 4, 1), ("bf16", 64, 2, 2), ("f32", 64, 2, 1), ("f32", 128, 4, 4)]
SIZES = [(1, 290), (132, 290)]   # (with lse, 290 keys of a window beyond 64 are more than the rows with two operands for P have)


def prefill(x, n, **kw):
    """The one sequence of x, n times; every copy gives the same bits (NaN for NaN)."""
    import paper_2605_09877_amd as kvm
    many = [x[m].expand(n, -1, -1, -1).contiguous() for m in "qkv"]
    out, lse = kvm.window_prefill(*many, want_lse=True, **kw)
    plain = kvm.window_prefill(*many, **kw)
    for t in (out, lse, plain):
        assert torch.equal(t.nan_to_num(nan=12345.0), t[:1].nan_to_num(nan=12345.0).expand_as(t))
    return out[:1], lse[:1], plain[:1]


def check(io, clean, got, window, n_sink, bad):
    """bad [T, Hq] or [T, Hq, d]: results that have to be NaN; the others are the clean problem's."""
    out, lse, plain = got
    y = {n: f64(t) for n, t in clean.items()}
    ref, rlse = mo.window(y["q"], y["k"], y["v"], window, n_sink)
    tol = out_bound(io, clean, ref, window, n_sink, None, None)
    rows = bad if bad.ndim == 2 else np.zeros(bad.shape[:2], bool)
    every = np.broadcast_to(bad if bad.ndim == 3 else bad[:, :, None], ref.shape[1:])
    for o in (out, plain):
        o = f64(o)
        assert np.array_equal(np.isnan(o[0]), every), np.argwhere(np.isnan(o[0]) != every)[:5]
        within(torch.as_tensor(np.where(every, 0, o[0])), np.where(every, 0, ref[0]), tol[0], "out")
    lse = f64(lse)[0]
    assert np.array_equal(np.isnan(lse), rows)
    # (bf16: the sum is over P as rounded, 2^-8 of it at most)
    tol = (2.0 ** -8 if io == "bf16" else 0) + noise(clean, None, ref.shape[1]) * (2 + np.abs(rlse).max())
    assert np.all(np.abs(lse - rlse[0])[~rows] <= tol)


@pytest.mark.parametrize("n,T", SIZES)
@pytest.mark.parametrize("io,d,Hq,Hkv", KINDS)
def test_a_query_that_is_not_a_number(io, d, Hq, Hkv, n, T):
    """NaN in one channel of one head's query: its row is NaN, its lse too, and no other's."""
    x = make(io, 1, T, T, Hq, Hkv, d)
    got_x = {m: t.clone() for m, t in x.items()}
    bad = np.zeros((T, Hq), bool)
    for t, h in ((0, 0), (77, Hq - 1), (T - 1, 0)):
        got_x["q"][0, t, h, 5] = NAN
        bad[t, h] = True
    check(io, x, prefill(got_x, n, window=90, n_sink=3), 90, 3, bad)


@pytest.mark.parametrize("n,T", SIZES)
@pytest.mark.parametrize("io,d,Hq,Hkv", KINDS)
@pytest.mark.parametrize("window,n_sink,key", [(90, 0, 0), (90, 0, 130), (1, 0, 40), (90, 2, 0), (90, 2, 1), (300, 0, 0), (70, 1, 130)])
def test_a_key_that_is_not_a_number(io, d, Hq, Hkv, n, T, window, n_sink, key):
    """Every query that sees it is NaN: also where it is the first key seen (key 0, a sink, the oldest of the window) or the only one."""
    x = make(io, 1, T, T, Hq, Hkv, d)
    got_x = {m: t.clone() for m, t in x.items()}
    got_x["k"][0, key, 0, 7] = NAN
    bad = np.zeros((T, Hq), bool)
    for t in range(key, T):
        bad[t, :Hq // Hkv] = t - key < window or key < n_sink
    check(io, x, prefill(got_x, n, window=window, n_sink=n_sink), window, n_sink, bad)


@pytest.mark.parametrize("n,T", SIZES)
@pytest.mark.parametrize("io,d,Hq,Hkv", KINDS)
@pytest.mark.parametrize("key", [0, 120])
def test_a_value_behind_a_key_of_no_weight(io, d, Hq, Hkv, n, T, key):
    """A key of -infinity (q is positive) has weight 0, and 0 times a NaN value is NaN, wherever the key stands; in that channel alone."""
    x = make(io, 1, T, T, Hq, Hkv, d)
    x["q"] = x["q"].abs() + 0.5
    got_x = {m: t.clone() for m, t in x.items()}
    got_x["k"][0, key, 0, 7] = -INF
    got_x["v"][0, key, 0, 3] = NAN
    W = 90
    bad = np.zeros((T, Hq, d), bool)
    bad[key:key + W, :Hq // Hkv, 3] = True
    out, _, plain = prefill(got_x, n, window=W)
    y = {m: f64(t) for m, t in got_x.items()}
    y["k"][0, key, 0, 7] = -1e300
    y["v"][0, key, 0, 3] = 0
    alone = np.zeros((T, Hq), bool)
    alone[0, :Hq // Hkv] = key == 0      # (query 0 sees this key alone: no logit above -infinity, zeros)
    bad[alone] = False
    ref = mo.window(y["q"], y["k"], y["v"], W)[0]
    ref[0][alone] = 0
    mag = mo.window(y["q"], y["k"], np.abs(y["v"]), W)[0]
    tol = noise(x, None, W) * mag + (2.0 ** -8 * (2 * np.abs(ref) + mag) if io == "bf16" else 0)
    for o in (out, plain):
        o = f64(o)[0]
        assert np.array_equal(np.isnan(o), bad), np.argwhere(np.isnan(o) != bad)[:5]
        within(torch.as_tensor(np.where(bad, 0, o)), np.where(bad, 0, ref[0]), tol[0], "out")


@pytest.mark.parametrize("n", [1, 132])
@pytest.mark.parametrize("io,d,Hq,Hkv", KINDS)
def test_logits_of_infinity(io, d, Hq, Hkv, n):
    """A key with a logit of +infinity: infinity less itself is NaN for every query that sees it, first of its keys or not."""
    x = make(io, 1, 290, 290, Hq, Hkv, d)
    x["q"] = x["q"].abs() + 0.5
    for key in (0, 100):
        got_x = {m: t.clone() for m, t in x.items()}
        got_x["k"][0, key, 0, 7] = INF
        bad = np.zeros((290, Hq), bool)
        bad[key:key + 80, :Hq // Hkv] = True
        out, lse, plain = prefill(got_x, n, window=80)
        for o in (out, plain):
            assert np.array_equal(torch.isnan(o[0]).all(-1).cpu().numpy(), bad) and np.array_equal(torch.isnan(o[0]).any(-1).cpu().numpy(), bad)
