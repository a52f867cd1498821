"""Outputs of the mixers whose strides make rows share memory: refused before any launch (what the rows would hold depends on the order
in which workgroups write them).  No GPU."""
import ctypes as C

import pytest

from paper_2605_09877_amd import binding as kb

P = 0x10000000   # aligned, never dereferenced: every call below returns an error first
B, T, HQ, HKV, D = 2, 70, 4, 2, 64
DENSE = dict(b=T * HQ * D, t=HQ * D, h=D)


def strides(o, lse=None):
    s = kb.kvm_strides()
    for n, h in (("q", HQ), ("k", HKV), ("v", HKV)):
        setattr(s, n + "_b", T * h * D)
        setattr(s, n + "_t", h * D)
        setattr(s, n + "_h", D)
    s.o_b, s.o_t, s.o_h = o["b"], o["t"], o["h"]
    s.lse_b, s.lse_t, s.lse_h = lse or (T * HQ, HQ, 1)
    return C.byref(s)


def window(s, lse=P):
    cfg = kb.kvm_window_config(B, HQ, HKV, D, kb.KVM_F32, 4, 100, 0.0)
    return kb.load_library().kvm_window_prefill(cfg, P, P, P, None, P, None, lse, T, T, s, None)


def linear(s):
    cfg = kb.kvm_linear_config(B, HQ, HKV, D, kb.KVM_F32, 0.0)
    return kb.load_library().kvm_linear_prefill(cfg, P, P, P, P, None, None, P, None, T, s, P, 1 << 62, None)


@pytest.mark.parametrize("bad", [dict(b=0), dict(t=D), dict(b=HQ * D), dict(h=HQ * D, t=HQ * D), dict(b=(T - 1) * HQ * D),
                                 dict(t=(HQ - 1) * D, b=T * HQ * D), dict(b=T * HQ * D - 4)], ids=str)
def test_rows_that_share_memory(bad):
    s = strides(DENSE | bad)
    assert window(s) == linear(s) == kb.KVM_ERR_ARG


@pytest.mark.parametrize("bad", [(0, HQ, 1), (T * HQ, 1, 1), (T * HQ - 1, HQ, 1), (T * HQ, HQ, HQ), (HQ, HQ, 1)], ids=str)
def test_sums_that_share_memory(bad):
    assert window(strides(DENSE, bad)) == kb.KVM_ERR_ARG
