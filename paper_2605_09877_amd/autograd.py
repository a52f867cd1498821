"""torch.autograd front end of the layer, and of the mixers beside it: one differentiable call for a whole sequence.

Marshalling only.  The forward is kvm_prefill_chunked on a fresh state with the fold record
switched on; the backward is kvm_prefill_backward on that state.  Every step runs in the
library's HIP kernels.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd import forward_ad

from .binding import (KVM_BF16, KVM_BUDGET_FIXED, KVM_F32, KVMState, _number, _sizes, _steps, linear_backward, linear_prefill,
                      window_backward, window_prefill)


class _KVMAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, gate, ln_gamma, ln_beta, tau_state, tau_bswa, cfg: dict):
        B, T, Hq, d = q.shape
        Hkv = k.shape[2]
        st = KVMState(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d,
                      io_dtype=KVM_BF16 if q.dtype == torch.bfloat16 else KVM_F32,
                      ln_gamma=ln_gamma, ln_beta=ln_beta, tau_state=tau_state, tau_bswa=tau_bswa,
                      max_tokens=T, device=str(q.device), **cfg)
        n_folds = T // cfg["chunk_len"] + 1
        assign, score = st._record(n_folds)   # (the backward pass reads the folds done alone)
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        gate = None if gate is None else gate.to(torch.float32).contiguous()
        out, lse = st.prefill(q, k, v, gate, want_lse=True)
        ctx.state, ctx.record = st, (assign, score)
        ctx.save_for_backward(q, k, v, gate if gate is not None else q.new_empty(0), out, lse)
        ctx.has_gate = gate is not None
        ctx.param_shapes = tuple(None if p is None else (p.dtype, p.shape) for p in (ln_gamma, ln_beta, tau_state, tau_bswa))
        return out

    @staticmethod
    def backward(ctx, dout):
        q, k, v, gate, out, lse = ctx.saved_tensors
        assign, score = ctx.record
        g = ctx.state.backward(q, k, v, gate if ctx.has_gate else None, out, lse, dout.contiguous(), assign, score)
        ctx.state.close()
        params = []
        for name, spec in zip(("dgamma", "dbeta", "dtau_state", "dtau_bswa"), ctx.param_shapes):
            params.append(None if spec is None else g[name].to(spec[0]).reshape(spec[1]))
        return (g["dq"], g["dk"], g["dv"], g["dgate"] if ctx.has_gate else None, *params, None)


def kvm_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, gate: Optional[torch.Tensor] = None, *,
                  chunk_len: int, rope_dims: int, n_bswa_chunks: int = 2, n_sink: int = 1,
                  budget_kind: int = KVM_BUDGET_FIXED, budget_fixed: int = 0, budget_scale: float = 0.0,
                  budget_table=None, ln_gamma: Optional[torch.Tensor] = None, ln_beta: Optional[torch.Tensor] = None,
                  tau_state: Optional[torch.Tensor] = None, tau_bswa: Optional[torch.Tensor] = None,
                  ln_eps: float = 1e-5, norm_eps: float = 1e-12) -> torch.Tensor:
    """The KVM layer over a whole sequence from an empty state, differentiable in q, k, v, the merge
    gate, the LN_s parameters and the temperatures.  q [B, T, Hq, d]; k, v [B, T, Hkv, d] (bf16 or
    fp32, prepared: normalised and rotated); gate [B, T, Hkv] fp32 or None.  Returns out like q."""
    cfg = dict(chunk_len=chunk_len, rope_dims=rope_dims, n_bswa_chunks=n_bswa_chunks, n_sink=n_sink,
               budget_kind=budget_kind, budget_fixed=budget_fixed, budget_scale=budget_scale,
               budget_table=budget_table, ln_eps=ln_eps, norm_eps=norm_eps)
    return _KVMAttention.apply(q, k, v, gate, ln_gamma, ln_beta, tau_state, tau_bswa, cfg)


def _once(ctx) -> None:
    """A gradient of these gradients does not exist: refused where one is asked for (create_graph), not left out."""
    if torch.is_grad_enabled():
        raise RuntimeError(f"{type(ctx).__name__}: the gradients are not differentiable again (create_graph)")


def _gradient_wanted(*tensors) -> bool:
    """Also of tensors with tangents (forward mode), which autograd.Function refuses."""
    tensors = [t for t in tensors if t is not None]
    return torch.is_grad_enabled() and any(t.requires_grad for t in tensors) or (
        forward_ad._current_level >= 0 and any(forward_ad.unpack_dual(t).tangent is not None for t in tensors))


def _rows(t: torch.Tensor) -> torch.Tensor:
    """t where the forward calls take it as it lies, a dense copy otherwise (broadcast heads, rows off 16-byte borders, ..)."""
    if t.dim() != 4 or t.numel() == 0:
        return t
    (b, row, head), d, vec = _steps(t), t.shape[3], 16 // t.element_size()
    apart = b % vec == row % vec == head % vec == 0 and head >= d and d <= row <= 1 << 23
    return t if apart and t.stride(3) == 1 and t.data_ptr() % 16 == 0 else t.contiguous()


class _LinearAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, state, lens, scale):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        keep = []
        out, end = linear_prefill(q, k, v, log_decay, state=state, lens=lens, scale=scale, keep=keep)
        ctx.save_for_backward(q, k, v, log_decay, state, lens, *keep)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return out, end

    @staticmethod
    def backward(ctx, dout, dend):
        _once(ctx)
        q, k, v, log_decay, state, lens, kept = ctx.saved_tensors
        dout = torch.zeros_like(q) if dout is None else dout.contiguous()
        dend = None if dend is None else dend.contiguous()
        dq, dk, dv, dstate = linear_backward(q, k, v, log_decay, dout, state=state, dstate_out=dend, lens=lens, scale=ctx.scale,
                                             want_dstate=state is not None and ctx.needs_input_grad[4], kept=kept)
        return dq, dk, dv, None, dstate, None, None


def kvm_linear_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_decay: torch.Tensor, *,
                         state: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None,
                         scale: Optional[float] = None):
    """Linear attention with a decay for each KV head over a whole sequence, differentiable in q, k, v and the state it
    starts from: S_t = exp(log_decay) S_{t-1} + k_t v_t^T, out_t = scale q_t S_t.  Shapes and lens as in linear_prefill.  The decays
    are constants of the layer: a log_decay that requires a gradient is refused.  Returns (out, state behind the last token).
    The backward pass reads `state` again and raises an error if it has been advanced in place (linear_decode) since."""
    if log_decay.requires_grad:
        raise ValueError("log_decay: the decays are constants, they get no gradient")
    if not _gradient_wanted(q, k, v, state):   # (the same bits, no copies of rows)
        return linear_prefill(_rows(q), _rows(k), _rows(v), log_decay, state=state, lens=lens, scale=scale)
    return _LinearAttention.apply(q, k, v, log_decay, state, lens, _number(scale))


class _WindowAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, window, n_sink, lens, scale):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        rest = torch.empty_like(q) if q.dtype is torch.bfloat16 else None   # (D = dout . out to 16 bits of out)
        out, lse = window_prefill(q, k, v, window=window, n_sink=n_sink, lens=lens, scale=scale, want_lse=True, out_rest=rest)
        ctx.save_for_backward(q, k, v, lens, out, rest, lse)
        ctx.window, ctx.n_sink, ctx.scale = window, n_sink, scale
        return out

    @staticmethod
    def backward(ctx, dout):
        _once(ctx)
        q, k, v, lens, out, rest, lse = ctx.saved_tensors
        dq, dk, dv = window_backward(q, k, v, out, lse, dout.contiguous(), window=ctx.window, n_sink=ctx.n_sink, lens=lens,
                                     scale=ctx.scale, out_rest=rest)
        return dq, dk, dv, None, None, None, None


def kvm_window_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, window: int, n_sink: int = 0,
                         lens: Optional[torch.Tensor] = None, scale: Optional[float] = None) -> torch.Tensor:
    """Attention over the last `window` keys and the first `n_sink` ones, differentiable in q, k and v.  Shapes and lens as in
    window_prefill."""
    if not _gradient_wanted(q, k, v):   # (the same bits, which follow lse being asked for, and neither copies of rows nor out_rest)
        return window_prefill(_rows(q), _rows(k), _rows(v), window=window, n_sink=n_sink, lens=lens, scale=scale, want_lse=True)[0]
    return _WindowAttention.apply(q, k, v, *_sizes(window, n_sink), lens, _number(scale))
