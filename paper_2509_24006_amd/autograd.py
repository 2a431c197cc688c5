"""torch.autograd wrapper over the C-ABI calls of binding.py (fine-tuning use of Section 5).

    O = sla_attention(Q, K, V, W, k_h=0.05, k_l=0.10)

runs sla_build_mask + sla_forward and records sla_backward; every step is a kernel of
libsla_hip.so, this module only keeps the buffers alive between the two passes.  The mask is a
constant of the graph (no gradient flows into the block scores); a mask built once can be passed
back in through `mask=` and reused, e.g. across the steps of a diffusion sampler.

The layers around it:

    O = dense_attention(Q, K, V, causal=..., k_len=..., table=..., buckets=position_buckets(32, 128))
    O = cached_attention(Q, K_cache, V_cache, k_len=lengths, prefix=(K_prompt, V_prompt))

softmax attention with gradients (cross attention, dense or causal layers, shared K, V heads, learned position
bias), and its serving form for the newest tokens of every sequence of a batch.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd import forward_ad

from . import binding as sla
from .binding import position_buckets  # noqa: F401  (the buckets of dense_attention's and cached_attention's bias)


class _SLAFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, W, p, Mc, luts, grad):
        # the library reads W in the storage type of Q, K, V (a float parameter next to bf16
        # activations is cast here; its gradient goes back in the parameter's own type)
        ctx.w_dtype = W.dtype
        W = W.detach()
        if W.dtype != Q.dtype or not W.is_contiguous():
            W = W.to(Q.dtype).contiguous()
        # without a backward pass to come (grad false) O^s, O^l, L stay on the chip and H, Z in the
        # workspace: two thirds of the forward kernel's stores (16 x 16 heads x 1024 tokens, d = 64: 53 -> 46 us)
        if Mc is None:
            Mc, luts, O, saved = sla.sla_mask_forward(p, Q, K, V, W, need_saved=grad)
        else:
            O, saved = sla.sla_forward(p, Q, K, V, W, Mc, luts, need_saved=grad)
        if grad:
            ctx.p = p
            ctx.save_for_backward(Q, K, V, W, Mc, luts, saved)
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, W, Mc, luts, saved = ctx.saved_tensors
        dt = torch.bfloat16 if ctx.w_dtype == torch.bfloat16 else torch.float32
        dQ, dK, dV, dW = sla._backward(ctx.p, Q, K, V, W, Mc, luts, saved, dO.contiguous(), None, None, dt)
        return dQ, dK, dV, dW.to(ctx.w_dtype), None, None, None, None


def _params(Q, k_h, k_l, phi, token_major, bq) -> sla.sla_params:
    if token_major:
        B, N, H, d = Q.shape
    else:
        B, H, N, d = Q.shape
    return sla.make_params(B, H, N, d, k_h, k_l, Q.dtype, phi=phi, bq=bq,
                           layout=sla.SLA_BNHD if token_major else sla.SLA_BHND)


def build_mask(Q: torch.Tensor, K: torch.Tensor, k_h: float, k_l: float,
               phi: int = sla.SLA_PHI_SOFTMAX, token_major: bool = False, bq: int = 64
               ) -> Tuple[sla.sla_params, torch.Tensor, torch.Tensor]:
    """(params, M_c int8 [B,H,ceil(N/bq),ceil(N/64)], lookup tables) for contiguous [B,H,N,d]
    tensors, or [B,N,H,d] ones with token_major.  bq: query block size of the mask (64 .. 256)."""
    p = _params(Q, k_h, k_l, phi, token_major, bq)
    Mc, luts, _ = sla.sla_build_mask(p, Q, K)   # (only the tensors' memory is handed on: no part of a graph)
    return p, Mc, luts


def sla_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, W: torch.Tensor,
                  k_h: float = 0.05, k_l: float = 0.10, phi: int = sla.SLA_PHI_SOFTMAX,
                  mask: Optional[Tuple[sla.sla_params, torch.Tensor, torch.Tensor]] = None,
                  token_major: bool = False, bq: int = 64) -> torch.Tensor:
    """O = O^s + Proj(O^l) (Eq. 6) with gradients to Q, K, V and the Proj weight W [d, d].
    Q, K, V (and O, and the gradients) are [B,H,N,d], or [B,N,H,d] with token_major -- the order
    in which a transformer block's projections leave them, no transpose needed."""
    p, Mc, luts = mask if mask is not None else (_params(Q, k_h, k_l, phi, token_major, bq), None, None)
    grad = torch.is_grad_enabled() and any(
        getattr(t, "requires_grad", False) for t in (Q, K, V, W))
    return _SLAFunction.apply(Q, K, V, W, p, Mc, luts, grad)


class _AttnFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Q, K, V, table, p, q_len, k_len, token_major):
        O, L = sla.sla_attn_forward(p, Q, K, V, table, q_len, k_len, token_major=token_major)
        ctx.p, ctx.token_major = p, token_major
        ctx.save_for_backward(Q, K, V, table, O, L, q_len, k_len)
        return O

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dO):
        _no_tangents("dense_attention's backward pass", dO)
        Q, K, V, table, O, L, q_len, k_len = ctx.saved_tensors
        grads = sla.sla_attn_backward(ctx.p, Q, K, V, O, _laid_out(dO, ctx.token_major), L, table, q_len, k_len, ctx.token_major)
        return (*grads, None, None, None, None)


def _no_trace(what: str):
    """A trace would record the allocation of the output and nothing that fills it."""
    if torch.jit.is_tracing():
        raise sla.SLAError(f"{what} cannot be traced")


def _no_tangents(what: str, *tensors):
    """Refuses inputs of forward-mode differentiation: the kernels would take them for constants."""
    if any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise sla.SLAError(f"{what} has no forward-mode derivative")


def _laid_out(t: torch.Tensor, token_major: bool) -> torch.Tensor:
    """The tensor itself where the library reads its strides (features contiguous, everything at multiples of 16
    bytes, rows next to or apart from each other), else a copy of it."""
    s, n, q, rows = t.stride(), t.shape, 16 // t.element_size(), t.dim() - (3 if token_major else 2)
    fits = s[-1] == 1 and t.data_ptr() % 16 == 0
    for i in range(t.dim() - 1):
        if n[i] > 1:
            fits = fits and s[i] % q == 0 and (i != rows or n[-1] <= s[i] <= (1 << 24) // t.element_size())
    return t if fits else t.clone(memory_format=torch.contiguous_format)   # (contiguous() would hand back a tensor at an odd address)


def _attn_params(Q, K, causal, scale, table, buckets, token_major, prefix_rows=0, from_end=False):
    if Q.dim() != 4 or K.dim() != 4:
        raise sla.SLAError("Q, K, V: expected tensors of four dimensions")
    if (table is None) != (buckets is None):
        raise sla.SLAError("table: a bias takes both, the buckets and the table")
    B, H, Nq, d = Q.shape if not token_major else (Q.shape[0], Q.shape[2], Q.shape[1], Q.shape[3])
    Hkv, Nk = (K.shape[2], K.shape[1]) if token_major else (K.shape[1], K.shape[2])
    return sla.make_attn_params(B, H, Hkv, Nq, Nk, d, Q.dtype, causal, scale, prefix_rows,
                                -Nq if from_end else Nk - Nq, from_end, buckets,
                                torch.float32 if table is None else table.dtype)


def _attend(Q, K, V, prefix, table, q_len, k_len, buckets, causal, scale, token_major, cached):
    """The call as compiled code makes it (csrc/host_calls.cpp), or None: the Python code then lays tensors out, goes through the
    same steps and raises what does not fit.  (A training step of 2 heads x 100 queries of 37 keys, d = 64, floats: 98 -> 67 us; one token over 1000, 12 heads: 14 -> 11.)"""
    Kp, Vp = (None, None) if prefix is None else prefix
    return sla._host_calls().attend(Q, K, V, Kp, Vp, table, q_len, k_len, 0 if buckets is None else sla.ctypes.addressof(buckets),
                                    causal, scale, token_major, cached)


def dense_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, causal: bool = False,
                    scale: Optional[float] = None, q_len: Optional[torch.Tensor] = None,
                    k_len: Optional[torch.Tensor] = None, table: Optional[torch.Tensor] = None,
                    buckets: Optional[sla.sla_buckets] = None, token_major: bool = False) -> torch.Tensor:
    """O = softmax(scale Q K^T + bias) V with gradients to Q, K, V and the bias table.

    Q [B,H,Nq,d], K, V [B,Hkv,Nk,d] with Hkv a divisor of H (query head h reads K, V head h // (H // Hkv)), or
    with token_major [B,Nq,H,d], [B,Nk,Hkv,d]; bf16 or float32, d 64 or 128; O as Q.  scale: 1 / sqrt(d) unless given.
    causal: query n sees the keys up to n + Nk - Nq.  q_len, k_len (int32 [B], on the device): valid queries and
    keys of every sequence; what lies behind them is not read, and comes back as zeros.  table [n_buckets,H] (float32
    or bf16) with buckets = position_buckets(...): table[bucket(key position - query position), head] is added
    to the scaled scores; an entry of -1e30 or below hides its pairs, and others should stay below 1e4 in magnitude where a row
    sees nothing else (its scores and their statistic are floats: the gradients are lost from 1e8 on).  A row that sees no key is
    zero.  Keys and values that only the causal order or the table hides have to be finite: they meet a probability of zero
    in a product.
    Forward-mode differentiation (dual tensors) and torch.jit.trace are refused, here and in cached_attention."""
    O = _attend(Q, K, V, None, table, q_len, k_len, buckets, causal, scale, token_major, False)
    if O is not None:
        return O
    _no_trace("dense_attention")
    _no_tangents("dense_attention", Q, K, V, table)
    Q, K, V = (_laid_out(t, token_major) for t in (Q, K, V))
    p = _attn_params(Q, K, causal, scale, table, buckets, token_major)
    if table is not None and not table.is_contiguous():
        table = table.contiguous()
    if torch.is_grad_enabled() and any(getattr(t, "requires_grad", False) for t in (Q, K, V, table)):
        return _AttnFunction.apply(Q, K, V, table, p, q_len, k_len, token_major)
    return sla.sla_attn_forward(p, Q, K, V, table, q_len, k_len, token_major=token_major, need_L=False)[0]


def cached_attention(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, k_len: Optional[torch.Tensor] = None,
                     prefix: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, causal: bool = True,
                     scale: Optional[float] = None, table: Optional[torch.Tensor] = None,
                     buckets: Optional[sla.sla_buckets] = None, token_major: bool = False) -> torch.Tensor:
    """Attention of the newest Nq tokens of every sequence over its cache, without gradients.

    K, V [B,Hkv,Nk,d] (token_major: [B,Nk,Hkv,d]) are the caches, the new tokens' rows among them; k_len (int32 [B]): rows
    that are in use, all unless given.  prefix = (K, V) [Hkv,Np,d] (token_major: [Np,Hkv,d]): rows that come before
    every sequence's own, fetched once for the whole batch.  The queries are the last Nq tokens in use (causal among
    themselves); a sequence with fewer than Nq of them, behind no prefix, has rows without a key, which are zeros."""
    O = _attend(Q, K, V, prefix, table, None, k_len, buckets, causal, scale, token_major, True)
    if O is not None:
        return O
    _no_trace("cached_attention")
    _no_tangents("cached_attention", Q, K, V, table, *(prefix or ()))
    with torch.no_grad():
        Q, K, V = (_laid_out(t, token_major) for t in (Q, K, V))
        if prefix is not None:
            prefix = tuple(_laid_out(t, token_major) for t in prefix)
        Np = 0 if prefix is None else prefix[0].shape[0 if token_major else 1]
        if prefix is not None and Np == 0:
            prefix = None
        p = _attn_params(Q, K, causal, scale, table, buckets, token_major, Np, True)
        if table is not None and not table.is_contiguous():
            table = table.contiguous()
        return sla.sla_attn_forward(p, Q, K, V, table, None, k_len, prefix, token_major, need_L=False)[0]
