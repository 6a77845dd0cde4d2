"""Rotary positions with several axes over device tensors (argument marshalling
for ``statekv_mrope``)."""
from __future__ import annotations

import functools

import torch

from .statekv import check, packed_call, raw_stream, statekv_mrope_args


def mrope_frequencies(sections, theta: float, *, interleaved=False, per_axis=False):
    """(freq, axis) of the rotated pairs: CPU tensors fp64 and int32 [sum(sections)].

    ``sections[a]`` pairs turn by axis ``a``, in runs (time, height, width), or
    with ``interleaved`` taking turns over the axes while they have pairs left.
    Pair p of P turns at theta^(-p/P) per position; with ``per_axis`` pair i of an
    axis' n turns at theta^(-i/n)."""
    if interleaved:
        axis, left = [], list(sections)
        while any(left):
            for a, n in enumerate(left):
                if n:
                    axis.append(a)
                    left[a] -= 1
    else:
        axis = [a for a, n in enumerate(sections) for _ in range(n)]
    P, seen, freq = len(axis), [0] * len(sections), []
    for p, a in enumerate(axis):
        freq.append(theta ** -(seen[a] / sections[a] if per_axis else p / P))
        seen[a] += 1
    return torch.tensor(freq, dtype=torch.float64), torch.tensor(axis, dtype=torch.int32)


@functools.cache
def _call():
    return packed_call("statekv_mrope", statekv_mrope_args, "8if3Pq4P4q")


def _rows(x, tokens, heads, d, device, name):
    """Elements between the tokens of x, which has to be bf16 [tokens][heads][d] on
    the positions' device with contiguous tokens."""
    st = x.stride()
    if x.dtype != torch.bfloat16 or x.shape != (tokens, heads, d) or st[2] != 1 or \
            (st[1] != d and heads > 1) or x.get_device() != device:
        raise ValueError(f"{name}: a bf16 tensor {(tokens, heads, d)} on the positions' device whose tokens are "
                         "contiguous rows")
    return st[0] if tokens > 1 else heads * d


class _Turn(torch.autograd.Function):
    """``mrope`` and, as its gradient, the call that turns the other way."""

    @staticmethod
    def forward(ctx, q, k, positions, freq, axis, how, transpose, stream):
        ctx.save_for_backward(positions, freq, axis)  # autograd refuses them once changed in place
        ctx.set_materialize_grads(False)
        ctx.how, ctx.transpose = how, transpose
        return mrope(q, k, positions, freq, axis, transpose=transpose, stream=stream, **how)

    @staticmethod
    def backward(ctx, dq, dk):
        dq, dk = (x.contiguous() if x is not None and wanted else None
                  for x, wanted in zip((dq, dk), ctx.needs_input_grad))
        if dq is not None or dk is not None:
            dq, dk = mrope(dq, dk, *ctx.saved_tensors, transpose=not ctx.transpose, **ctx.how)
        return dq, dk, None, None, None, None, None, None


def mrope(q, k, positions, freq, axis, *, scale=1.0, adjacent=False, transpose=False, q_out=None,
          k_out=None, stream=None):
    """q and k (bf16 [tokens][heads][d], the rows of a token contiguous; either may
    be None) turned at ``positions`` (int32 [axes][tokens], device; for text, whose
    axes are equal, ``expand`` of one row will do); returns (q_out, k_out), made here
    unless given (``q_out=q`` turns in place).
    ``freq``, ``axis``: CPU tensors as from ``mrope_frequencies``.  ``transpose``
    turns the other way: the gradient with respect to q and k, which autograd forms
    for those that require one (not with ``q_out`` or ``k_out``).  Raises StateKVError
    on a bad argument."""
    if q is None and k is None:
        raise ValueError("q and k are both None")
    if ((q is not None and q.requires_grad) or (k is not None and k.requires_grad)) and torch.is_grad_enabled():
        if q_out is not None or k_out is not None:
            raise ValueError("q_out, k_out: not for q or k that require a gradient")
        return _Turn.apply(q, k, positions, freq, axis, dict(scale=scale, adjacent=adjacent), transpose, stream)
    tokens, _, d = (k if q is None else q).shape
    pairs, (axes, width), ps = freq.numel(), positions.shape, positions.stride()
    if freq.dtype != torch.float64 or axis.dtype != torch.int32 or axis.numel() != pairs or \
            freq.is_cuda or axis.is_cuda or not freq.is_contiguous() or not axis.is_contiguous():
        raise ValueError("freq and axis: contiguous CPU tensors, fp64 and int32, one entry per pair")
    device = positions.get_device()  # -1: not a device tensor
    if positions.dtype != torch.int32 or width < tokens or (ps[1] != 1 and width > 1) or device < 0:
        raise ValueError("positions: an int32 device tensor [axes][tokens]")
    axis_stride = ps[0] if axes > 1 else width  # of one axis it has no meaning
    if 0 < axis_stride < tokens:
        raise ValueError("positions: axes that overlap (expanded from one, or at least a call's tokens apart)")
    hq = hk = q_ptr = k_ptr = qo_ptr = ko_ptr = qs = ks = qos = kos = 0
    if q is not None:
        hq = q.shape[1]
        qs = _rows(q, tokens, hq, d, device, "q")
        if q_out is None:
            q_out, qos = torch.empty((tokens, hq, d), dtype=torch.bfloat16, device=q.device), hq * d
        else:
            qos = _rows(q_out, tokens, hq, d, device, "q_out")
        q_ptr, qo_ptr = q.data_ptr(), q_out.data_ptr()
    if k is not None:
        hk = k.shape[1]
        if k.shape[0] != tokens or k.shape[2] != d:
            raise ValueError("k: other tokens or another head dim than q")
        ks = _rows(k, tokens, hk, d, device, "k")
        if k_out is None:
            k_out, kos = torch.empty((tokens, hk, d), dtype=torch.bfloat16, device=k.device), hk * d
        else:
            kos = _rows(k_out, tokens, hk, d, device, "k_out")
        k_ptr, ko_ptr = k.data_ptr(), k_out.data_ptr()
    call, pack = _call()
    check(call(pack(tokens, hq, hk, d, axes, pairs, adjacent, transpose, scale, freq.data_ptr(), axis.data_ptr(),
                    positions.data_ptr(), axis_stride, q_ptr, k_ptr, qo_ptr, ko_ptr, qs, ks, qos, kos),
               raw_stream(stream, positions)), "statekv_mrope")
    return q_out, k_out
