"""Layers whose weight gradients come apart by language in one backward pass.

The resolve needs one gradient per language.  BucketMOO gets them from K
backward passes; where a batch holds the rows of all K languages one after
another, these layers give them in one: a linear layer's weight gradient is a
sum over rows, so language k's is the sum over its own rows
(bkmoo_gate_backward, bkmoo_language_wgrad).  `rows` are K + 1 bounds: language k
has the batch's rows from rows[k] to rows[k + 1].

Inside BucketMOO.begin_batch() ... finish() the gradients are added to the
parameters' `language_grads`, their places in the K flat buffers; outside, the
layers' weights receive the ordinary gradient of the whole batch.  The gradients
have no graph: gradients of gradients are refused.  Weights and
activations are bfloat16 on a GPU; the products that no language splits
(y = x W^T and its dx of LanguageLinear) are torch's.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import native


def _languages(weight, rows, T):
    """The language places of `weight` and its bounds, or one place for all of
    the batch."""
    places = getattr(weight, "language_grads", None)
    if places is not None:
        if rows is None or len(rows) != len(places) + 1:
            raise ValueError("rows must be the bounds of the %d languages" % len(places))
        return places, rows, None
    whole = torch.zeros_like(weight, memory_format=torch.contiguous_format)
    return [whole], [0, T], whole


def _enter(to):
    """Before a kernel writes what _languages gave: in the order of the streams
    (hook.LanguageGrads)."""
    if to is not None and hasattr(to[0], "enter"):
        to[0].enter()


def _leave(to):
    if to is not None and hasattr(to[0], "leave"):
        to[0].leave()


def _on_rows(t):
    """t as a matrix whose rows start on 16 bytes."""
    t = t.reshape(-1, t.shape[-1])
    n = t.shape[1]
    if t.stride(1) == 1 and t.stride(0) % 8 == 0 and t.stride(0) >= n and t.data_ptr() % 16 == 0:
        return t
    return t.new_empty(t.shape[0], (n + 7) // 8 * 8)[:, :n].copy_(t)


def _room(t, rows, cols):
    return t.new_empty(rows, (cols + 7) // 8 * 8)[:, :cols]


class _Gate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, act, rows):
        lead, m = x.shape[:-1], _on_rows(x)
        T, F = m.shape[0], w_gate.shape[0]
        g, u = _on_rows(w_gate), _on_rows(w_up)
        h = _room(m, T, F)
        a = b = None
        if any(ctx.needs_input_grad[:3]):
            a, b = _room(m, T, F), _room(m, T, F)
        native.bkmoo_gate_forward(m, g, u, act, h, a, b)
        ctx.save_for_backward(m, w_gate, w_up, a, b)
        ctx.act, ctx.rows, ctx.lead = act, rows, lead
        return h.view(*lead, F) if len(lead) != 1 else h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        m, w_gate, w_up, a, b = ctx.saved_tensors
        T, D = m.shape
        F = w_gate.shape[0]
        dx = _room(m, T, D) if ctx.needs_input_grad[0] else None
        dh, g, u = _on_rows(dh), _on_rows(w_gate), _on_rows(w_up)
        # [places, bounds, gradient of the whole batch or None] of the weights that are trained
        to = [_languages(w, ctx.rows, T) if need else None
              for w, need in zip((w_gate, w_up), ctx.needs_input_grad[1:3])]
        for t in to:
            _enter(t)
        if all(to) and (to[0][2] is None) == (to[1][2] is None):
            native.bkmoo_gate_backward(dh, a, b, m, g, u, ctx.act, to[0][1], dx, to[0][0], to[1][0],
                                       accumulate=True)
        elif not any(to):
            native.bkmoo_gate_backward(dh, a, b, m, g, u, ctx.act, [0, T], dx)
        else:
            # one of them is frozen, or they are apart by different bounds: da and db, which
            # the call leaves in its workspace, and each weight's gradients from its own
            ws = m.new_empty(native.bkmoo_gate_backward_workspace_size(T, F), dtype=torch.uint8)
            native.bkmoo_gate_backward(dh, a, b, m, g, u, ctx.act, [0, T],
                                       dx if dx is not None else _room(m, T, D), ws=ws)
            ld, half = (F + 7) // 8 * 8, ws.numel() // 2
            for i, place in enumerate(to):
                if place is not None:
                    d = ws[i * half:i * half + T * ld * 2].view(torch.bfloat16).view(T, ld)[:, :F]
                    native.bkmoo_language_wgrad(d, m, place[1], place[0], accumulate=True)
        for t in to:
            _leave(t)
        if dx is not None:
            dx = dx.reshape(*ctx.lead, D)
        return (dx, *(t[2] if t is not None else None for t in to), None, None)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, rows):
        ctx.save_for_backward(x, weight)
        ctx.rows = rows
        return torch.matmul(x, weight.t())

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        dx = torch.matmul(dy, weight) if ctx.needs_input_grad[0] else None
        whole = None
        if ctx.needs_input_grad[1]:
            m = _on_rows(x)
            to = places, rows, whole = _languages(weight, ctx.rows, m.shape[0])
            _enter(to)
            native.bkmoo_language_wgrad(_on_rows(dy), m, rows, places, accumulate=True)
            _leave(to)
        return dx, whole, None


class LanguageLinear(torch.nn.Module):
    """y = x W^T, W [out, in], without a bias."""

    def __init__(self, in_features: int, out_features: int, device="cuda"):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device,
                                                     dtype=torch.bfloat16))
        torch.nn.init.normal_(self.weight, std=in_features ** -0.5)

    def forward(self, x, rows=None):
        return _Linear.apply(x, self.weight, rows)


class GatedFeedForward(torch.nn.Module):
    """y = (act(x Wg^T) * (x Wu^T)) Wd^T; act "silu", "gelu" or "gelu_tanh"."""

    def __init__(self, width: int, hidden: int, act: str = "silu", device="cuda"):
        super().__init__()
        if act not in native.ACTS:
            raise ValueError("act must be one of %s, got %r" % (sorted(native.ACTS), act))
        self.act = act
        self.w_gate, self.w_up = (
            torch.nn.Parameter(torch.empty(hidden, width, device=device, dtype=torch.bfloat16))
            for _ in range(2))
        for w in (self.w_gate, self.w_up):
            torch.nn.init.normal_(w, std=width ** -0.5)
        self.down = LanguageLinear(hidden, width, device=device)

    def forward(self, x, rows=None):
        return self.down(_Gate.apply(x, self.w_gate, self.w_up, self.act, rows), rows)
