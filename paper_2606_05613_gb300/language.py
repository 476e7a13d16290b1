"""Layers whose weight gradients come apart by language in one backward pass.

The resolve needs one gradient per language.  BucketMOO gets them from K
backward passes; where a batch holds the rows of all K languages one after
another, these layers give them in one: a linear layer's weight gradient is a
sum over rows, so language k's is the sum over its own rows
(bkmoo_gate_backward, bkmoo_language_wgrad); so are an embedding's, over the rows
that hold a token, and that of the weights that scale normed queries and keys
(bkmoo_embedding_backward, bkmoo_qk_norm_backward).  `rows` are K + 1 bounds:
language k has the batch's rows from rows[k] to rows[k + 1].

Inside BucketMOO.begin_batch() ... finish() the gradients are added to the
parameters' `language_grads`, their places in the K flat buffers; outside, the
layers' weights receive the ordinary gradient of the whole batch.  The gradients
have no graph: gradients of gradients are refused.  Weights and
activations are bfloat16 on a GPU (an embedding's and the logits of
token_log_probs may be float32); the products that no language splits
(y = x W^T and its dx of LanguageLinear) are torch's.

The forward and the backward pass may be captured (torch.cuda.graph) on
begin_batch()'s stream, between it and finish(); a step is then begin_batch(),
a replay there and finish().  No graph of an eager pass over the same weights
may be alive during the capture: autograd would tie it to that pass's stream.
"""
from __future__ import annotations

import collections
import ctypes
import functools

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
        if all(to) and (to[0][2] is None) == (to[1][2] is None) and to[0][0] is not to[1][0]:
            native.bkmoo_gate_backward(dh, a, b, m, g, u, ctx.act, to[0][1], dx, to[0][0], to[1][0],
                                       accumulate=True)
        elif not any(to):
            native.bkmoo_gate_backward(dh, a, b, m, g, u, ctx.act, [0, T], dx)
        else:
            # one of them is frozen, they are apart by different bounds, or they are one parameter:
            # da and db, which the call leaves in its workspace, and each weight's gradients from its own
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


def _matrix(t):
    """t as a matrix with contiguous rows that do not overlap."""
    t = t.reshape(-1, t.shape[-1])
    return t if t.stride(1) == 1 and t.stride(0) >= t.shape[1] else t.contiguous()


def _on_heads(t):
    """t as [tokens, heads, width], a token's heads side by side and on 16 bytes."""
    heads, width = t.shape[-2:]
    t = t.reshape(-1, heads, width)
    ld, between, step = t.stride()
    if step == 1 and (between == width or heads == 1) and ld % 8 == 0 and ld >= heads * width and t.data_ptr() % 16 == 0:
        return t
    return torch.empty(t.shape, dtype=t.dtype, device=t.device).copy_(t)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, weight, scale, rows):
        flat = ids.reshape(-1).contiguous()
        # (results are no views, here and below: they may be changed in place)
        y = weight.new_empty(*ids.shape, weight.shape[1])
        native.bkmoo_embedding_forward(_matrix(weight), flat, y.view(-1, weight.shape[1]), scale)
        ctx.save_for_backward(flat, weight)
        ctx.scale, ctx.rows = scale, rows
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        flat, weight = ctx.saved_tensors
        if not ctx.needs_input_grad[1]:
            return None, None, None, None
        to = places, rows, whole = _languages(weight, ctx.rows, flat.numel())
        _enter(to)
        native.bkmoo_embedding_backward(_matrix(dy), flat, rows, places, ctx.scale, accumulate=True)
        _leave(to)
        return None, whole, None, None


class _QueryKeyNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, w_q, w_k, positions, inv_freq, eps, interleaved, rows):
        a, b = _on_heads(q), _on_heads(k)
        u, v = w_q.contiguous(), w_k.contiguous()
        pos = positions.reshape(-1).contiguous()
        qo, ko = torch.empty(q.shape, dtype=a.dtype, device=a.device), torch.empty(k.shape, dtype=b.dtype, device=b.device)
        native.bkmoo_qk_norm_forward(a, b, u, v, pos, inv_freq, qo.view(a.shape), ko.view(b.shape), eps, interleaved)
        ctx.save_for_backward(a, b, w_q, w_k, pos)
        ctx.fixed = inv_freq, eps, interleaved
        ctx.rows, ctx.shapes = rows, (q.shape, k.shape)
        return qo, ko

    @staticmethod
    @once_differentiable
    def backward(ctx, dqo, dko):
        q, k, w_q, w_k, pos = ctx.saved_tensors
        inv_freq, eps, interleaved = ctx.fixed
        T = q.shape[0]
        dqo, dko, u, v = _on_heads(dqo), _on_heads(dko), w_q.contiguous(), w_k.contiguous()
        dq, dk = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=k.dtype, device=k.device)
        # [places, bounds, gradient of the whole batch or None] of the weights that are trained
        to = [_languages(w, ctx.rows, T) if need else None for w, need in zip((w_q, w_k), ctx.needs_input_grad[2:4])]

        def call(rows, dw_q=None, dw_k=None):
            native.bkmoo_qk_norm_backward(dqo, dko, q, k, u, v, pos, inv_freq, rows, dq, dk, dw_q, dw_k, eps, interleaved,
                                          accumulate=True)

        for t in to:
            _enter(t)
        if all(to) and (to[0][2] is None) == (to[1][2] is None) and to[0][0] is not to[1][0]:
            call(to[0][1], to[0][0], to[1][0])
        elif not any(to):
            call([0, T])
        else:
            # one of them is frozen, they are apart by different bounds, or they are one parameter:
            # each with a place beside it for what the other one would get
            for i, t in enumerate(to):
                if t is not None:
                    other = [torch.zeros_like(g) for g in t[0]]
                    call(t[1], *((t[0], other) if i == 0 else (other, t[0])))
        for t in to:
            _leave(t)
        return (dq.view(ctx.shapes[0]), dk.view(ctx.shapes[1]), *(t[2] if t is not None else None for t in to),
                None, None, None, None, None)


class _TokenLogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, entropy, top):
        z, lead = _matrix(logits), logits.shape[:-1]
        t = targets.reshape(-1).contiguous()
        T = z.shape[0]
        f32 = dict(dtype=torch.float32, device=z.device)
        logp, stats = torch.empty(lead, **f32), torch.empty(T, 2, **f32)
        H = torch.empty(lead, **f32) if entropy else None
        ids = torch.empty(*lead, top, dtype=torch.int64, device=z.device) if top else None
        best = torch.empty(*lead, top, **f32) if top else None
        native.bkmoo_token_logp_forward(z, t, logp.view(T), stats, None if H is None else H.view(T),
                                        *((ids.view(T, top), best.view(T, top)) if top else ()))
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(z, t, stats, H)
        ctx.shape = logits.shape
        out = [logp]
        if entropy:
            out.append(H)
        if top:
            out += [ids, best]
            ctx.mark_non_differentiable(*out[-2:])
        return tuple(out)

    @staticmethod
    @once_differentiable
    def backward(ctx, g, *more):
        z, t, stats, H = ctx.saved_tensors
        h = more[0] if H is not None else None
        g = torch.zeros(z.shape[0], dtype=torch.float32, device=z.device) if g is None else g.reshape(-1).contiguous()
        dz = _room(z, *z.shape)
        native.bkmoo_token_logp_backward(z, t, stats, g, dz, None if H is None else H.view(-1),
                                         None if h is None else h.reshape(-1).contiguous())
        return dz.reshape(ctx.shape), None, None, None


TokenLogProbs = collections.namedtuple("TokenLogProbs", "logp entropy top_ids top_logp")


def token_log_probs(logits, targets, entropy=False, top=0):
    """Log probability of each row's target (0 where it is outside the vocabulary: padding), and
    where asked for the rows' entropy and their `top` (32 at most) most likely tokens with their
    log probabilities.  logits [..., vocabulary], float32 or bfloat16; targets [...], int64
    or int32.  logp and entropy have gradients; the backward pass reads entropy, so it is not to be
    changed in place ahead of that."""
    if targets.shape != logits.shape[:-1]:
        raise ValueError("one target for each row of logits, got %s and %s" % (tuple(targets.shape), tuple(logits.shape)))
    out = list(_TokenLogProbs.apply(logits, targets, entropy, top))
    logp = out.pop(0)
    H = out.pop(0) if entropy else None
    return TokenLogProbs(logp, H, *(out if top else (None, None)))


class Embedding(torch.nn.Module):
    """y = scale W[token], W [tokens, width]; 0 for a token outside the table (padding)."""

    def __init__(self, tokens: int, width: int, scale: float = 1.0, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.scale = scale
        self.weight = torch.nn.Parameter(torch.empty(tokens, width, device=device, dtype=dtype))
        torch.nn.init.normal_(self.weight, std=1.0 / max(abs(scale), 1.0))

    def forward(self, ids, rows=None):
        return _Embedding.apply(ids, self.weight, self.scale, rows)


# Arrays that kernels read; no caller is handed one.
_frequencies = functools.lru_cache(maxsize=64)(native.rope_frequencies)


@functools.lru_cache(maxsize=64)
def _given_frequencies(inv_freq):
    return (ctypes.c_double * len(inv_freq))(*inv_freq)


class QueryKeyNorm(torch.nn.Module):
    """Queries [..., heads, width] and keys [..., key heads, width] normed head by head, scaled by
    a weight each and their first `rotated` elements turned by the token's position: by
    base^(-2i / rotated) radians a position, or by `inv_freq`, rotated / 2 numbers of the layer's own."""

    _given = None

    def __init__(self, width: int, rotated=None, base: float = 10000.0, interleaved=False, eps: float = 1e-6, device="cuda",
                 inv_freq=None):
        super().__init__()
        self.eps, self.interleaved = eps, interleaved
        if inv_freq is not None:
            self._given = tuple(float(f) for f in inv_freq)
            rotated = 2 * len(self._given) if rotated is None else rotated
            if 2 * len(self._given) != rotated:
                raise ValueError("inv_freq must be rotated / 2 numbers, %d rotated, got %d" % (rotated, len(self._given)))
        rotated = width if rotated is None else rotated
        if rotated % 16 or not 0 <= rotated <= width:
            raise ValueError("rotated must be a multiple of 16 from 0 to the width, %d, got %s" % (width, rotated))
        self.rotated, self.base = rotated, base
        self.w_q, self.w_k = (torch.nn.Parameter(torch.ones(width, device=device, dtype=torch.bfloat16)) for _ in range(2))

    def _array(self):
        return _frequencies(self.rotated, self.base) if self._given is None else _given_frequencies(self._given)

    @property
    def inv_freq(self):
        """The frequencies, a copy."""
        return tuple(self._array())

    def forward(self, q, k, positions, rows=None):
        if q.shape[:-2] != k.shape[:-2] or positions.shape != q.shape[:-2]:
            raise ValueError("queries, keys and positions must have the same tokens, got %s, %s and %s"
                             % (tuple(q.shape[:-2]), tuple(k.shape[:-2]), tuple(positions.shape)))
        return _QueryKeyNorm.apply(q, k, self.w_q, self.w_k, positions, self._array(), self.eps, self.interleaved, rows)


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
