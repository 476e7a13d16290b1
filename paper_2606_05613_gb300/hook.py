"""Per-bucket resolve inside the backward pass (Algorithm 1, Figure 4).

The method intercepts gradients bucket by bucket during the backward pass
("when bucket k is full") and resolves each bucket's conflict before the next
one arrives.  On one GPU the K languages' gradients come from K backward
passes of the same model.  BucketMOO lays them out as K flat buffers in the
bucket order of the method -- tensors in reverse registration order, which is
the order backward produces them, cut into buckets by bkmoo_plan -- and makes
every parameter's .grad a view into the buffer of the language whose backward
pass runs (autograd then accumulates straight into it, no copy).  During the
last language's backward pass a post-accumulate hook counts the tensors of
each bucket; once a bucket is complete its resolve (bkmoo_resolve_buckets) is
queued on a side stream behind an event on the backward stream, so it
overlaps the rest of the backward pass.  finish() resolves what is left
(buckets whose tensors got no gradient), joins the side stream and points
every .grad at the resolved direction d for the optimizer step.

Argument marshalling and bookkeeping only: the resolve runs in the CUDA
library through its C ABI.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Sequence

import numpy as np

from . import native


@dataclass
class BucketLayout:
    """Flat layout of a model's gradient in bucket order.

    offsets: bucket boundaries (elements) from bkmoo_plan.
    starts[i]: flat position of parameter i (registration order); parameters
      are laid out last-registered first.
    first[i], last[i]: the buckets parameter i spans (last inclusive; a
      parameter larger than a bucket spans several); -1 for empty ones.
    need[b]: number of parameters that touch bucket b.
    """
    offsets: np.ndarray
    starts: List[int]
    first: List[int]
    last: List[int]
    need: List[int]

    @property
    def n_elems(self) -> int:
        return int(self.offsets[-1])

    @property
    def n_buckets(self) -> int:
        return len(self.offsets) - 1


def bucket_layout(sizes: Sequence[int], elem_bytes: int, bucket_bytes: int) -> BucketLayout:
    offsets = native.bkmoo_plan(list(sizes), elem_bytes, bucket_bytes)
    starts = [0] * len(sizes)
    pos = 0
    for i in reversed(range(len(sizes))):
        starts[i] = pos
        pos += int(sizes[i])
    assert pos == int(offsets[-1])
    B = len(offsets) - 1
    first, last = [-1] * len(sizes), [-1] * len(sizes)
    need = [0] * B
    for i, n in enumerate(sizes):
        if n == 0:
            continue
        first[i] = int(np.searchsorted(offsets, starts[i], side="right")) - 1
        last[i] = int(np.searchsorted(offsets, starts[i] + int(n) - 1, side="right")) - 1
        for b in range(first[i], last[i] + 1):
            need[b] += 1
    return BucketLayout(offsets, starts, first, last, need)


class LanguageGrads(list):
    """A parameter's K places in the flat buffers, which are zeroed and resolved on
    stream `home`.  A layer that writes them calls enter() before and leave() after: on
    another stream than `home` it then runs behind what is queued there, and what is
    queued there later behind it.  (Autograd does this for the gradients that it
    accumulates itself.)"""

    def __init__(self, places, home, device_index: int):
        super().__init__(places)
        self.home, self.device_index = home, device_index

    def _other(self):
        import torch
        if torch._C._cuda_getCurrentRawStream(self.device_index) == self.home.cuda_stream:
            return None
        return torch.cuda.current_stream(self.device_index)

    def enter(self) -> None:
        here = self._other()
        if here is not None:
            here.wait_stream(self.home)

    def leave(self) -> None:
        here = self._other()
        if here is not None:
            self.home.wait_stream(here)


class BucketMOO:
    """K per-language gradients of `params`, resolved bucket by bucket.

    Use:
        moo = BucketMOO(model.parameters(), K, bucket_bytes, rule="mgda")
        for k in range(K):
            moo.begin(k)
            loss_k(model, batch_k).backward()
        d = moo.finish()        # every p.grad is now a view of d
        optimizer.step()

    or, with the layers of language.py, one pass over a batch of all languages:
        moo.begin_batch()
        loss(model, batch, rows).backward()
        d = moo.finish()

    All parameters that require gradients must share one device and one
    dtype, float32 or bfloat16.  The buffers (K gradients, the direction, the
    workspace) are allocated once, here.
    """

    def __init__(self, params, K: int, bucket_bytes: int, rule: str = "mgda",
                 moo_params: "native.bkmoo_params | None" = None):
        import torch
        self.params = [p for p in params if p.requires_grad]
        if not self.params:
            raise ValueError("no parameter requires a gradient")
        dev, dt = self.params[0].device, self.params[0].dtype
        if dt not in (torch.float32, torch.bfloat16):
            raise TypeError("parameters must be float32 or bfloat16, got %s" % dt)
        for p in self.params:
            if p.device != dev or p.dtype != dt:
                raise TypeError("all parameters must share one device and dtype")
        if not 1 <= K <= 16:
            raise ValueError("K must be in [1, 16]")
        self.K, self.rule, self.device, self.dtype = K, rule, dev, dt
        self.moo_params = moo_params if moo_params is not None else native.bkmoo_default_params()
        sizes = [p.numel() for p in self.params]
        self.layout = bucket_layout(sizes, 4 if dt == torch.float32 else 2, bucket_bytes)
        N, B = self.layout.n_elems, self.layout.n_buckets
        self.grads = [torch.zeros(N, dtype=dt, device=dev) for _ in range(K)]
        self.direction = torch.zeros(N, dtype=dt, device=dev)
        self.weights = torch.zeros(B, K, dtype=torch.float32, device=dev)
        self.status = torch.zeros(B, dtype=torch.int32, device=dev)
        self.resolver = native.Resolver(K, dt, self.layout.offsets, dev)
        self.side = torch.cuda.Stream(device=dev)
        self._lang = None
        self._home = None        # stream of begin_batch()
        self._op_word = self._op_read = None
        self._left = list(self.layout.need)
        self._done = [False] * B
        self._hooks = [p.register_post_accumulate_grad_hook(self._make_hook(i))
                       for i, p in enumerate(self.params)]

    def _view(self, buf, i):
        p = self.params[i]
        s = self.layout.starts[i]
        return buf[s:s + p.numel()].view_as(p)

    def begin(self, k: int) -> None:
        """Zero language k's buffer and make every .grad a view into it."""
        if not 0 <= k < self.K:
            raise ValueError("language %d out of range" % k)
        import torch
        self._check_ops()
        # language k's buffer may still be read by last step's resolves
        torch.cuda.current_stream(self.device).wait_stream(self.side)
        self.grads[k].zero_()
        for i, p in enumerate(self.params):
            p.grad = self._view(self.grads[k], i)
            p.language_grads = None
        self._home = None
        self._lang = k
        if k == self.K - 1:
            self._left = list(self.layout.need)
            self._done = [False] * self.layout.n_buckets

    def begin_batch(self) -> None:
        """For one backward pass over a batch of all K languages, instead of K
        passes: zero every language's buffer and give every parameter
        `language_grads`, its K places in them.  The layers of language.py add
        each language's gradient to its own place; a parameter that no such
        layer uses keeps a gradient of 0 in every language.  finish() then
        resolves the whole plan at once."""
        import torch
        self._check_ops()
        home = torch.cuda.current_stream(self.device)
        home.wait_stream(self.side)
        for g in self.grads:
            g.zero_()
        for i, p in enumerate(self.params):
            p.grad = None
            p.language_grads = LanguageGrads([self._view(g, i) for g in self.grads], home,
                                             p.get_device())
        self._home = home
        self._lang = self.K - 1
        self._left = list(self.layout.need)
        self._done = [False] * self.layout.n_buckets

    def _make_hook(self, i):
        def hook(p):
            if self._lang != self.K - 1 or getattr(p, "language_grads", None) is not None:
                return
            for b in range(self.layout.first[i], self.layout.last[i] + 1):
                self._left[b] -= 1
                if self._left[b] == 0:
                    self._resolve(b, b + 1)
        return hook

    def _resolve(self, b_lo: int, b_hi: int) -> None:
        import torch
        ev = torch.cuda.Event()
        ev.record(torch.cuda.current_stream(self.device))
        self.side.wait_event(ev)
        self.resolver.resolve_buckets(self.grads, b_lo, b_hi, self.rule, self.direction,
                                      params=self.moo_params, out_weights=self.weights,
                                      out_status=self.status, stream=self.side)
        for b in range(b_lo, b_hi):
            self._done[b] = True

    def finish(self):
        """Resolve the buckets not resolved yet, join the side stream and
        point every .grad at the direction.  Returns the flat direction."""
        import torch
        if self._lang != self.K - 1:
            raise RuntimeError("finish() before the last language's backward pass")
        if any(getattr(p, "language_grads", None) is not None and p.grad is not None
               for p in self.params):
            raise RuntimeError("a parameter got a gradient that is not apart by language: in a "
                               "batch of all languages only language.py's layers may use them")
        if self._home is not None:
            here = torch.cuda.current_stream(self.device)
            if here != self._home:
                here.wait_stream(self._home)
            self._home = None
        b = 0
        B = self.layout.n_buckets
        while b < B:                        # runs of unresolved buckets
            if self._done[b]:
                b += 1
                continue
            e = b
            while e < B and not self._done[e]:
                e += 1
            self._resolve(b, e)
            b = e
        torch.cuda.current_stream(self.device).wait_stream(self.side)
        for i, p in enumerate(self.params):
            p.grad = self._view(self.direction, i)
            p.language_grads = None
        self._lang = None
        self._check_ops()
        self._read_ops()
        return self.direction

    def _read_ops(self) -> None:
        """Queue a read of the status word of language.py's kernels, where any ran and the
        last read has been looked at."""
        import torch
        dev = self.params[0].get_device()
        if self._op_read is not None or not native.ops_called(dev) or \
                torch.cuda.is_current_stream_capturing():
            return
        if self._op_word is None:
            self._op_word = torch.zeros(1, dtype=torch.int32, pin_memory=True)
        with torch.cuda.device(dev):
            native.bkmoo_op_status_copy(self._op_word)
            self._op_read = torch.cuda.Event()
            self._op_read.record()

    def _check_ops(self) -> None:
        """Raise if a kernel of language.py gave up in a step whose status has been read by now
        (no wait: bkmoo_adamw does not take the steps in between)."""
        import torch
        if self._op_read is None or torch.cuda.is_current_stream_capturing() or \
                not self._op_read.query():
            return
        self._op_read = None
        if int(self._op_word) != native.BKMOO_OK:
            code = native.bkmoo_op_status(self.device)
            raise native.BkmooError(code or int(self._op_word), "a gate or weight-gradient kernel of an earlier step")

    def remove(self) -> None:
        for h in self._hooks:
            h.remove()
        self._hooks = []
