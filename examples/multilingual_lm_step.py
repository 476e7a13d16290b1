"""A few training steps of a small language model in K languages, on one GPU.

One batch holds whole sequences of all languages, unevenly; the embedding, the norms of
queries and keys and every projection leave their gradients apart by language in one
backward pass (language.py), the resolve turns them into one direction and AdamW takes
the clipped step.  The loss is the tokens' log probability; attention is written out.
The data are synthetic: in every language the next token follows from the last one, by
a table of its own for one token in three and by a shared one else.

    python examples/multilingual_lm_step.py --steps 20 --rule mgda
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_05613_gb300.hook import BucketMOO           # noqa: E402
from paper_2606_05613_gb300.language import (Embedding, GatedFeedForward, LanguageLinear,      # noqa: E402
                                             QueryKeyNorm, token_log_probs)
from paper_2606_05613_gb300.optim import AdamW              # noqa: E402


def _normed(x):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).bfloat16()


class Attention(torch.nn.Module):
    def __init__(self, width, heads, key_heads, head_width):
        super().__init__()
        self.heads, self.key_heads, self.head_width = heads, key_heads, head_width
        self.project = LanguageLinear(width, (heads + 2 * key_heads) * head_width)
        self.norm = QueryKeyNorm(head_width)
        self.out = LanguageLinear(heads * head_width, width)

    def forward(self, x, positions, rows):
        B, S = x.shape[:2]
        q, k, v = self.project(x, rows).unflatten(-1, (-1, self.head_width)).split(
            [self.heads, self.key_heads, self.key_heads], -2)
        q, k = self.norm(q, k, positions, rows)
        group = self.heads // self.key_heads
        q, k, v = (t.float().transpose(1, 2) for t in (q, k.repeat_interleave(group, 2), v.repeat_interleave(group, 2)))
        scores = q @ k.transpose(-1, -2) / math.sqrt(self.head_width)
        scores = scores.masked_fill(torch.ones(S, S, dtype=torch.bool, device=x.device).triu(1), -math.inf)
        y = (scores.softmax(-1) @ v).transpose(1, 2).reshape(B, S, -1)
        return self.out(y.bfloat16(), rows)


class Model(torch.nn.Module):
    def __init__(self, tokens, width, hidden, layers, heads, key_heads, head_width):
        super().__init__()
        self.embedding = Embedding(tokens, width, scale=math.sqrt(width))
        self.attention = torch.nn.ModuleList(Attention(width, heads, key_heads, head_width) for _ in range(layers))
        self.feed = torch.nn.ModuleList(GatedFeedForward(width, hidden) for _ in range(layers))
        self.head = LanguageLinear(width, tokens)

    def forward(self, ids, positions, rows):
        x = self.embedding(ids, rows)
        for attention, feed in zip(self.attention, self.feed):
            x = x + attention(_normed(x), positions, rows)
            x = x + feed(_normed(x), rows)
        return self.head(_normed(x), rows)


def sequences(K, count, length, tokens):
    """[count[0] + ..., length + 1] tokens, language after language."""
    shared = torch.randperm(tokens)
    out = []
    for k in range(K):
        own = torch.where(torch.rand(tokens) < 1 / 3, torch.randperm(tokens), shared)
        rows = [torch.randint(0, tokens, (count[k],))]
        for _ in range(length):
            rows.append(own[rows[-1]])
        out.append(torch.stack(rows, 1))
    return torch.cat(out).cuda()


def run(steps=20, K=4, rule="mgda", tokens=211, width=128, hidden=320, layers=2, heads=4, key_heads=2, head_width=32,
        length=48, sequences_each=(6, 3, 5, 2), state="e4m3", seed=0):
    """Every step's losses a token, [steps, K]."""
    torch.manual_seed(seed)
    count = [sequences_each[k % len(sequences_each)] for k in range(K)]
    rows = [0]
    for n in count:
        rows.append(rows[-1] + n * length)
    data = sequences(K, count, length, tokens)
    ids, targets = data[:, :-1].contiguous(), data[:, 1:].contiguous()
    targets[:, 0] = -100                            # the first token is a prompt
    positions = torch.arange(length, device="cuda").expand(ids.shape)
    model = Model(tokens, width, hidden, layers, heads, key_heads, head_width)
    moo = BucketMOO(model.parameters(), K, 1 << 18, rule=rule)
    opt = AdamW(moo.params, lr=2e-3, betas=(0.9, 0.95), weight_decay=0.01, max_norm=1.0, state=state, master=True, seed=seed)
    losses = []
    for _ in range(steps):
        moo.begin_batch()
        logp = token_log_probs(model(ids, positions, rows), targets).logp.reshape(-1)
        per = torch.stack([-logp[i:j].sum() / ((j - i) * (length - 1) / length) for i, j in zip(rows, rows[1:])])
        per.sum().backward()
        opt.step(moo.finish())
        losses.append(per.detach())
    return torch.stack(losses).cpu()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--languages", type=int, default=4)
    ap.add_argument("--rule", default="mgda", choices=("mgda", "pcgrad", "cagrad", "mean"))
    a = ap.parse_args()
    for i, per in enumerate(run(a.steps, a.languages, a.rule)):
        print("step %3d  loss by language: %s" % (i, "  ".join("%.4f" % v for v in per)))
