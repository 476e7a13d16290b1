"""A few training steps of a small feed-forward model in K languages, on one GPU.

One batch holds the rows of all languages, unevenly; one backward pass leaves K
gradients (language.py), the resolve turns them into one direction bucket by
bucket, and AdamW with 8-bit moments takes the clipped step.  The data are
synthetic: every language has a teacher of its own beside a shared one, so the
languages agree in part.

    python examples/multilingual_step.py --steps 20 --rule mgda
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_05613_gb300.hook import BucketMOO           # noqa: E402
from paper_2606_05613_gb300.language import GatedFeedForward, LanguageLinear   # noqa: E402
from paper_2606_05613_gb300.optim import AdamW              # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, width, hidden, layers, classes):
        super().__init__()
        self.blocks = torch.nn.ModuleList(GatedFeedForward(width, hidden) for _ in range(layers))
        self.head = LanguageLinear(width, classes)

    def forward(self, x, rows):
        for block in self.blocks:
            y = x.float()
            x = x + block((y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).bfloat16(), rows)
        return self.head(x, rows)


def run(steps=20, K=4, rule="mgda", width=256, hidden=704, layers=2, classes=64, tokens=1000,
        state="e4m3", seed=0):
    """Every step's losses, [steps, K]."""
    torch.manual_seed(seed)
    share = torch.rand(K) + 0.5
    rows = [0] + [int(tokens * s) for s in (torch.cumsum(share, 0) / share.sum())[:-1]] + [tokens]
    model = Model(width, hidden, layers, classes)
    moo = BucketMOO(model.parameters(), K, 1 << 20, rule=rule)
    opt = AdamW(moo.params, lr=2e-3, betas=(0.9, 0.95), weight_decay=0.01, max_norm=1.0, state=state,
                master=True, seed=seed)
    shared = torch.randn(width, classes, device="cuda")
    own = torch.randn(K, width, classes, device="cuda")
    x = torch.randn(tokens, width, device="cuda")
    labels = torch.cat([(x[i:j] @ (shared + 0.5 * own[k])).argmax(1)
                        for k, (i, j) in enumerate(zip(rows, rows[1:]))])
    losses = []
    for _ in range(steps):
        moo.begin_batch()
        each = torch.nn.functional.cross_entropy(model(x.bfloat16(), rows).float(), labels,
                                                 reduction="none")
        per = torch.stack([each[i:j].mean() for i, j in zip(rows, rows[1:])])
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
