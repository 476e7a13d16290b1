"""Timed cases of the operators that a language model needs around the layers of a training step in K
languages, through the package's public entry points.

Three operators, each with its backward pass:

- embedding:   y_t = s W[id_t]; backward every language's own dW_k, the sum of s dy_t over the rows of the batch
  that belong to language k and hold the token (an id outside the table is padding: y = 0 and no gradient);
- qk_norm:     queries and keys normed per head, times a weight, rotated by their position; backward dq, dk and
  every language's own gradients of the two weights;
- token_logp:  log probability of a given token under a row of logits, with the row's entropy and its n most
  likely tokens where they are wanted; backward the gradient of the logits (a row whose target is outside the
  vocabulary is padding: log probability 0).

Sizes are those of this repository's workloads (GPT-2 small, Llama-3.2-1B, Qwen3-8B) or generic ones around them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


def _embed(name, op, T, V, D, dtype, scale=1.0, K=1, out="bf16", accumulate=False, empty=False):
    return {"name": name, "op": op, "T": T, "V": V, "D": D, "dtype": dtype, "scale": scale, "K": K, "out": out,
            "accumulate": accumulate, "empty": empty}


def _qk(name, op, T, hq, hk, hd, rot, base, neighbours=False, far=False, K=1, out="bf16", accumulate=False,
        empty=False):
    return {"name": name, "op": op, "T": T, "hq": hq, "hk": hk, "hd": hd, "rot": rot, "base": base,
            "neighbours": neighbours, "far": far, "K": K, "out": out, "accumulate": accumulate, "empty": empty}


def _logp(name, op, T, V, dtype, entropy=False, top=0, masked=False):
    return {"name": name, "op": op, "T": T, "V": V, "dtype": dtype, "entropy": entropy, "top": top,
            "masked": masked}


def listed():
    return [
        # Serving: the last tokens of 32 sequences enter a Qwen3-8B model.
        _embed("embed-fwd-32-qwen", "embed", 32, 151936, 4096, "bf16"),
        # Training: a Llama-3.2-1B batch of long sequences, rows scaled by the root of their width.
        _embed("embed-fwd-16384-llama", "embed", 16384, 128256, 2048, "bf16", scale=math.sqrt(2048)),
        # Training: four languages' gradients of the Llama-3.2-1B embedding added to what the head has left there.
        _embed("embed-bwd-8192-llama-k4", "embed_grad", 8192, 128256, 2048, "bf16", K=4, accumulate=True),
        # Training: a small 32-bit model of odd sizes, gradients written, one language without a row.
        _embed("embed-bwd-odd-k3-f32", "embed_grad", 1531, 10007, 771, "f32", scale=0.5, K=3, out="f32", empty=True),
        # Serving: the last tokens of 16 sequences, far into their contexts.
        _qk("qk-fwd-16-qwen", "qk", 16, 32, 8, 128, 128, 1e6, far=True),
        # Training: a Qwen3-8B layer.
        _qk("qk-fwd-8192-qwen", "qk", 8192, 32, 8, 128, 128, 1e6),
        # Training: the same layer's gradients in four languages.
        _qk("qk-bwd-8192-qwen-k4", "qk_grad", 8192, 32, 8, 128, 128, 1e6, K=4),
        # Training: heads of which half are rotated, neighbours paired, summed over micro-batches in 32 bits.
        _qk("qk-bwd-odd-k3-f32", "qk_grad", 1357, 10, 2, 96, 48, 1e4, neighbours=True, K=3, out="f32",
            accumulate=True, empty=True),
        # Serving: one next token over the Qwen3-8B vocabulary, with its 20 best alternatives.
        _logp("logp-fwd-1-qwen", "logp", 1, 151936, "bf16", entropy=True, top=20, masked=True),
        # Scoring: 32-bit logits of GPT-2 small, an odd number of rows, 5 alternatives each.
        _logp("logp-fwd-1531-gpt2-f32", "logp", 1531, 50257, "f32", entropy=True, top=5),
        # Training: the loss of a Llama-3.2-1B batch.
        _logp("logp-fwd-8192-llama", "logp", 8192, 128256, "bf16"),
        # Training: its gradient; a quarter of the rows are prompts, which count for nothing.
        _logp("logp-bwd-8192-llama", "logp_grad", 8192, 128256, "bf16"),
    ]


def draw(rng):
    def log_between(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    op = rng.choice(["embed", "embed_grad", "qk", "qk_grad", "logp", "logp", "logp_grad"])
    K = rng.choice([1, 2, 3, 4, 8, 16])
    if op in ("embed", "embed_grad"):
        D = log_between(64, 8192)
        if rng.random() < 0.7:                    # most models are whole multiples
            D = (D + 63) // 64 * 64
        dtype, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
        scale = rng.choice([1.0, math.sqrt(D)])
        if op == "embed":
            c = _embed("", op, min(log_between(1, 65536), 60_000_000 // D), log_between(1000, 262144), D, dtype, scale)
        else:
            V = min(log_between(1000, 200_000), 850_000_000 // (K * D))
            c = _embed("", op, min(log_between(K, 65536), 60_000_000 // D), V, D, dtype, scale, K, out,
                       rng.random() < 0.5, rng.random() < 0.3)
    elif op in ("qk", "qk_grad"):
        hk = rng.choice([1, 2, 4, 8, 16])
        hq = hk * rng.choice([1, 2, 3, 4, 5, 8])
        hd = rng.choice([64, 64, 80, 96, 112, 128, 128, 192, 256])
        rot = rng.choice([hd, hd, hd // 32 * 16])
        T = min(log_between(max(K, 1), 32768), 45_000_000 // ((hq + hk) * hd))
        c = _qk("", op, T, hq, hk, hd, rot, rng.choice([1e4, 5e5, 1e6]), rng.random() < 0.3, rng.random() < 0.3)
        if op == "qk_grad":
            c.update(K=K, out=rng.choice(["bf16", "bf16", "f32"]), accumulate=rng.random() < 0.5,
                     empty=rng.random() < 0.3)
    else:
        V = log_between(500, 262144)
        if rng.random() < 0.5:
            V = (V + 63) // 64 * 64
        dtype = rng.choice(["bf16", "bf16", "f32"])
        T = min(log_between(1, 32768), (450_000_000 if dtype == "f32" else 900_000_000) // V)
        c = _logp("", op, T, V, dtype, rng.random() < 0.5)
        if op == "logp":
            # (the alternatives of some hundreds of millions of logits take the plain form seconds)
            c["top"] = rng.choice([0, 1, 5, 20, 32]) if T * V <= 300_000_000 else 0
            c["masked"] = rng.random() < 0.3
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------

def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _languages(case, seed):
    """Row bounds of the K languages: uneven shares, and one language without a row where the case says so."""
    rng = np.random.default_rng([seed, 41])
    K, T = case["K"], case["T"]
    share = rng.uniform(0.3, 1.0, K)
    if case["empty"] and K > 1:
        share[rng.integers(0, K)] = 0.0
    ends = np.floor(np.cumsum(share) / share.sum() * T + 0.5).astype(np.int64)
    ends[-1] = T
    return [0] + [int(e) for e in ends]


def _token_share(V):
    """How often the tokens of a vocabulary occur, the most frequent first (Zipf with Mandelbrot's shift)."""
    p = 1.0 / (torch.arange(V, dtype=torch.float64) + 2.7)
    return p / p.sum()


def _tokens(gen, rows, V, padding):
    """Tokens of each language's rows, whose frequent tokens are its own; the last `padding` of a language's rows
    are padding."""
    T = rows[-1]
    order = torch.cumsum(_token_share(V), 0).to(DEV)
    rank = torch.searchsorted(order, torch.rand(T, generator=gen, device=DEV, dtype=torch.float64)).clamp_(max=V - 1)
    ids = torch.empty(T, dtype=torch.int64, device=DEV)
    for k, (i, j) in enumerate(zip(rows, rows[1:])):
        ids[i:j] = (rank[i:j] * 7919 + 104729 * k) % V if V % 7919 else (rank[i:j] + 104729 * k) % V
        ids[j - int(padding * (j - i)):j] = -1
    return ids


def _embed_inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, V, D, dt = case["T"], case["V"], case["D"], _type(case["dtype"])
    if case["op"] == "embed":
        table = torch.empty(V, D, dtype=dt, device=DEV).normal_(0.0, 0.02, generator=gen)
        return {"table": table, "ids": _tokens(gen, [0, T], V, 0.05)}
    s = {"rows": _languages(case, seed)}
    s["ids"] = _tokens(gen, s["rows"], V, 0.05)
    s["dy"] = torch.empty(T, D, dtype=dt, device=DEV).normal_(0.0, 0.01, generator=gen)
    dw = torch.zeros(case["K"], V, D, dtype=_type(case["out"]), device=DEV)
    s["dw"] = dw.normal_(0.0, 0.01, generator=gen) if case["accumulate"] else dw
    return s


def _qk_inputs(case, seed):
    """Queries and keys are columns of the fused projection's output, [T, (hq + 2 hk) hd]."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, hq, hk, hd = case["T"], case["hq"], case["hk"], case["hd"]

    def fused():
        scale = torch.rand((hq + 2 * hk) * hd, generator=gen, device=DEV) * 3 + 0.2
        m = (torch.randn(T, (hq + 2 * hk) * hd, generator=gen, device=DEV) * scale).bfloat16().view(T, -1, hd)
        return m[:, :hq], m[:, hq:hq + hk]

    s = {}
    s["q"], s["k"] = fused()
    s["wq"], s["wk"] = ((1.0 + 0.2 * torch.randn(hd, generator=gen, device=DEV)).bfloat16() for _ in range(2))
    if case["far"]:
        s["pos"] = torch.randint(0, 1 << 20, (T,), generator=gen, device=DEV)
    else:
        s["pos"] = torch.arange(T, device=DEV) % 4096
    s["freq"] = [case["base"] ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
    if case["op"] == "qk_grad":
        s["rows"] = _languages(case, seed)
        s["dqo"], s["dko"] = ((0.01 * torch.randn(T, h, hd, generator=gen, device=DEV)).bfloat16() for h in (hq, hk))
        dw = torch.zeros(2, case["K"], hd, dtype=_type(case["out"]), device=DEV)
        s["dw"] = dw.normal_(0.0, 0.1, generator=gen) if case["accumulate"] else dw
    return s


def _prompts(case):
    return case["T"] // 4 if case["op"] == "logp_grad" else 0


def _logp_inputs(case, seed):
    """Logits of a model that knows something: the target is often among the likely ones.  A masked row has an
    eighth of the vocabulary at minus infinity."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, V = case["T"], case["V"]
    logits = torch.empty(T, V, dtype=_type(case["dtype"]), device=DEV).normal_(0.0, 2.0, generator=gen)
    targets = torch.randint(0, V, (T,), generator=gen, device=DEV)
    at = torch.arange(T, device=DEV)
    sure = torch.rand(T, generator=gen, device=DEV) * 10.0
    logits[at, targets] = (logits[at, targets].float() + sure).to(logits.dtype)
    if case["masked"]:
        out = torch.rand(V, generator=gen, device=DEV) < 0.125
        logits.masked_fill_(out, -math.inf)
        targets = torch.where(out[targets], -1, targets)
    s = {"logits": logits, "targets": targets}
    if case["op"] == "logp_grad":
        targets[:_prompts(case)] = -100
        s["g"] = torch.where(targets >= 0, -1.0 / T, 0.0)
        s["h"] = torch.where(targets >= 0, -1e-3 / T, 0.0) if case["entropy"] else None
    return s


def prepare(case, seed):
    op, T = case["op"], case["T"]
    if op in ("embed", "embed_grad"):
        s = _embed_inputs(case, seed)
        if op == "embed":
            s["y"] = torch.empty(T, case["D"], dtype=_type(case["dtype"]), device=DEV)
    elif op in ("qk", "qk_grad"):
        s = _qk_inputs(case, seed)
        if op == "qk":
            s["qo"], s["ko"] = (torch.empty(T, case[h], case["hd"], dtype=torch.bfloat16, device=DEV) for h in ("hq", "hk"))
        else:
            m = torch.empty(T, case["hq"] + 2 * case["hk"], case["hd"], dtype=torch.bfloat16, device=DEV)
            s["dq"], s["dk"] = m[:, :case["hq"]], m[:, case["hq"]:case["hq"] + case["hk"]]
        if own:
            from paper_2606_05613_gb300 import native as bk

            s["freq"] = bk.rope_frequencies(case["rot"], case["base"])
    else:
        s = _logp_inputs(case, seed)
        if op == "logp":
            s["logp"] = torch.empty(T, device=DEV)
            s["stats"] = torch.empty(T, 2, device=DEV)
            s["entropy"] = torch.empty(T, device=DEV) if case["entropy"] else None
            s["top_ids"] = torch.empty(T, case["top"], dtype=torch.int64, device=DEV) if case["top"] else None
            s["top_logp"] = torch.empty(T, case["top"], device=DEV) if case["top"] else None
        else:
            s["dz"] = torch.empty_like(s["logits"])
            s["stats"], s["entropy"] = _statistics(s["logits"], case["entropy"])
    s["case"] = case
    return s


# ---------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------

def _embedding(s):
    table, ids = s["table"], s["ids"]
    V = table.shape[0]
    ok = (ids >= 0) & (ids < V)
    return {"y": (table[ids.clamp(0, V - 1)].float() * (ok * s["case"]["scale"]).float()[:, None]).to(table.dtype)}


def _embedding_grad(s):
    case, dw, V = s["case"], s["dw"], s["case"]["V"]
    if not case["accumulate"]:
        dw.zero_()
    for k, (i, j) in enumerate(zip(s["rows"], s["rows"][1:])):
        ids = s["ids"][i:j]
        ok, at = (ids >= 0) & (ids < V), ids.clamp(0, V - 1)
        g = s["dy"][i:j].float() * (ok * case["scale"]).float()[:, None]
        first = torch.searchsorted(torch.sort(at).values, at)       # one place for each distinct token
        total = torch.zeros_like(g).index_add_(0, first, g)
        dw[k][at] = (dw[k][at].float() + total[first]).to(dw.dtype)
    return {"dw": dw}


def _angles(s):
    a = s["pos"].double()[:, None] * torch.tensor(s["freq"], dtype=torch.float64, device=DEV)
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _rotate(x, cos, sin, case):
    rot, half = case["rot"], case["rot"] // 2
    out = x.clone()
    if case["neighbours"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :half], x[..., half:rot]
        out[..., :half], out[..., half:rot] = a * cos - b * sin, b * cos + a * sin
    return out


def _normed(x):
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _qk_norm(s):
    cos, sin = _angles(s)
    return {o: _rotate(_normed(s[x])[0] * s[w].float(), cos, sin, s["case"]).bfloat16()
            for o, x, w in (("qo", "q", "wq"), ("ko", "k", "wk"))}


def _qk_norm_grad(s):
    case, dw = s["case"], s["dw"]
    cos, sin = _angles(s)
    out = {"dw": dw}
    for i, (name, x, do, w) in enumerate((("dq", "q", "dqo", "wq"), ("dk", "k", "dko", "wk"))):
        n, r = _normed(s[x])
        dy = _rotate(s[do].float(), cos, -sin, case)
        each = (dy * n).sum(1)
        sums = torch.stack([each[a:b].sum(0) for a, b in zip(s["rows"], s["rows"][1:])])
        dw[i].copy_(dw[i].float() + sums if case["accumulate"] else sums)
        dn = dy * s[w].float()
        out[name] = s[name].copy_(r * (dn - n * (dn * n).mean(-1, keepdim=True)))
    return out


def _statistics(logits, entropy):
    z = logits.float()
    m = z.amax(-1)
    x = z - m[:, None]
    e = torch.exp(x)
    total = e.sum(-1)
    L = torch.log(total)
    return torch.stack([m, L], 1), L - torch.where(e > 0, e * x, 0.0).sum(-1) / total if entropy else None


def _token_logp(s):
    case, logits, targets = s["case"], s["logits"], s["targets"]
    T, V = logits.shape
    stats, entropy = _statistics(logits, case["entropy"])
    m, L = stats[:, 0], stats[:, 1]
    ok = (targets >= 0) & (targets < V)
    z = logits[torch.arange(T, device=DEV), targets.clamp(0, V - 1)].float()
    out = {"logp": torch.where(ok, z - m - L, 0.0), "stats": stats}
    if case["entropy"]:
        out["entropy"] = entropy
    if case["top"]:
        # the order of the values as whole numbers, the lower index first among equal ones
        bits = logits.float().view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 24) + (V - 1 - torch.arange(V, device=DEV))
        ids = V - 1 - (torch.topk(key, case["top"], -1).values & ((1 << 24) - 1))
        out["top_ids"] = ids
        out["top_logp"] = torch.gather(logits, 1, ids).float() - m[:, None] - L[:, None]
    return out


def _token_logp_grad(s):
    logits, targets, g, h = s["logits"], s["targets"], s["g"], s["h"]
    T, V = logits.shape
    lp = logits.float() - s["stats"][:, :1] - s["stats"][:, 1:]
    p = torch.exp(lp)
    d = p * -g[:, None]
    if h is not None:
        d -= h[:, None] * torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0)
    ok = (targets >= 0) & (targets < V)
    d[torch.arange(T, device=DEV), targets.clamp(0, V - 1)] += torch.where(ok, g, 0.0)
    return {"dz": d.to(logits.dtype)}


def _own(s):
    from paper_2606_05613_gb300 import native as bk

    case, op = s["case"], s["case"]["op"]
    if op == "embed":
        bk.bkmoo_embedding_forward(s["table"], s["ids"], s["y"], scale=case["scale"])
        return {"y": s["y"]}
    if op == "embed_grad":
        bk.bkmoo_embedding_backward(s["dy"], s["ids"], s["rows"], s["dw"].unbind(0), scale=case["scale"],
                                    accumulate=case["accumulate"])
        return {"dw": s["dw"]}
    if op == "qk":
        bk.bkmoo_qk_norm_forward(s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["freq"], s["qo"], s["ko"], eps=EPS,
                                 interleaved=case["neighbours"])
        return {"qo": s["qo"], "ko": s["ko"]}
    if op == "qk_grad":
        bk.bkmoo_qk_norm_backward(s["dqo"], s["dko"], s["q"], s["k"], s["wq"], s["wk"], s["pos"], s["freq"], s["rows"],
                                  s["dq"], s["dk"], s["dw"][0].unbind(0), s["dw"][1].unbind(0), eps=EPS,
                                  interleaved=case["neighbours"], accumulate=case["accumulate"])
        return {"dw": s["dw"], "dq": s["dq"], "dk": s["dk"]}
    if op == "logp":
        bk.bkmoo_token_logp_forward(s["logits"], s["targets"], s["logp"], s["stats"], s["entropy"], s["top_ids"],
                                    s["top_logp"])
        return {k: s[k] for k in ("logp", "stats", "entropy", "top_ids", "top_logp") if s[k] is not None}
    bk.bkmoo_token_logp_backward(s["logits"], s["targets"], s["stats"], s["g"], s["dz"], s["entropy"], s["h"])
    return {"dz": s["dz"]}


def run(state):
    if own:
        return _own(state)
    return {"embed": _embedding, "embed_grad": _embedding_grad, "qk": _qk_norm, "qk_grad": _qk_norm_grad,
            "logp": _token_logp, "logp_grad": _token_logp_grad}[state["case"]["op"]](state)


def _distinct(n, V):
    """Distinct tokens to be expected among n."""
    return float((-torch.expm1(n * torch.log1p(-_token_share(V)))).sum())


def work(case):
    op, T = case["op"], case["T"]
    size = {"f32": 4, "bf16": 2}
    if op == "embed":
        e = size[case["dtype"]]
        return {"bytes": int((T + min(T, _distinct(0.95 * T, case["V"]))) * case["D"] * e) + 8 * T, "flops": T * case["D"]}
    if op == "embed_grad":
        V, D, K = case["V"], case["D"], case["K"]
        if case["accumulate"]:
            rows = 2 * K * min(T / K, _distinct(0.95 * T / K, V))
        else:
            rows = K * V
        return {"bytes": int(0.95 * T * D * size[case["dtype"]] + rows * D * size[case["out"]]) + 8 * T, "flops": 2 * T * D}
    if op in ("qk", "qk_grad"):
        n = T * (case["hq"] + case["hk"]) * case["hd"]
        return {"bytes": n * (4 if op == "qk" else 6) + 8 * T, "flops": n * (8 if op == "qk" else 20)}
    n, e = T * case["V"], size[case["dtype"]]
    if op == "logp":
        return {"bytes": n * e + T * (20 + 4 * case["entropy"] + 12 * case["top"]), "flops": n * (6 if case["entropy"] else 4)}
    return {"bytes": (2 * T - _prompts(case)) * case["V"] * e + 28 * T, "flops": n * 4}


# ---------------------------------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------------------------------

def _exact_qk(x, w, pos, freq, case):
    """Norm, weight and rotation of [T, heads, hd], the pairs as complex numbers."""
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    rot = case["rot"]
    z = y[..., :rot]
    z = z.unflatten(-1, (rot // 2, 2)) if case["neighbours"] else z.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    turn = torch.polar(torch.ones_like(freq), pos.double()[:, None] * freq)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None])
    z = z.flatten(-2) if case["neighbours"] else z.transpose(-1, -2).flatten(-2)
    return torch.cat([z, y[..., rot:]], -1)


def exact(case, seed):
    op = case["op"]
    if op in ("embed", "embed_grad"):
        s = _embed_inputs(case, seed)
        keep = (s["ids"] >= 0).nonzero()[:, 0]
        if op == "embed":
            y = torch.zeros(case["T"], case["D"], dtype=torch.float64, device=DEV)
            y[keep] = torch.index_select(s["table"], 0, s["ids"][keep]).double() * case["scale"]
            return {"y": y}
        dw = s["dw"].double()
        for k in range(case["K"]):
            mine = keep[(keep >= s["rows"][k]) & (keep < s["rows"][k + 1])]
            dw[k].index_add_(0, s["ids"][mine], s["dy"][mine].double(), alpha=case["scale"])
        return {"dw": dw}
    if op in ("qk", "qk_grad"):
        s = _qk_inputs(case, seed)
        freq = torch.tensor(s["freq"], dtype=torch.float64, device=DEV)
        out = {}
        if op == "qk":
            for o, x, w in (("qo", "q", "wq"), ("ko", "k", "wk")):
                out[o] = _exact_qk(s[x].double(), s[w].double(), s["pos"], freq, case)
            return out
        out["dw"] = s["dw"].double() if case["accumulate"] else torch.zeros(s["dw"].shape, dtype=torch.float64, device=DEV)
        for i, (name, x, do, w) in enumerate((("dq", "q", "dqo", "wq"), ("dk", "k", "dko", "wk"))):
            out[name] = torch.zeros(s[x].shape, dtype=torch.float64, device=DEV)
            for k in range(case["K"]):
                a, b = s["rows"][k], s["rows"][k + 1]
                if a == b:
                    continue
                xk, wk = s[x][a:b].double().requires_grad_(), s[w].double().requires_grad_()
                y = _exact_qk(xk, wk, s["pos"][a:b], freq, case)
                dx, dw = torch.autograd.grad(y, (xk, wk), s[do][a:b].double())
                out[name][a:b] = dx
                out["dw"][i, k] += dw
        return out
    s = _logp_inputs(case, seed)
    z = s["logits"].double()
    T, V = z.shape
    lse = torch.logsumexp(z, -1)
    safe = s["targets"].clamp(0, V - 1)[:, None]
    ok = s["targets"] >= 0
    if op == "logp":
        m = s["logits"].double().max(-1).values
        out = {"logp": torch.where(ok, torch.gather(z, 1, safe)[:, 0] - lse, 0.0), "stats": torch.stack([m, lse - m], 1)}
        if case["entropy"]:
            out["entropy"] = torch.special.entr(torch.softmax(z, -1)).sum(-1)
        if case["top"]:
            value, ids = torch.sort(s["logits"], stable=True, dim=-1, descending=True)
            out["top_ids"] = ids[:, :case["top"]].clone()
            out["top_logp"] = value[:, :case["top"]].double() - lse[:, None]
        return out
    p = torch.softmax(z, -1)
    d = p * -s["g"].double()[:, None]
    d.scatter_add_(1, safe, torch.where(ok, s["g"].double(), 0.0)[:, None])
    if s["h"] is not None:
        entropy = torch.special.entr(p)
        d += s["h"].double()[:, None] * (entropy - p * entropy.sum(-1, keepdim=True))
    return {"dz": d}
