"""Timed cases of a training step's operators around the resolve, through the package's public entry points.

Four operators of fine-tuning in K languages with per-language gradients, and of serving the same model:

- gate_forward:  a = x Wg^T, b = x Wu^T, h = act(a) * b, the gated projections of a feed-forward block;
- gate_backward: from dh the input's gradient dx and every language's own dWg_k, dWu_k (the rows of the batch
  that belong to language k), which is what the resolve reads;
- language_wgrad: every language's weight gradient dW_k = dy_k^T x_k of a linear layer;
- adamw: one AdamW step of all the model's tensors with the resolved direction, its norm clipped, with moments
  of 32 bits or of 8 bits (e4m3 values, one scale for 256 elements, rounded stochastically by a keyed hash).

Sizes are those of this repository's workloads (the tensor lists of GPT-2 small, Llama-3.2-1B and Qwen3-8B
layers) or generic ones around them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.95, 1e-8, 3e-4, 0.1
BLOCK = 256                      # elements that share a scale of 8-bit moments
STEP, SEED = 1000, 11            # of the AdamW step: bias corrections, and the key of the 8-bit rounding
GOLD = 0x9E3779B97F4A7C15
M64 = (1 << 64) - 1


def _gate(name, op, T, D, F, act, K=1, save=False, empty=False):
    return {"name": name, "op": op, "T": T, "D": D, "F": F, "act": act, "K": K, "save": save, "empty": empty}


def _wgrad(name, T, M, N, K, out, accumulate, empty=False):
    return {"name": name, "op": "wgrad", "T": T, "M": M, "N": N, "K": K, "out": out, "accumulate": accumulate,
            "empty": empty}


def _adamw(name, model, n, param, grad, state, clip, master=False):
    return {"name": name, "op": "adamw", "model": model, "n": n, "param": param, "grad": grad, "state": state,
            "clip": clip, "master": master}


def listed():
    return [
        # Serving: one token through a Llama-3.2-1B layer; the weights' bytes are what it costs.
        _gate("gate-fwd-1-llama", "forward", 1, 2048, 8192, "silu"),
        # Serving: a few dozen sequences' tokens at once, a layer of odd sizes.
        _gate("gate-fwd-37-odd", "forward", 37, 1003, 2731, "gelu_tanh"),
        # Training: the forward pass of a Llama-3.2-1B layer, a and b kept for the backward pass.
        _gate("gate-fwd-8192-llama", "forward", 8192, 2048, 8192, "silu", save=True),
        # Training: the forward pass of a Qwen3-8B layer over a shorter batch.
        _gate("gate-fwd-4096-qwen", "forward", 4096, 4096, 12288, "silu", save=True),
        # Training: a small layer, an odd number of tokens, a batch in which one language has none.
        _gate("gate-bwd-small-k4", "backward", 1357, 768, 2048, "gelu", K=4, empty=True),
        # Training: eight languages share a Llama-3.2-1B batch unevenly.
        _gate("gate-bwd-llama-k8", "backward", 8192, 2048, 8192, "silu", K=8),
        # Training: four languages, a Qwen3-8B layer, the benchmark's model.
        _gate("gate-bwd-qwen-k4", "backward", 4096, 4096, 12288, "silu", K=4),
        # Training: the down projection's gradients of a Llama-3.2-1B layer in four languages.
        _wgrad("wgrad-llama-k4-bf16", 8192, 2048, 8192, 4, "bf16", False),
        # Training: a small projection of odd sizes, summed over micro-batches in 32 bits.
        _wgrad("wgrad-odd-k3-f32", 1531, 771, 517, 3, "f32", True, empty=True),
        # One step of GPT-2 small in 32 bits, the direction's norm clipped.
        _adamw("adamw-gpt2-f32", "gpt2", 0, "f32", "f32", "f32", True),
        # One step of Llama-3.2-1B: bf16 weights and direction, 8-bit moments, clipped.
        _adamw("adamw-llama1b-bf16-e4m3", "llama", 0, "bf16", "bf16", "e4m3", True),
        # A small adapter of odd tensors: bf16 weights with a 32-bit master copy, 8-bit moments.
        _adamw("adamw-ragged-master-e4m3", "ragged", 1_000_003, "bf16", "f32", "e4m3", False, master=True),
    ]


def draw(rng):
    def log_between(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    op = rng.choice(["forward", "forward", "backward", "wgrad", "adamw", "adamw"])
    if op == "adamw":
        c = _adamw("", "ragged", log_between(20_000, 600_000_000) | rng.choice([0, 1]), *rng.choice([("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")]),
                   rng.choice(["f32", "e4m3"]), rng.random() < 0.5, rng.random() < 0.3)
        c["master"] = c["master"] and c["param"] == "bf16"
    elif op == "wgrad":
        M, N = log_between(128, 8192), log_between(128, 8192)
        K = rng.choice([1, 2, 3, 4, 8, 16])
        c = _wgrad("", min(log_between(K, 16384), 550_000_000_000 // (2 * M * N)), M, N, K, rng.choice(["bf16", "f32"]),
                   rng.random() < 0.3, rng.random() < 0.3)
    else:
        D, F = log_between(256, 4096), log_between(256, 12288)
        if rng.random() < 0.7:                    # most layers are whole multiples
            D, F = (D + 127) // 128 * 128, (F + 127) // 128 * 128
        D, F = (d + 8 if d == 3072 else d for d in (D, F))
        act = rng.choice(["silu", "silu", "gelu", "gelu_tanh"])
        if op == "forward":
            T = min(log_between(1, 16384), 800_000_000_000 // (4 * D * F))
            c = _gate("", "forward", T, D, F, act, save=rng.random() < 0.5)
        else:
            K = rng.choice([1, 2, 3, 4, 8, 16])
            T = min(log_between(max(K, 16), 16384), 1_600_000_000_000 // (8 * D * F))
            c = _gate("", "backward", T, D, F, act, K=K, empty=rng.random() < 0.3)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------

def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _rows(n):
    return (n + 7) // 8 * 8                       # rows start on 16 bytes: odd widths are padded


def _matrix(gen, rows, cols, scale):
    m = torch.randn(rows, _rows(cols), generator=gen, device=DEV).mul_(scale).to(torch.bfloat16)
    return m[:, :cols]


def _room(rows, cols):
    return torch.empty(rows, _rows(cols), dtype=torch.bfloat16, device=DEV)[:, :cols]


def _languages(case, seed):
    """Row bounds of the K languages: uneven shares, and one language without a row where the case says so."""
    rng = np.random.default_rng([seed, 29])
    K, T = case["K"], case["T"]
    share = rng.uniform(0.3, 1.0, K)
    if case["empty"] and K > 1:
        share[rng.integers(0, K)] = 0.0
    ends = np.floor(np.cumsum(share) / share.sum() * T + 0.5).astype(np.int64)
    ends[-1] = T
    return [0] + [int(e) for e in ends]


def _sizes(case):
    """Element counts of the model's tensors, in the order of the flat direction."""
    if case["model"] == "gpt2":
        d, f, v, p = 768, 4 * 768, 50257, 1024
        layer = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, d * f, f, f * d, d]
        return list(reversed([v * d, p * d] + 12 * layer + [d, d]))
    if case["model"] == "llama":
        h, kv, f, v = 2048, 512, 8192, 128256
        layer = [h * h, kv * h, kv * h, h * h, f * h, f * h, h * f, h, h]
        return list(reversed([v * h] + 16 * layer + [h]))
    # ragged: large odd tensors with small ones between, n elements in all
    n = case["n"]
    rng, sizes, left = np.random.default_rng(n), [], n
    while left > 0:
        t = int(min(left, rng.integers(1, 700) if len(sizes) % 3 else rng.integers(n // 60 + 1, n // 20 + 2)))
        sizes.append(t)
        left -= t
    return sizes


def _gate_inputs(case, seed):
    T, D, F = case["T"], case["D"], case["F"]
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"x": _matrix(gen, T, D, 1.0), "wg": _matrix(gen, F, D, 1.3 / math.sqrt(D)), "wu": _matrix(gen, F, D, 1.0 / math.sqrt(D))}
    if case["op"] == "backward":
        s["a"], s["b"], s["dh"] = _matrix(gen, T, F, 1.3), _matrix(gen, T, F, 1.0), _matrix(gen, T, F, 0.01)
        s["rows"] = _languages(case, seed)
    return s


def _wgrad_inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"dy": _matrix(gen, case["T"], case["M"], 0.01), "x": _matrix(gen, case["T"], case["N"], 1.0), "rows": _languages(case, seed)}
    dw = torch.zeros(case["K"], case["M"], case["N"], dtype=_type(case["out"]), device=DEV)
    s["dw"] = dw.normal_(0.0, 0.1, generator=gen) if case["accumulate"] else dw
    return s


def _adamw_inputs(case, seed):
    """A model in training: weights, a direction, and moments of earlier directions of the same scale; a tensor in
    eight is an embedding of which most rows have not been seen yet (all zeros)."""
    sizes = np.array(_sizes(case), dtype=np.int64)
    n = int(sizes.sum())
    rng = np.random.default_rng([seed, 31])
    sigma = torch.tensor(np.exp(rng.standard_normal(len(sizes))) * 1e-3, dtype=torch.float32, device=DEV)
    unseen = torch.tensor(rng.random(len(sizes)) < 0.125, device=DEV)
    lens = torch.tensor(sizes, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    scale = torch.repeat_interleave(sigma, lens, output_size=n)
    scale *= 1.0 - torch.repeat_interleave(unseen, lens, output_size=n).float() * (torch.arange(n, device=DEV) // 64 % 4 != 0)
    s = {"sizes": sizes, "grad": torch.randn(n, generator=gen, device=DEV).mul_(scale).to(_type(case["grad"]))}
    w = torch.randn(n, generator=gen, device=DEV).mul_(0.02)
    s["flat"] = w.to(_type(case["param"]))
    s["params"] = list(torch.split(s["flat"], sizes.tolist()))
    s["decay"] = [DECAY if k > 2000 else 0.0 for k in sizes.tolist()]      # matrices decay, norms and biases do not
    s["master"] = w if case["master"] else None
    m = torch.randn(n, generator=gen, device=DEV).mul_(scale).mul_(0.3)
    r = torch.rand(n, generator=gen, device=DEV).add_(0.5).mul_(scale)     # the root of the second moment
    if case["state"] == "f32":
        s["m"], s["v"] = m, r.square_()
    else:
        s["m"], s["m_scale"] = _blocks(m)
        s["v"], s["v_scale"] = _blocks(r)
    s["step"] = STEP
    return s


def _blocks(x):
    n = x.numel()
    y = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = y.abs().amax(1) / 448.0
    return (y / scale.clamp_min(1e-30)[:, None]).to(torch.float8_e4m3fn).view(-1)[:n].clone(), scale


def prepare(case, seed):
    if case["op"] == "adamw":
        s = _adamw_inputs(case, seed)
    elif case["op"] == "wgrad":
        s = _wgrad_inputs(case, seed)
    else:
        s = _gate_inputs(case, seed)
        T, D, F, K = case["T"], case["D"], case["F"], case["K"]
        if case["op"] == "forward":
            s["h"] = _room(T, F)
            s["a"], s["b"] = (_room(T, F), _room(T, F)) if case["save"] else (None, None)
        else:
            s["dx"] = _room(T, D)
            s["dwg"], s["dwu"] = (torch.zeros(K, F, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    s["case"] = case
    return s


# ---------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------

def _act(name, a):
    """act(a) and its derivative."""
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-a))
        return a * s, s * (1.0 + a * (1.0 - s))
    if name == "gelu":
        c = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * c, c + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    k = math.sqrt(2.0 / math.pi)
    t = torch.tanh(k * (a + 0.044715 * a * a * a))
    return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * a * a)


def _forward(s):
    x = s["x"].float()
    a, b = x @ s["wg"].float().T, x @ s["wu"].float().T
    h = (_act(s["case"]["act"], a)[0] * b).bfloat16()
    return {"h": h, "a": a.bfloat16(), "b": b.bfloat16()} if s["case"]["save"] else {"h": h}


def _by_language(dy, x, rows):
    return torch.stack([dy[i:j].T @ x[i:j] for i, j in zip(rows, rows[1:])])


def _backward(s):
    act, slope = _act(s["case"]["act"], s["a"].float())
    dh, x, rows = s["dh"].float(), s["x"].float(), s["rows"]
    da, db = dh * s["b"].float() * slope, dh * act
    dx = da @ s["wg"].float() + db @ s["wu"].float()
    return {"dx": dx.bfloat16(), "dwg": _by_language(da, x, rows).bfloat16(), "dwu": _by_language(db, x, rows).bfloat16()}


def _language_wgrad(s):
    dw = _by_language(s["dy"].float(), s["x"].float(), s["rows"])
    s["dw"].copy_(s["dw"].float() + dw if s["case"]["accumulate"] else dw)
    return {"dw": s["dw"]}


def _shift(z, k):
    return (z >> k) & ((1 << (64 - k)) - 1)       # of 64 bits without a sign


def _signed(c):
    return c - (1 << 64) if c >= 1 << 63 else c


def _mix(z):
    z = (z ^ _shift(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _shift(z, 27)) * _signed(0x94D049BB133111EB)
    return z ^ _shift(z, 31)


def _key(step):
    z = (SEED + (step + 1) * GOLD) & M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def _draws(n, step):
    """16 bits for the first and 16 for the second moment of every element, from (seed, step, index): a pair of
    elements shares a 64-bit word, the even one its low half."""
    pair = torch.arange(1, (n + 1) // 2 + 1, device=DEV)
    z = _mix(pair * _signed(GOLD) + _signed(_key(step)))
    half = torch.stack([z & 0xFFFFFFFF, _shift(z, 32)], 1).view(-1)[:n]
    return half & 0xFFFF, half >> 16


def _load8(code, scale):
    return code.float() * scale.repeat_interleave(BLOCK)[:code.numel()]


def _store8(x, u, code, scale, positive):
    """x in blocks as e4m3 values of 1/448 of the block's largest, rounded up with the chance that the rest gives;
    where `positive`, what is not zero does not become zero."""
    n = x.numel()
    y = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    top = y.abs().amax(1)
    top = torch.where(top < 2.0 ** -100, 0.0, top)
    scale.copy_(top / 448.0)
    inv = torch.where(top > 0, 448.0 / top, 0.0)
    bits = ((y.abs() * inv[:, None]).view(-1)[:n] * 2.0 ** -120).view(torch.int32)
    c = torch.clamp((bits + (u << 4)) >> 20, max=0x7E)
    if positive:
        c = torch.where((c == 0) & (bits > 0), 1, c)
    code.copy_((c | torch.where(x < 0, 0x80, 0)).to(torch.uint8).view(torch.float8_e4m3fn))


def _adamw_step(s):
    case, step = s["case"], s["step"]
    g, n = s["grad"].float(), s["grad"].numel()
    out = {}
    if case["clip"]:
        norm = torch.sqrt((g * g).sum())
        g = g * torch.clamp(1.0 / (norm + 1e-6), max=1.0)
        out["norm"] = norm
    eight = case["state"] == "e4m3"
    m = _load8(s["m"], s["m_scale"]) if eight else s["m"]
    v = _load8(s["v"], s["v_scale"]).square() if eight else s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    r = torch.sqrt(v)
    lens = torch.tensor(s["sizes"], device=DEV)
    keep = 1.0 - LR * torch.repeat_interleave(torch.tensor(s["decay"], device=DEV), lens, output_size=n)
    p = s["flat"].float() if s["master"] is None else s["master"]
    p = p * keep - m / (1.0 - BETA1 ** step) / (r / math.sqrt(1.0 - BETA2 ** step) + EPS) * LR
    if eight:
        um, uv = _draws(n, step)
        _store8(m, um, s["m"], s["m_scale"], False)
        _store8(r, uv, s["v"], s["v_scale"], True)
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    s["flat"].copy_(p)
    if s["master"] is not None:
        s["master"].copy_(p)
        out["master"] = s["master"]
    s["step"] += 1
    return dict(out, p=s["flat"], m=s["m"], v=s["v"])


def _own(s):
    from paper_2606_05613_gb300 import native as bk

    case = s["case"]
    if case["op"] == "forward":
        bk.bkmoo_gate_forward(s["x"], s["wg"], s["wu"], case["act"], s["h"], s["a"], s["b"])
        return {"h": s["h"], "a": s["a"], "b": s["b"]} if case["save"] else {"h": s["h"]}
    if case["op"] == "backward":
        bk.bkmoo_gate_backward(s["dh"], s["a"], s["b"], s["x"], s["wg"], s["wu"], case["act"], s["rows"], s["dx"],
                               s["dwg"].unbind(0), s["dwu"].unbind(0))
        return {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"]}
    if case["op"] == "wgrad":
        bk.bkmoo_language_wgrad(s["dy"], s["x"], s["rows"], s["dw"].unbind(0), accumulate=case["accumulate"])
        return {"dw": s["dw"]}
    out = {"p": s["flat"], "m": s["m"], "v": s["v"]}
    p = bk.bkmoo_adamw_default_params()
    p.lr, p.beta1, p.beta2, p.eps, p.step, p.seed = LR, BETA1, BETA2, EPS, s["step"], SEED
    if case["clip"]:
        out["norm"] = torch.empty((), device=DEV)
        bk.bkmoo_grad_norm(s["grad"], out["norm"])
        p.max_norm = 1.0
    bk.bkmoo_adamw(s["params"], s["grad"], s["m"], s["v"], params=p, weight_decay=s["decay"], master=s["master"],
                   m_scale=s.get("m_scale"), v_scale=s.get("v_scale"), grad_norm=out.get("norm"))
    s["step"] += 1
    if case["state"] == "e4m3":
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    if s["master"] is not None:
        out["master"] = s["master"]
    return out


def run(state):
    if own:
        return _own(state)
    return {"forward": _forward, "backward": _backward, "wgrad": _language_wgrad, "adamw": _adamw_step}[state["case"]["op"]](state)


def work(case):
    if case["op"] == "forward":
        T, D, F = case["T"], case["D"], case["F"]
        return {"bytes": 2 * (T * D + 2 * F * D + T * F * (3 if case["save"] else 1)), "flops": 4 * T * D * F}
    if case["op"] == "backward":
        T, D, F, K = case["T"], case["D"], case["F"], case["K"]
        return {"bytes": 2 * (3 * T * F + 2 * T * D + 2 * F * D + 2 * K * F * D), "flops": 8 * T * D * F}
    if case["op"] == "wgrad":
        T, M, N, K = case["T"], case["M"], case["N"], case["K"]
        e = (4 if case["out"] == "f32" else 2) * (2 if case["accumulate"] else 1)
        return {"bytes": 2 * T * (M + N) + K * M * N * e, "flops": 2 * T * M * N}
    n = int(sum(_sizes(case)))
    p, g = (4 if case[k] == "f32" else 2 for k in ("param", "grad"))
    weights = 8 + p if case["master"] else 2 * p
    return {"bytes": n * (g + weights + (16 if case["state"] == "f32" else 4)), "flops": 16 * n}


# ---------------------------------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------------------------------

def _exact_act(name, a):
    if name == "silu":
        s = torch.sigmoid(a)
        return a * s, s + a * s * (1 - s)
    if name == "gelu":
        c = torch.special.ndtr(a)
        return a * c, c + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    z = math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)
    s = torch.sigmoid(2 * z)                      # (1 + tanh z) / 2
    return a * s, s + a * 2 * s * (1 - s) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * a ** 2)


def _exact_round8(x, u, positive):
    """The value and the scale of each element, u in [0, 1)."""
    n = x.numel()
    y = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = y.abs().amax(1) / 448
    y = (y / torch.where(scale > 0, scale, 1.0)[:, None]).view(-1)[:n]
    q = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    c = torch.floor(y.abs() / q + u) * q
    if positive:
        c = torch.where(y > 0, c.clamp_min(2.0 ** -9), c)
    return c.clamp_max(448) * torch.sign(y), scale


def exact(case, seed):
    if case["op"] in ("forward", "backward"):
        s = {k: v.double() if torch.is_tensor(v) else v for k, v in _gate_inputs(case, seed).items()}
        if case["op"] == "forward":
            a, b = s["x"] @ s["wg"].T, s["x"] @ s["wu"].T
            h = _exact_act(case["act"], a)[0] * b
            return {"h": h, "a": a, "b": b} if case["save"] else {"h": h}
        f, df = _exact_act(case["act"], s["a"])
        da, db = s["dh"] * s["b"] * df, s["dh"] * f
        out = {"dx": torch.addmm(da @ s["wg"], db, s["wu"])}
        for name, d in (("dwg", da), ("dwu", db)):
            out[name] = torch.zeros(case["K"], case["F"], case["D"], dtype=torch.float64, device=DEV)
            for k in range(case["K"]):
                i, j = s["rows"][k], s["rows"][k + 1]
                torch.mm(d[i:j].T, s["x"][i:j], out=out[name][k])
        return out
    if case["op"] == "wgrad":
        s = _wgrad_inputs(case, seed)
        dw = s["dw"].double()
        for k in range(case["K"]):
            i, j = s["rows"][k], s["rows"][k + 1]
            dw[k] += s["dy"][i:j].double().T @ s["x"][i:j].double()
        return {"dw": dw}
    s = _adamw_inputs(case, seed)
    g, n, out = s["grad"].double(), s["grad"].numel(), {}
    if case["clip"]:
        out["norm"] = torch.linalg.vector_norm(g)
        g *= min(1.0, 1.0 / (float(out["norm"]) + 1e-6))
    m, v = s["m"].double(), s["v"].double()
    if case["state"] == "e4m3":
        m *= s["m_scale"].double().repeat_interleave(BLOCK)[:n]
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)[:n]) ** 2
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
    del g
    decay = torch.repeat_interleave(torch.tensor(s["decay"], dtype=torch.float64, device=DEV), torch.tensor(s["sizes"], device=DEV), output_size=n)
    p = (s["flat"] if s["master"] is None else s["master"]).double()
    p -= LR * (decay * p + m / (1 - BETA1 ** STEP) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS))
    out["p"] = p
    if s["master"] is not None:
        out["master"] = p
    if case["state"] == "f32":
        return dict(out, m=m, v=v)
    um, uv = _draws(n, STEP)
    out["m"], out["m_scale"] = _exact_round8(m, um / 65536.0, False)
    out["v"], out["v_scale"] = _exact_round8(torch.sqrt(v), uv / 65536.0, True)
    return out
