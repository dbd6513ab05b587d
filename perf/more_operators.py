"""The feed-forward block and the loss of a decoder, as a training or serving program calls them: the linear layer
with bias, activation and residual in its product, the gated pair of projections with their backward pass, their
inputs to the backward pass kept in 8 bits, and the log-probabilities of given tokens with entropy, best
alternatives and gradient.

`run` takes what `prepare` gives and makes one pass: with `own` false in elementary torch operations in 32 bits,
with `own` true through the library's entry points.  `exact` gives the same outputs in 64 bits from the definitions.
"""
import math

import torch

own = False

DEV = "cuda"
BF16 = torch.bfloat16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

_context = None


def _library():
    """The one context that a program keeps."""
    global _context
    if _context is None:
        from paper_2508_18182_b200 import binding
        _context = binding.Context(torch.cuda.current_device())
    return _context


# ------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # a micro-batch of 32 sequences of 1024 tokens of the model of width 768: the first layer of a feed-forward with
        # bias and activation; what the activation's derivative needs is kept
        {"name": "linear forward, micro-batch", "op": "linear", "M": 32768, "K": 768, "N": 2048, "act": "gelu", "bias": True, "residual": False, "keep": True, "type": "bf16"},
        # the way back through the second layer and that activation
        {"name": "linear backward, micro-batch", "op": "linear_back", "M": 32768, "K": 2048, "N": 768, "act": "gelu"},
        # odd sizes, into a residual stream in full precision (a debugging or fine-tuning run)
        {"name": "linear forward, odd, f32 stream", "op": "linear", "M": 1665, "K": 1001, "N": 777, "act": "none", "bias": True, "residual": True, "keep": False, "type": "f32"},
        # one token through a wide layer: the weight's bytes are all there is
        {"name": "linear, one token", "op": "linear", "M": 1, "K": 2048, "N": 8192, "act": "gelu_tanh", "bias": True, "residual": False, "keep": False, "type": "bf16"},
        # the gated feed-forward of the same micro-batch, both projections kept for the backward pass
        {"name": "gated forward, micro-batch", "op": "gated", "M": 32768, "d": 768, "f": 2048, "act": "silu", "keep": True},
        # the way back through the block's last layer, the product and the activation
        {"name": "gated backward, micro-batch", "op": "gated_back", "M": 32768, "d": 768, "f": 2048, "act": "silu"},
        # forward and backward of a wider block that keeps its projections in 8 bits and recomputes the rest
        {"name": "gated with 8-bit checkpoints, wide", "op": "gated_checkpoints", "M": 4096, "d": 2048, "f": 5632, "act": "silu"},
        # a few tokens of a generation through that block's first layers
        {"name": "gated, few tokens", "op": "gated", "M": 3, "d": 2048, "f": 5632, "act": "silu", "keep": False},
        # a layer's input back from 8 bits, for the weight's gradient and its per-sample norms
        {"name": "restore a checkpoint, micro-batch", "op": "restore", "M": 32768, "d": 768, "type": "bf16"},
        # the loss of 8 sequences of 1024 tokens over the vocabulary of 50257, with entropy and the 8 best tokens
        {"name": "log-probabilities, micro-batch", "op": "logprobs", "rows": 8192, "V": 50257, "top": 8, "type": "bf16", "banned": False},
        # its gradient: of the given tokens and of the entropy (a bonus for exploring)
        {"name": "log-probabilities backward, micro-batch", "op": "logprobs_back", "rows": 8192, "V": 50257, "type": "bf16", "entropy": True},
        # the next token of four generations, a tenth of the vocabulary ruled out, 20 alternatives
        {"name": "log-probabilities, few rows", "op": "logprobs", "rows": 4, "V": 131072, "top": 20, "type": "f32", "banned": True},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    n = _spread(rng, low, high)
    return max(low, n // 16 * 16) if rng.random() < 0.6 else n


def draw(rng):
    """One more case of the listed ones' ranges; at most the work of the largest of its operator."""
    op = rng.choice(["linear", "linear", "linear_back", "gated", "gated", "gated_back", "gated_checkpoints", "restore", "logprobs", "logprobs", "logprobs_back"])
    few = rng.random() < 0.25      # tokens of a generation
    if op in ("linear", "linear_back"):
        K, N = _width(rng, 64, 4096), _width(rng, 64, 8192)
        M = rng.randint(1, 16) if few else min(32768, _spread(rng, 17, max(18, 32768 * 768 * 2048 // (K * N) // 2)))
        act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
        if op == "linear_back":
            return {"op": op, "M": M, "K": K, "N": N, "act": act}
        return {"op": op, "M": M, "K": K, "N": N, "act": act, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5,
                "keep": rng.random() < 0.3, "type": rng.choice(["bf16", "bf16", "f32"])}
    if op in ("gated", "gated_back", "gated_checkpoints"):
        d, f = _width(rng, 64, 4096), _width(rng, 128, 8192)
        M = rng.randint(1, 16) if few else min(32768, _spread(rng, 17, max(18, 32768 * 768 * 2048 // (d * f) // 2)))
        case = {"op": op, "M": M, "d": d, "f": f, "act": rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])}
        return {**case, "keep": rng.random() < 0.5} if op == "gated" else case
    if op == "restore":
        d = _width(rng, 64, 8192)
        return {"op": op, "M": _spread(rng, 1, 32768 * 768 // d), "d": d, "type": rng.choice(["bf16", "f32"])}
    V = _spread(rng, 200, 200000)
    rows = rng.randint(1, 16) if few else min(65536, _spread(rng, 1, max(2, 8192 * 50257 // V // 3)))
    case = {"op": op, "rows": rows, "V": V, "type": rng.choice(["bf16", "bf16", "f32"])}
    if op == "logprobs_back":
        return {**case, "entropy": rng.random() < 0.5}
    return {**case, "top": rng.choice([0, 1, 5, 8, 20]), "banned": rng.random() < 0.3}


def work(case):
    op = case["op"]
    if op in ("linear", "linear_back"):
        M, K, N = case["M"], case["K"], case["N"]
        if op == "linear_back":      # dy, w, z -> dx and the activation's value
            return {"bytes": 2 * M * N + 2 * N * K + (6 if case["act"] != "none" else 2) * M * K, "flops": 2.0 * M * K * N}
        e = 2 if case["type"] == "bf16" else 4
        return {"bytes": 2 * M * K + 2 * N * K + M * N * (e * (2 if case["residual"] else 1) + (2 if case["keep"] else 0)) + (4 * N if case["bias"] else 0),
                "flops": 2.0 * M * K * N}
    if op in ("gated", "gated_back", "gated_checkpoints"):
        M, d, f = case["M"], case["d"], case["f"]
        if op == "gated":
            return {"bytes": 2 * M * d + 4 * d * f + M * f * (6 if case["keep"] else 2), "flops": 4.0 * M * d * f}
        if op == "gated_back":       # dy, w, gate, up -> three more
            return {"bytes": 2 * M * d + 2 * d * f + 10 * M * f, "flops": 2.0 * M * d * f}
        return {"bytes": 4 * M * d + 6 * d * f + 12 * M * f + 4 * M * -(-f // 128), "flops": 6.0 * M * d * f}
    if op == "restore":
        n = case["M"] * case["d"]
        return {"bytes": n * (3 if case["type"] == "bf16" else 5) + case["M"] * -(-case["d"] // 128), "flops": 1.0 * n}
    n, e = case["rows"] * case["V"], 2 if case["type"] == "bf16" else 4
    if op == "logprobs_back":
        return {"bytes": 2 * n * e + case["rows"] * (20 if case["entropy"] else 12), "flops": 6.0 * n}
    return {"bytes": n * e + case["rows"] * (16 + 8 * case["top"]), "flops": 6.0 * n}


# ----------------------------------------------------------------------------------------- inputs

def _pitched(rows, cols, dtype, unit):
    """[rows, cols] with rows that start at multiples of `unit` elements."""
    return torch.zeros(rows, -(-cols // unit) * unit, dtype=dtype, device=DEV)[:, :cols]


def _bytes_for(rows, cols):
    """A matrix in 8 bits, and a power-of-two scale for each 128 elements of a row (biased exponents in a byte)."""
    return _pitched(rows, cols, torch.float8_e4m3fn, 16), _pitched(rows, -(-cols // 128), torch.uint8, 4)


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.shape[1] % 128)).view(x.shape[0], -1, 128)


def _powers(blocks):
    """2^e with the smallest whole e for which a block's largest magnitude over 2^e is at most 448, the largest number
    of the 8-bit format (4 exponent bits, 3 of the fraction); 1 for a block of zeros."""
    amax = blocks.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)
    e = (e - 9 + (m > 0.875)).clamp(-127, 127)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEV).mul_(std)

    def rows(*shape, std=1.0):      # an operand of a product
        x = _pitched(*shape, BF16, 8)
        x.copy_(normal(*shape, std=std))
        return x

    s = dict(case)
    op = case["op"]
    if own:
        s["ctx"] = _library()
    if op == "linear":
        M, K, N, dt = case["M"], case["K"], case["N"], TYPES[case["type"]]
        s["x"], s["w"] = rows(M, K), rows(N, K, std=K ** -0.5)
        s["b"] = normal(N, std=0.2) if case["bias"] else None
        s["r"] = normal(M, N, std=2.0).to(dt) if case["residual"] else None
        s["out"] = {"y": torch.empty(M, N, dtype=dt, device=DEV)}
        if case["keep"]:
            s["out"]["z"] = _pitched(M, N, BF16, 8)
    elif op == "linear_back":
        M, K, N = case["M"], case["K"], case["N"]
        s["dy"], s["w"] = rows(M, N, std=1e-2), rows(N, K, std=K ** -0.5)
        s["out"] = {"dx": _pitched(M, K, BF16, 8)}
        if case["act"] != "none":
            s["z"] = rows(M, K)
            s["out"]["a"] = _pitched(M, K, BF16, 8)
    elif op in ("gated", "gated_back", "gated_checkpoints"):
        M, d, f = case["M"], case["d"], case["f"]
        s["out"] = {"a": _pitched(M, f, BF16, 8)}
        if op != "gated_back":
            s["x"], s["w_gate"], s["w_up"] = rows(M, d), rows(f, d, std=d ** -0.5), rows(f, d, std=d ** -0.5)
        if op != "gated":
            s["dy"], s["w_down"] = rows(M, d, std=1e-2), rows(d, f, std=f ** -0.5)
            s["out"]["d_gate"], s["out"]["d_up"] = _pitched(M, f, BF16, 8), _pitched(M, f, BF16, 8)
        if op == "gated_back":
            s["gate"], s["up"] = rows(M, f), rows(M, f)
        elif op == "gated_checkpoints":
            s["gate"], s["up"] = _bytes_for(M, f), _bytes_for(M, f)
            s["out"]["again"] = _pitched(M, f, BF16, 8)
        elif case["keep"]:
            s["out"]["gate"], s["out"]["up"] = _pitched(M, f, BF16, 8), _pitched(M, f, BF16, 8)
    elif op == "restore":
        M, d = case["M"], case["d"]
        s["q"], s["scale"] = _bytes_for(M, d)
        blocks = _blocks(normal(M, d) * torch.exp(normal(d)))
        p = _powers(blocks)
        s["q"].copy_((blocks / p).view(M, -1)[:, :d].to(torch.float8_e4m3fn))
        s["scale"].copy_((torch.log2(p[..., 0]) + 127).to(torch.uint8))
        s["out"] = {"x": torch.empty(M, d, dtype=TYPES[case["type"]], device=DEV)}
    else:
        n, V, dt = case["rows"], case["V"], TYPES[case["type"]]
        s["logits"] = torch.empty(n, V, dtype=dt, device=DEV)
        for part in s["logits"].split(1024):
            part.copy_(normal(*part.shape, std=2.5))
        if case.get("banned"):
            s["logits"].masked_fill_(torch.rand(V, generator=g, device=DEV) < 0.1, float("-inf"))
        s["targets"] = torch.randint(0, V, (n,), generator=g, device=DEV, dtype=torch.int32)
        s["targets"][torch.rand(n, generator=g, device=DEV) < 0.1] = -1           # tokens of a prompt have no loss

        def vector(dtype=torch.float32):
            return torch.empty(n, dtype=dtype, device=DEV)
        if op == "logprobs":
            s["out"] = {"logp": vector(), "entropy": vector(), "lse": vector()}
            if case["top"]:
                s["out"]["top_values"] = torch.empty(n, case["top"], device=DEV)
                s["out"]["top_ids"] = torch.empty(n, case["top"], dtype=torch.int32, device=DEV)
        else:
            s["lse"] = torch.cat([part.double().logsumexp(1).float() for part in s["logits"].split(1024)])
            s["d_logp"] = normal(n, std=1e-3)
            if case["entropy"]:
                s["entropy"] = torch.cat([_exact_entropy(part.double()) for part in s["logits"].split(1024)]).float()
                s["d_entropy"] = normal(n, std=1e-4)
            s["out"] = {"d_logits": torch.empty(n, V, dtype=dt, device=DEV)}
    return s


# ------------------------------------------------------------------------------------- plain forms

def _act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z


def _slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        sig = 1 / (1 + torch.exp(-z))
        return sig * (1 + z * (1 - sig))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if name == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _kept_8_bits(x):
    """What x stands for after its rows' blocks of 128 have gone to 8 bits."""
    blocks = _blocks(x)
    p = _powers(blocks)
    return ((blocks / p).to(torch.float8_e4m3fn).float() * p).view(x.shape[0], -1)[:, :x.shape[1]]


def _plain_gated_back(s, gate, up):
    da = s["dy"].float() @ s["w_down"].float()
    act = _act(gate, s["act"])
    return {"d_gate": (da * up * _slope(gate, s["act"])).to(BF16), "d_up": (da * act).to(BF16)}, (act * up).to(BF16)


def _plain_logprobs(s):
    l = s["logits"].float()
    m = l.amax(1, keepdim=True)
    e = torch.exp(l - m)
    total = e.sum(1, keepdim=True)
    lse = (m + torch.log(total))[:, 0]
    t = s["targets"].long()
    logp = torch.where(t >= 0, l.gather(1, t.clamp_min(0)[:, None])[:, 0] - lse, 0.0)
    mean = torch.where(e > 0, e * (l - m), 0.0).sum(1) / total[:, 0]
    out = {"logp": logp, "entropy": torch.log(total[:, 0]) - mean, "lse": lse}
    if s["top"]:      # a number's place and then its index, in one whole number
        del e
        order = (l + 0.0).view(torch.int32)
        order = (order ^ ((order >> 31) & 0x7FFFFFFF)).long()
        key = (order << 32).add_(torch.arange(l.shape[1] - 1, -1, -1, device=DEV))
        ids = l.shape[1] - 1 - (key.topk(s["top"], 1).values & 0xFFFFFFFF)
        out["top_values"], out["top_ids"] = l.gather(1, ids) - lse[:, None], ids.int()
    return out


def _plain_logprobs_back(s):
    l = s["logits"].float()
    logp = l - s["lse"][:, None]
    p = torch.exp(logp)
    t = s["targets"].long()
    scale = torch.where(t >= 0, s["d_logp"], 0.0)[:, None]
    d = -scale * p
    if s["entropy"] is not False:
        d -= s["d_entropy"][:, None] * p * (logp + s["entropy"][:, None])
    d.scatter_add_(1, t.clamp_min(0)[:, None], scale)
    return {"d_logits": d.to(s["logits"].dtype)}


def run(state):
    s, op = state, state["op"]
    if own:
        return _run_library(s)
    if op == "linear":
        z = s["x"].float() @ s["w"].float().t()
        if s["b"] is not None:
            z = z + s["b"]
        y = _act(z, s["act"])
        if s["r"] is not None:
            y = s["r"].float() + y
        out = {"y": y.to(TYPES[s["type"]])}
        if s["keep"]:
            out["z"] = z.to(BF16)
        return out
    if op == "linear_back":
        dx = s["dy"].float() @ s["w"].float()
        if s["act"] == "none":
            return {"dx": dx.to(BF16)}
        z = s["z"].float()
        return {"dx": (dx * _slope(z, s["act"])).to(BF16), "a": _act(z, s["act"]).to(BF16)}
    if op in ("gated", "gated_checkpoints"):
        gate, up = s["x"].float() @ s["w_gate"].float().t(), s["x"].float() @ s["w_up"].float().t()
        out = {"a": (_act(gate, s["act"]) * up).to(BF16)}
        if op == "gated_checkpoints":
            back, out["again"] = _plain_gated_back(s, _kept_8_bits(gate), _kept_8_bits(up))
            out.update(back)
        elif s["keep"]:
            out["gate"], out["up"] = gate.to(BF16), up.to(BF16)
        return out
    if op == "gated_back":
        out, a = _plain_gated_back(s, s["gate"].float(), s["up"].float())
        return {**out, "a": a}
    if op == "restore":
        scale = torch.exp2(s["scale"].float() - 127).repeat_interleave(128, 1)[:, :s["d"]]
        return {"x": (s["q"].float() * scale).to(TYPES[s["type"]])}
    return _plain_logprobs(s) if op == "logprobs" else _plain_logprobs_back(s)


# ------------------------------------------------------------------------------- the library's calls

def _run_library(s):
    ctx, out, op = s["ctx"], s["out"], s["op"]
    if op == "linear":
        ctx.linear(s["x"], s["w"], out["y"], bias=s["b"], activation=s["act"], residual=s["r"], z=out.get("z"))
    elif op == "linear_back":
        ctx.linear_backward(s["dy"], s["w"], out["dx"], activation=s["act"], z=s.get("z"), a=out.get("a"))
    elif op == "gated":
        ctx.gated_linear(s["x"], s["w_gate"], s["w_up"], out["a"], activation=s["act"], gate=out.get("gate"), up=out.get("up"))
    elif op == "gated_back":
        ctx.gated_linear_backward(s["dy"], s["w_down"], s["gate"], s["up"], out["d_gate"], out["d_up"], activation=s["act"], a=out["a"])
    elif op == "gated_checkpoints":
        (gate, gate_scale), (up, up_scale) = s["gate"], s["up"]
        ctx.gated_linear(s["x"], s["w_gate"], s["w_up"], out["a"], activation=s["act"], gate=gate, gate_scale=gate_scale, up=up, up_scale=up_scale)
        ctx.gated_linear_backward(s["dy"], s["w_down"], gate, up, out["d_gate"], out["d_up"], activation=s["act"], gate_scale=gate_scale,
                                  up_scale=up_scale, a=out["again"])
    elif op == "restore":
        ctx.blockscale_dequantize(s["q"], s["scale"], out["x"])
    elif op == "logprobs":
        ctx.token_logprobs(s["logits"], s["targets"], out["logp"], entropy=out["entropy"], lse=out["lse"], top_values=out.get("top_values"),
                           top_ids=out.get("top_ids"))
    else:
        given = {"entropy": s["entropy"], "d_entropy": s["d_entropy"]} if "d_entropy" in s else {}
        ctx.token_logprobs_backward(s["logits"], s["targets"], s["lse"], s["d_logp"], out["d_logits"], **given)
    return out


# --------------------------------------------------------------------------------------- in 64 bits

def _exact_entropy(l):
    p = torch.softmax(l, 1)
    return -torch.special.xlogy(p, p).sum(1)


def _exact_act(z, name):
    """Value and derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return torch.relu(z), torch.heaviside(z, torch.zeros_like(z))
    if name == "silu":
        h = torch.sigmoid(z)
        return z * h, h + z * h * torch.sigmoid(-z)
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * cdf, cdf + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    k = math.sqrt(8 / math.pi)      # (1 + tanh(v)) / 2 is the logistic function of 2 v
    h = torch.sigmoid(k * z * (1 + 0.044715 * z.square()))
    return z * h, h + z * h * (1 - h) * k * (1 + 0.134145 * z.square())


def _exact_8_bits(x):
    """Rounded to the nearest number of 8 bits, ties to even, relative to the scale of its row's block of 128: a multiple
    of the step at its magnitude, which stays that of 2^-6 below it."""
    v = _blocks(x)
    amax = v.abs().amax(2, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(amax / 448.0)))
    scale = torch.where(amax > 448.0 * scale, 2 * scale, torch.where(2 * amax <= 448.0 * scale, scale / 2, scale))
    scale = torch.where(amax > 0, scale, torch.ones_like(scale))
    step = torch.exp2(torch.floor(torch.log2((v.abs() / scale).clamp_min(2.0 ** -6))) - 3) * scale
    return (torch.round(v / step) * step).reshape(x.shape[0], -1)[:, :x.shape[1]]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "linear":
        z = torch.einsum("mk,nk->mn", s["x"].double(), s["w"].double())
        if s["b"] is not None:
            z += s["b"].double()
        y = _exact_act(z, case["act"])[0]
        out = {"y": y if s["r"] is None else y + s["r"].double()}
        if case["keep"]:
            out["z"] = z
        return out
    if op == "linear_back":
        dx = torch.einsum("mn,nk->mk", s["dy"].double(), s["w"].double())
        if case["act"] == "none":
            return {"dx": dx}
        a, slope = _exact_act(s["z"].double(), case["act"])
        return {"dx": dx * slope, "a": a}
    if op in ("gated", "gated_back", "gated_checkpoints"):
        if op == "gated_back":
            gate, up = s["gate"].double(), s["up"].double()
        else:
            gate, up = (torch.einsum("md,fd->mf", s["x"].double(), s[w].double()) for w in ("w_gate", "w_up"))
        act, slope = _exact_act(gate, case["act"])
        out = {"a": act * up}
        if op == "gated":
            if case["keep"]:      # before the rounding to the type that they are kept in
                out["gate"], out["up"] = gate, up
            return out
        if op == "gated_checkpoints":
            gate, up = _exact_8_bits(gate), _exact_8_bits(up)
            act, slope = _exact_act(gate, case["act"])
            out["again"] = act * up
        da = torch.einsum("md,df->mf", s["dy"].double(), s["w_down"].double())
        out["d_gate"], out["d_up"] = da * up * slope, da * act
        return out
    if op == "restore":
        at = torch.arange(case["d"], device=DEV) // 128
        return {"x": s["q"].double() * torch.exp2(s["scale"].double() - 127)[:, at]}
    t = s["targets"].long()
    if op == "logprobs_back":
        d = torch.empty(*s["logits"].shape, dtype=torch.float64, device=DEV)
        for i in range(0, case["rows"], 1024):
            part = slice(i, i + 1024)
            logp = s["logits"][part].double() - s["lse"][part, None].double()
            hit = torch.arange(case["V"], device=DEV) == t[part, None]
            d[part] = (t[part, None] >= 0) * s["d_logp"][part, None].double() * (hit.double() - logp.exp())
            if case["entropy"]:
                d[part] -= s["d_entropy"][part, None].double() * logp.exp() * (logp + s["entropy"][part, None].double())
        return {"d_logits": d}
    found = []
    for i in range(0, case["rows"], 1024):
        l = s["logits"][i:i + 1024].double()
        lse, ti = torch.logsumexp(l, 1), t[i:i + 1024]
        of = torch.where(ti >= 0, l[torch.arange(len(l), device=DEV), ti.clamp_min(0)] - lse, torch.zeros_like(lse))
        one = {"logp": of, "entropy": _exact_entropy(l), "lse": lse}
        if case["top"]:
            best, ids = torch.sort(l, dim=1, descending=True, stable=True)
            one["top_values"], one["top_ids"] = best[:, :case["top"]] - lse[:, None], ids[:, :case["top"]].int()
        found.append(one)
    return {k: torch.cat([f[k] for f in found]) for k in found[0]}
