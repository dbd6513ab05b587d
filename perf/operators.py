"""The operators that stand between the linear layers of a decoder block, as a training or serving
program calls them: root-mean-square norm with the residual's addition and dropout (forward, backward
with the gain's per-sample gradient norms), rotary positions, dropout from a counter, and the linear
layer in 8-bit floating point with a power-of-two scale for each block of 128.

`run` takes what `prepare` gives and makes one pass: with `own` false in elementary torch operations
in 32 bits, with `own` true through the library's entry points.  `exact` gives the same outputs in 64
bits from the definitions.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SEED, OFFSET = 0x5EED0123456789, 0x1_0000_0007      # of the dropout masks

_context = None


def _library():
    """The binding and the one context that a program keeps."""
    global _context
    from paper_2508_18182_b200 import binding
    if _context is None:
        _context = binding.Context(torch.cuda.current_device())
    return binding, _context


# ------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # a micro-batch of 32 sequences of 1024 tokens of the 12-layer model of width 768: what a block's
        # output goes through on its way into the next block
        {"name": "norm forward, micro-batch", "op": "norm", "B": 32, "T": 1024, "d": 768, "type": "bf16", "stream": "bf16", "p": 0.1},
        # the same place on the way back, with the gain's per-sample norms for the norm test
        {"name": "norm backward, micro-batch", "op": "norm_back", "B": 32, "T": 1024, "d": 768, "type": "bf16", "stream": "bf16", "p": 0.1},
        # full precision, an odd width and short sequences (a debugging or fine-tuning run)
        {"name": "norm backward, odd f32", "op": "norm_back", "B": 5, "T": 333, "d": 1001, "type": "f32", "stream": "f32", "p": 0.0},
        # queries and keys of the same micro-batch, still inside the packed product of the qkv layer
        {"name": "rope forward, micro-batch", "op": "rope", "B": 32, "T": 1024, "Hq": 12, "Hk": 12, "D": 64, "R": 64, "type": "bf16",
         "interleaved": False, "inverse": False, "scaling": "none", "factor": 1.0, "first": 0, "packed": True},
        # gradients of a long-context batch with shared key heads, half of each head rotated
        {"name": "rope backward, long context", "op": "rope", "B": 2, "T": 8192, "Hq": 32, "Hk": 8, "D": 128, "R": 64, "type": "bf16",
         "interleaved": True, "inverse": True, "scaling": "by_parts", "factor": 8.0, "first": 0, "packed": False},
        # one new token for each of 8 sequences, far into their contexts
        {"name": "rope, one token", "op": "rope", "B": 8, "T": 1, "Hq": 16, "Hk": 4, "D": 96, "R": 96, "type": "f32",
         "interleaved": False, "inverse": False, "scaling": "ntk", "factor": 4.0, "first": 100000, "packed": True},
        # dropout of a block's output (forward; the backward pass is the same call on the gradient)
        {"name": "dropout, micro-batch", "op": "dropout", "rows": 32768, "d": 768, "type": "bf16", "residual": False, "p": 0.1},
        # an odd number of elements in full precision, added to a residual
        {"name": "dropout and add, odd f32", "op": "dropout", "rows": 1, "d": 1000003, "type": "f32", "residual": True, "p": 0.5},
        # the qkv layer of the same model in 8 bits: activations quantised in the pass, weights beforehand
        {"name": "linear forward, micro-batch", "op": "linear", "M": 32768, "K": 768, "N": 2304, "back": False},
        # its gradient for the input: the output's gradient times the transposed weight
        {"name": "linear backward, micro-batch", "op": "linear", "M": 32768, "K": 768, "N": 2304, "back": True},
        # one token through a wide layer: the weight's bytes and the launch are all there is
        {"name": "linear, one token", "op": "linear", "M": 1, "K": 2048, "N": 8192, "back": False},
        # a few tokens through the norm with the 8-bit output and the layer that reads it
        {"name": "norm to 8 bits, linear, few tokens", "op": "norm_linear", "M": 3, "K": 2048, "N": 2048},
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of the listed ones' ranges; at most the work of the largest of its operator."""
    op = rng.choice(["norm", "norm_back", "rope", "dropout", "linear", "norm_linear"])
    if op in ("norm", "norm_back"):
        d = _spread(rng, 64, 4096)
        if rng.random() < 0.7:
            d = max(64, d // 16 * 16)
        tokens = _spread(rng, 1, 32 * 1024 * 768 // d // 2)
        B = min(64, _spread(rng, 1, tokens))
        kind = rng.choice([("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
        return {"op": op, "B": B, "T": max(1, tokens // B), "d": d, "type": kind[0], "stream": kind[1], "p": rng.choice([0.0, 0.1, 0.3])}
    if op == "rope":
        D = rng.choice([32, 64, 80, 96, 128, 256])
        R = rng.choice([D, D, D // 2, D // 4 // 2 * 2])
        Hk = rng.choice([1, 2, 4, 8, 12])
        Hq = Hk * rng.choice([1, 1, 2, 4])
        tokens = _spread(rng, 1, 32 * 1024 * 768 * 2 // ((Hq + Hk) * D) // 2)
        B = min(64, _spread(rng, 1, tokens))
        return {"op": op, "B": B, "T": max(1, tokens // B), "Hq": Hq, "Hk": Hk, "D": D, "R": R, "type": rng.choice(["bf16", "bf16", "f32"]),
                "interleaved": rng.random() < 0.5, "inverse": rng.random() < 0.5, "scaling": rng.choice(["none", "linear", "ntk", "by_parts"]),
                "factor": rng.choice([2.0, 4.0, 8.0]), "first": rng.choice([0, _spread(rng, 1, 500000)]), "packed": rng.random() < 0.5}
    if op == "dropout":
        d = _spread(rng, 64, 8192)
        return {"op": op, "rows": _spread(rng, 1, 32 * 1024 * 768 // d // 2), "d": d, "type": rng.choice(["bf16", "f32"]),
                "residual": rng.random() < 0.5, "p": rng.choice([0.05, 0.1, 0.2, 0.5])}
    K, N = _spread(rng, 128, 4096), _spread(rng, 128, 4096)
    if rng.random() < 0.7:
        K, N = max(128, K // 16 * 16), max(128, N // 16 * 16)
    if op == "linear":
        return {"op": op, "M": min(32768, _spread(rng, 1, 32768 * 768 * 2304 // (K * N) // 2)), "K": K, "N": N, "back": rng.random() < 0.5}
    return {"op": op, "M": min(8192, _spread(rng, 1, 32768 * 768 * 2304 // (K * N) // 2)), "K": K, "N": N}


def work(case):
    op = case["op"]
    if op in ("norm", "norm_back"):
        rows, d = case["B"] * case["T"], case["d"]
        x, s = (2 if case[k] == "bf16" else 4 for k in ("type", "stream"))
        if op == "norm":      # x, residual -> h, y and one reciprocal root a row; the gain
            return {"bytes": rows * d * (2 * x + 2 * s) + 4 * rows + 4 * d, "flops": 6.0 * rows * d}
        # dy, h, the stream's gradient -> its gradient and, under dropout, the branch's; the gain, its sum, the norms
        return {"bytes": rows * d * (x + 3 * s + (x if case["p"] > 0 else 0)) + 4 * rows + 8 * d + 4 * case["B"], "flops": 12.0 * rows * d}
    if op == "rope":
        n = case["B"] * case["T"] * (case["Hq"] + case["Hk"]) * case["D"]
        return {"bytes": 2 * n * (2 if case["type"] == "bf16" else 4) + 4 * case["B"] * case["T"], "flops": 3.0 * n * case["R"] / case["D"]}
    if op == "dropout":
        n = case["rows"] * case["d"]
        return {"bytes": n * (2 if case["type"] == "bf16" else 4) * (3 if case["residual"] else 2), "flops": 2.0 * n}
    M, K, N = case["M"], case["K"], case["N"]
    scales = -(-K // 128) * -(-N // 128)
    if op == "linear":
        return {"bytes": 2 * M * K + 2 * M * N + K * N + scales, "flops": 2.0 * M * K * N}
    return {"bytes": 6 * M * K + 2 * M * N + K * N + scales + 4 * K, "flops": 2.0 * M * K * N + 6.0 * M * K}


# ----------------------------------------------------------------------------------------- inputs

def _frequencies(R, base, scaling, factor, context, low, high):
    """Radians a position, one for each pair of a head's rotated part."""
    if scaling == "ntk":
        base = base * factor ** (R / (R - 2)) if R > 2 else base
    w = base ** (-2.0 * np.arange(R // 2, dtype=np.float64) / R)
    if scaling == "linear":
        w = w / factor
    if scaling == "by_parts":      # pairs that turn often within the trained context keep their speed
        keep = np.clip((w * context / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        w = w * keep + w / factor * (1.0 - keep)
    return w


ROPE = {"base": 10000.0, "context": 4096, "low": 1.0, "high": 32.0}


def _magnitude(case):
    return 1.0 + 0.1 * math.log(case["factor"]) if case["scaling"] == "by_parts" else 1.0


def _powers(amax):
    """2^e with the smallest whole e for which amax / 2^e is at most 448, the largest number of the
    8-bit format (4 exponent bits, 3 of the fraction); 1 for a block of zeros."""
    m, e = torch.frexp(amax)
    e = (e - 9 + (m > 0.875)).clamp(-127, 127)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def _padded(x, r, c):
    return torch.nn.functional.pad(x, (0, -x.shape[1] % c, 0, -x.shape[0] % r))


def _quantised_weight(W):
    """Values in 8 bits, and a power-of-two scale for each 128 x 128 block (biased exponents in a byte)."""
    N, K = W.shape
    blocks = _padded(W, 128, 128).view(-(-N // 128), 128, -(-K // 128), 128)
    s = _powers(blocks.abs().amax((1, 3)))
    q = (blocks / s[:, None, :, None]).reshape(-(-N // 128) * 128, -1)[:N, :K].to(torch.float8_e4m3fn)
    return q, (torch.log2(s) + 127).to(torch.uint8)


def _pitched(rows, cols, dtype, unit):
    """[rows, cols] with rows that start at multiples of `unit` elements."""
    return torch.zeros(rows, -(-cols // unit) * unit, dtype=dtype, device=DEV)[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device=DEV).mul_(std).to(dtype)

    s = dict(case)
    op = case["op"]
    if own:
        s["A"], s["ctx"] = _library()
    if op in ("norm", "norm_back"):
        B, T, d, x, h = case["B"], case["T"], case["d"], TYPES[case["type"]], TYPES[case["stream"]]
        s["gain"] = 1.0 + normal(d, std=0.1)
        # a mask for each seed: a training program counts its steps
        s["mask"] = (case["p"], SEED + seed, OFFSET) if case["p"] > 0 else None
        if op == "norm":
            s["x"], s["residual"] = normal(B, T, d, dtype=x), normal(B, T, d, std=2.0, dtype=h)
            s["out"] = {"h": torch.empty(B, T, d, dtype=h, device=DEV), "y": torch.empty(B, T, d, dtype=x, device=DEV),
                        "rstd": torch.empty(B, T, device=DEV)}
        else:
            s["h"] = normal(B, T, d, std=2.0, dtype=h)
            s["rstd"] = torch.rsqrt(s["h"].float().square().mean(-1) + EPS)
            s["dy"], s["dh_residual"] = normal(B, T, d, std=1e-2, dtype=x), normal(B, T, d, std=1e-2, dtype=h)
            s["out"] = {"dh": torch.empty(B, T, d, dtype=h, device=DEV), "norms": torch.empty(B, device=DEV), "sum": torch.empty(d, device=DEV)}
            if case["p"] > 0:
                s["out"]["dx"] = torch.empty(B, T, d, dtype=x, device=DEV)
    elif op == "rope":
        B, T, Hq, Hk, D, R, dt = (case[k] for k in ("B", "T", "Hq", "Hk", "D", "R", "type"))
        if case["packed"]:     # queries, keys and values side by side, as the layer before gives them
            qkv = normal(B, T, Hq + 2 * Hk, D, dtype=TYPES[dt])
            s["q"], s["k"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk]
        else:
            s["q"], s["k"] = normal(B, T, Hq, D, dtype=TYPES[dt]), normal(B, T, Hk, D, dtype=TYPES[dt])
        s["out"] = {"q": torch.empty(B, T, Hq, D, dtype=TYPES[dt], device=DEV), "k": torch.empty(B, T, Hk, D, dtype=TYPES[dt], device=DEV)}
        # each sequence starts at its own place, in `first` tokens from where the others do at most
        start = torch.randint(0, case["first"] + 1, (B, 1), generator=g, device=DEV, dtype=torch.int32)
        s["positions"] = start + torch.arange(T, device=DEV, dtype=torch.int32)
        w = _frequencies(R, ROPE["base"], case["scaling"], case["factor"], ROPE["context"], ROPE["low"], ROPE["high"])
        # turns a position, in units of 2^-64: a position's phase is then a product of whole numbers
        turns = np.floor(w / (2 * np.pi) * 2.0 ** 64 + 0.5).astype(np.uint64).view(np.int64)
        s["turns"] = torch.from_numpy(turns).to(DEV)
        if own:
            s["table"] = s["A"].RopeTable(R, base=ROPE["base"], scaling=case["scaling"], factor=case["factor"], context=ROPE["context"],
                                          low=ROPE["low"], high=ROPE["high"], magnitude=_magnitude(case))
    elif op == "dropout":
        dt = TYPES[case["type"]]
        s["x"] = normal(case["rows"], case["d"], dtype=dt)
        s["residual"] = normal(case["rows"], case["d"], dtype=dt) if case["residual"] else None
        s["mask"] = (case["p"], SEED + seed, OFFSET)
        s["out"] = {"y": torch.empty(case["rows"], case["d"], dtype=dt, device=DEV)}
    else:
        M, K, N = case["M"], case["K"], case["N"]
        back = case.get("back", False)
        W = normal(N, K, std=0.02)
        q, s["w_scale"] = _quantised_weight(W)
        s["w"] = _pitched(K, N, torch.float8_e4m3fn, 16) if back else _pitched(N, K, torch.float8_e4m3fn, 16)
        s["w"].copy_(q.t() if back else q)
        rows, cols = M, (N if back else K)
        s["out"] = {"y": torch.empty(M, K if back else N, dtype=torch.bfloat16, device=DEV)}
        s["q"], s["q_scale"] = _pitched(rows, cols, torch.float8_e4m3fn, 16), _pitched(rows, -(-cols // 128), torch.uint8, 4)
        if op == "linear":     # activations have columns of very different size; gradients are small
            s["x"] = (normal(M, cols) * torch.exp(normal(cols, std=1.0)) * (1e-3 if back else 1.0)).to(torch.bfloat16)
        else:
            s["x"], s["residual"], s["gain"] = normal(M, K, dtype=torch.bfloat16), normal(M, K, std=2.0, dtype=torch.bfloat16), torch.exp(normal(K, std=0.5))
            s["out"]["h"] = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    return s


# ------------------------------------------------------------------------------------- plain forms

def _kept(n, p, seed, offset):
    """Which of n elements stay, and what they are multiplied by.  Eight elements share one call of the
    counter-based generator Philox-4x32 of ten rounds (Salmon and others, 2011): counter = (index of the
    eight, offset), key = seed; element e takes 16 bits, the low or high half of word e // 2, and stays
    where they are at least the drop probability in units of 2^-16."""
    low = 0xFFFFFFFF
    i = torch.arange(-(-n // 8), device=DEV)
    c0, c1 = i & low, i >> 32
    c2, c3 = torch.full_like(i, offset & low), torch.full_like(i, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    bits = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 1)
    drop = round(p * 65536)
    return bits.view(-1)[:n] >= drop, 65536.0 / (65536 - drop)


def _dropped(x, mask):
    if mask is None:
        return x.float()
    keep, scale = _kept(x.numel(), *mask)
    return torch.where(keep.view(x.shape), x.float() * scale, 0.0)


def _plain_norm(s):
    h = s["residual"].float() + _dropped(s["x"], s.get("mask"))
    rstd = torch.rsqrt(h.square().mean(-1) + EPS)
    return h, rstd, h * rstd[..., None] * s["gain"]


def _plain_norm_back(s):
    h, dy, rstd = s["h"].float(), s["dy"].float(), s["rstd"][..., None]
    hat = h * rstd
    gdy = dy * s["gain"]
    dh = s["dh_residual"].float() + rstd * (gdy - hat * (gdy * hat).mean(-1, keepdim=True))
    each = (dy * hat).sum(1)      # the gain's gradient, sample by sample
    out = {"dh": dh.to(s["h"].dtype), "norms": each.square().sum(1), "sum": each.sum(0)}
    if s["mask"] is not None:
        out["dx"] = _dropped(dh, s["mask"]).to(s["dy"].dtype)
    return out


def _turned(x, cos, sin, R, interleaved):
    v = x.float()
    a, b = (v[..., 0:R:2], v[..., 1:R:2]) if interleaved else (v[..., :R // 2], v[..., R // 2:R])
    u, w = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, v[..., R:]], -1).to(x.dtype)


def _plain_rope(s):
    phase = (s["positions"].long()[..., None] * s["turns"]) >> 40       # modulo a whole turn, in 2^-24 of it
    angle = phase.float() * (2 * math.pi / 2 ** 24)
    m = _magnitude(s)
    cos, sin = m * torch.cos(angle)[:, :, None], m * torch.sin(angle)[:, :, None]
    if s["inverse"]:
        sin = -sin
    return {n: _turned(s[n], cos, sin, s["R"], s["interleaved"]) for n in ("q", "k")}


def _block_rounded(x):
    """What x stands for after its rows' blocks of 128 have gone to 8 bits."""
    blocks = _padded(x, 1, 128).view(x.shape[0], -1, 128)
    p = _powers(blocks.abs().amax(-1, keepdim=True))
    return ((blocks / p).to(torch.float8_e4m3fn).float() * p).view(x.shape[0], -1)[:, :x.shape[1]]


def _plain_product(x, s):
    scale = torch.exp2(s["w_scale"].float() - 127)
    if s.get("back"):
        scale = scale.t()
    w = s["w"].float()
    w = w * scale.repeat_interleave(128, 0)[:w.shape[0]].repeat_interleave(128, 1)[:, :w.shape[1]]
    return (_block_rounded(x) @ w.t()).to(torch.bfloat16)


def run(state):
    s, op = state, state["op"]
    if own:
        return _run_library(s)
    if op == "norm":
        h, rstd, y = _plain_norm(s)
        return {"h": h.to(s["residual"].dtype), "y": y.to(s["x"].dtype), "rstd": rstd}
    if op == "norm_back":
        return _plain_norm_back(s)
    if op == "rope":
        return _plain_rope(s)
    if op == "dropout":
        y = _dropped(s["x"], s["mask"])
        return {"y": (y if s["residual"] is None else s["residual"].float() + y).to(s["x"].dtype)}
    if op == "linear":
        return {"y": _plain_product(s["x"].float(), s)}
    h, _, y = _plain_norm(s)
    return {"y": _plain_product(y, s), "h": h.to(torch.bfloat16)}


# ------------------------------------------------------------------------------- the library's calls

def _run_library(s):
    ctx, out, op = s["ctx"], s["out"], s["op"]
    if op == "norm":
        ctx.add_rmsnorm(s["x"], s["gain"], residual=s["residual"], h=out["h"], y=out["y"], rstd=out["rstd"], eps=EPS, dropout=s["mask"])
    elif op == "norm_back":
        ctx.add_rmsnorm_backward(s["dy"], s["h"], s["rstd"], s["gain"], out["dh"], dh_residual=s["dh_residual"], dx=out.get("dx"),
                                 dropout=s["mask"], per_sample_sqnorm=out["norms"], grad_sum=out["sum"])
    elif op == "rope":
        ctx.rope([s["q"], s["k"]], s["table"], outs=[out["q"], out["k"]], positions=s["positions"], interleaved=s["interleaved"],
                 inverse=s["inverse"])
    elif op == "dropout":
        ctx.dropout(s["x"], out["y"], p=s["mask"][0], seed=s["mask"][1], offset=s["mask"][2], residual=s["residual"])
    else:
        if op == "linear":
            ctx.blockscale_quantize(s["x"], s["q"], s["q_scale"])
        else:
            ctx.add_rmsnorm(s["x"], s["gain"], residual=s["residual"], h=out["h"], q=s["q"], q_scale=s["q_scale"], eps=EPS)
        ctx.blockscale_matmul(s["q"], s["q_scale"], s["w"], s["w_scale"], out["y"], scale_transposed=s.get("back", False))
    return out


# --------------------------------------------------------------------------------------- in 64 bits

def _stays(n, p, seed, offset):
    """The same definition of the mask in unsigned whole numbers."""
    u = np.uint64
    low = u(0xFFFFFFFF)
    i = np.arange((n + 7) // 8, dtype=u)
    c = [i & low, i >> u(32), np.full_like(i, offset & 0xFFFFFFFF), np.full_like(i, offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        c = [(b >> u(32)) ^ c[1] ^ u(key[0]), b & low, (a >> u(32)) ^ c[3] ^ u(key[1]), a & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    words = np.stack(c, 1).astype(np.uint32)
    halves = np.ascontiguousarray(words).view(np.uint16).reshape(-1)      # little-endian: low half first
    return torch.from_numpy(halves[:n] >= np.uint32(round(p * 65536))).to(DEV)


def _scaled_mask(x, mask):
    x = x.double()
    if mask is None:
        return x
    kept = _stays(x.numel(), *mask).view(x.shape)
    return torch.where(kept, x / (1.0 - round(mask[0] * 65536) / 65536), torch.zeros_like(x))


def _exact_norm(s):
    h = s["residual"].double() + _scaled_mask(s["x"], s.get("mask"))
    root = ((h * h).sum(-1) / h.shape[-1] + EPS) ** -0.5
    return h, root, s["gain"].double() * h * root.unsqueeze(-1)


def _exact_8_bits(x, amax):
    """Rounded to the nearest multiple of the step at each magnitude, ties to even, relative to the block's scale."""
    e = torch.ceil(torch.log2(amax / 448.0)).clamp(-127, 127)
    e = torch.where(amax * torch.exp2(-e) > 448.0, e + 1, e)
    e = torch.where(amax * torch.exp2(1.0 - e) <= 448.0, e - 1, e)
    scale = torch.where(amax > 0, torch.exp2(e), torch.ones_like(amax))
    v = x / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step * scale


def _exact_product(x, s):
    rows, cols = x.shape
    wide = torch.zeros(rows, -(-cols // 128) * 128, dtype=torch.float64, device=DEV)
    wide[:, :cols] = x
    v = wide.reshape(rows, -1, 128)
    x = _exact_8_bits(v, v.abs().max(-1, keepdim=True).values.expand_as(v)).reshape(rows, -1)[:, :cols]
    e = s["w_scale"].double() - 127
    e = e.T if s.get("back") else e
    r = torch.arange(s["w"].shape[0], device=DEV) // 128
    c = torch.arange(s["w"].shape[1], device=DEV) // 128
    return x @ (s["w"].double() * torch.exp2(e[r][:, c])).T


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm":
        h, root, y = _exact_norm(s)
        return {"h": h, "y": y, "rstd": root}
    if op == "norm_back":
        h, dy, r, g, d = s["h"].double(), s["dy"].double(), s["rstd"].double().unsqueeze(-1), s["gain"].double(), case["d"]
        dot = (dy * g * h).sum(-1, keepdim=True)
        dh = s["dh_residual"].double() + r * dy * g - h * r ** 3 * dot / d
        each = torch.einsum("btd,btd->bd", dy, h * r)
        out = {"dh": dh, "norms": (each ** 2).sum(1), "sum": each.sum(0)}
        if s["mask"] is not None:
            out["dx"] = _scaled_mask(dh, s["mask"])
        return out
    if op == "rope":
        R = case["R"]
        w = _frequencies(R, ROPE["base"], case["scaling"], case["factor"], ROPE["context"], ROPE["low"], ROPE["high"])
        angle = s["positions"].double().unsqueeze(-1) * torch.from_numpy(w).to(DEV) * (-1.0 if case["inverse"] else 1.0)
        z = torch.polar(torch.full_like(angle, _magnitude(case)), angle).unsqueeze(2)
        out = {}
        for n in ("q", "k"):
            v = s[n].double()
            if case["interleaved"]:
                pairs = torch.view_as_complex(v[..., :R].reshape(*v.shape[:3], R // 2, 2).contiguous())
                v[..., :R] = torch.view_as_real(pairs * z).reshape(*v.shape[:3], R)
            else:
                pairs = torch.complex(v[..., :R // 2], v[..., R // 2:R]) * z
                v[..., :R // 2], v[..., R // 2:R] = pairs.real, pairs.imag
            out[n] = v
        return out
    if op == "dropout":
        y = _scaled_mask(s["x"], s["mask"])
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    if op == "linear":
        return {"y": _exact_product(s["x"].double(), s)}
    h, _, y = _exact_norm(s)
    return {"y": _exact_product(y, s), "h": h}
