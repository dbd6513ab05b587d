"""Random calls of the linear layers and of the loss against the fp64 oracle: sizes, pitches, types, what is kept and what is
left out, each drawn from a seed.  Tolerances as in test_gpu_layers.py and test_gpu_token_logprobs.py."""
import random

import numpy as np
import pytest
import torch

import oracle.block_oracle as B
import oracle.layer_oracle as L
from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    assert c.device_status() == 0
    c.close()


def np64(t):
    return t.detach().double().cpu().numpy()


def matrix(r, n, d, std=1.0, dtype=BF, aligned=True):
    pad = r.choice([0, 0, 8, 24]) if aligned else r.choice([0, 1, 3, 5])
    pitch = (-(-d // 8) * 8 if aligned else d) + pad
    g = torch.Generator().manual_seed(r.randrange(1 << 30))
    t = torch.full((n, pitch), float("nan"), dtype=dtype, device=DEV)
    t[:, :d] = (torch.randn(n, d, generator=g) * std).to(dtype).to(DEV)
    return t[:, :d]


def empty(r, n, d, dtype=BF):
    pitch = d + r.choice([0, 0, 0, 1, 7, 8, 16 - d % 8])
    return torch.full((n, pitch), -5.0, dtype=dtype, device=DEV)[:, :d]


def eight_bits(ctx, n, d, x=None):
    q = torch.zeros(n, -(-d // 16) * 16, dtype=torch.uint8, device=DEV)[:, :d]
    s = torch.zeros(n, -(-d // 512) * 4, dtype=torch.uint8, device=DEV)[:, :-(-d // 128)]
    if x is not None:
        ctx.blockscale_quantize(x, q, s)
    return q, s


def values(q, s):
    return B.widen(np64(q.contiguous().view(torch.float8_e4m3fn)), s.cpu().numpy().astype(np.int64) - 127, 1)


def extent(r, most):
    n = int(round(2 ** r.uniform(0, np.log2(most))))
    return max(1, n // 8 * 8) if r.random() < 0.4 and n >= 8 else n


def close(got, ref, tol, what):
    off = ~(np.abs(np64(got) - ref) <= tol)
    assert not off.any(), f"{what}: {off.sum()} of {off.size}, worst {np.nanmax(np.abs(np64(got) - ref) / np.maximum(tol, 1e-300)):.3g} of the tolerance"


def step(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -24


@pytest.mark.parametrize("seed", range(60))
def test_random_layer(ctx, seed):
    r = random.Random(seed)
    M, N, K, act = extent(r, 3000), extent(r, 2500), extent(r, 1500), r.choice(ACTS)
    kind = r.choice(["linear", "linear_backward", "gated", "gated_backward"])
    what = f"{kind} M={M} N={N} K={K} {act}"
    fine = 2.0 ** -19
    if kind == "linear":
        x, w, dt = matrix(r, M, K), matrix(r, N, K, std=K ** -0.5), r.choice([BF, F32])
        bias = torch.randn(N, device=DEV) if r.random() < 0.5 else None
        res = matrix(r, M, N, dtype=dt, aligned=r.random() < 0.5) if r.random() < 0.5 else None
        keep = r.choice([None, "bf16", "bytes"])
        z = matrix(r, M, N) if keep == "bf16" else None
        q, s = eight_bits(ctx, M, N) if keep == "bytes" else (None, None)
        y = res if res is not None and r.random() < 0.3 else empty(r, M, N, dt)
        z_ref, y_ref = L.linear(np64(x), np64(w), None if bias is None else np64(bias), act, None if res is None else np64(res))
        err = (K + 2) * 2.0 ** -23 * (np.abs(np64(x)) @ np.abs(np64(w)).T) + 2.0 ** -23 * (np.abs(z_ref) + (0 if bias is None else np.abs(np64(bias))))
        size = np.abs(z_ref) + (0 if res is None else np.abs(np64(res)))
        ctx.linear(x, w, y, bias=bias, activation=act, residual=res, z=z if keep == "bf16" else q, z_scale=s)
        close(y, y_ref, step(dt) * np.abs(y_ref) + 1.2 * err + fine * size, what)
        if keep == "bf16":
            close(z, z_ref, step(BF) * np.abs(z_ref) + 1.01 * err, what + " z")
        elif keep:
            e = s.cpu().numpy().astype(np.int64) - 127
            scale = np.repeat(np.ldexp(1.0, e), 128, axis=1)[:, :N]
            assert (np.abs(values(q, s) - z_ref) <= 2.0 ** -4 * (np.abs(z_ref) + err) + 2.0 ** -10 * scale + err).all(), what
            assert (np.abs(z_ref) - err <= 448 * scale).all(), what
    elif kind == "linear_backward":
        dy, w, dt = matrix(r, M, N, std=0.1), matrix(r, N, K, std=N ** -0.5), r.choice([BF, F32])
        form = r.choice(["bf16", "bytes"] + (["none"] if act == "none" else []))
        res = matrix(r, M, K, std=0.1, dtype=dt, aligned=r.random() < 0.5) if r.random() < 0.5 else None
        z, s = (None, None) if form == "none" else (matrix(r, M, K), None) if form == "bf16" else eight_bits(ctx, M, K, matrix(r, M, K))
        z_ref = None if z is None else np64(z) if s is None else values(z, s)
        a = empty(r, M, K) if z is not None and r.random() < 0.5 else None
        dx = res if res is not None and r.random() < 0.3 else empty(r, M, K, dt)
        dx_ref, a_ref = L.linear_backward(np64(dy), np64(w), act, z_ref, None if res is None else np64(res))
        raw = np64(dy) @ np64(w)
        err = (N + 2) * 2.0 ** -23 * (np.abs(np64(dy)) @ np.abs(np64(w)))
        size = np.abs(raw) * (1 if z_ref is None else 1 + np.abs(z_ref)) + (0 if res is None else np.abs(np64(res)))
        ctx.linear_backward(dy, w, dx, activation=act, z=z, z_scale=s, a=a, residual=res)
        close(dx, dx_ref, step(dt) * np.abs(dx_ref) + 1.2 * err + fine * size, what + form)
        if a is not None:
            close(a, a_ref, step(BF) * np.abs(a_ref) + fine * np.abs(z_ref), what + form + " a")
    elif kind == "gated":
        x, wg, wu = matrix(r, M, K), matrix(r, N, K, std=K ** -0.5), matrix(r, N, K, std=K ** -0.5)
        keep = r.choice([None, "bf16", "bytes"])
        kept = {}
        if keep == "bf16":
            kept = {"gate": matrix(r, M, N), "up": matrix(r, M, N)}
        elif keep:
            (qg, sg), (qu, su) = eight_bits(ctx, M, N), eight_bits(ctx, M, N)
            kept = {"gate": qg, "gate_scale": sg, "up": qu, "up_scale": su}
        a = empty(r, M, N)
        ctx.gated_linear(x, wg, wu, a, activation=act, **kept)
        gate, up, a_ref = L.gated_linear(np64(x), np64(wg), np64(wu), act)
        eg, eu = ((K + 2) * 2.0 ** -23 * (np.abs(np64(x)) @ np.abs(np64(v)).T) for v in (wg, wu))
        close(a, a_ref, step(BF) * np.abs(a_ref) + (1.2 * eg + fine * np.abs(gate)) * (np.abs(up) + eu) + np.abs(L.act(gate, act)[0]) * eu, what + str(keep))
        for k, ref, err in (("gate", gate, eg), ("up", up, eu)):
            if keep == "bf16":
                close(kept[k], ref, step(BF) * np.abs(ref) + 1.01 * err, what + k)
            elif keep:
                scale = np.repeat(np.ldexp(1.0, kept[k + "_scale"].cpu().numpy().astype(np.int64) - 127), 128, axis=1)[:, :N]
                assert (np.abs(values(kept[k], kept[k + "_scale"]) - ref) <= 2.0 ** -4 * (np.abs(ref) + err) + 2.0 ** -10 * scale + err).all(), what + k
    else:
        dy, w = matrix(r, M, K, std=0.1), matrix(r, K, N, std=N ** -0.5)
        src = [matrix(r, M, N), matrix(r, M, N)]
        given = {}
        if r.random() < 0.5:
            both = [eight_bits(ctx, M, N, t) for t in src]
            src, given = [q for q, _ in both], {"gate_scale": both[0][1], "up_scale": both[1][1]}
            gate, up = (values(q, s) for q, s in both)
        else:
            gate, up = (np64(t) for t in src)
        over = not given and r.random() < 0.3
        dg, du = (src[0], src[1]) if over else (empty(r, M, N), empty(r, M, N))
        a = empty(r, M, N) if r.random() < 0.5 else None
        da, err = np64(dy) @ np64(w), (K + 2) * 2.0 ** -23 * (np.abs(np64(dy)) @ np.abs(np64(w)))
        dg_ref, du_ref, a_ref = L.gated_linear_backward(np64(dy), np64(w), gate, up, act)
        ctx.gated_linear_backward(dy, w, src[0], src[1], dg, du, activation=act, a=a, **given)
        f = fine * (1 + np.abs(gate))
        close(dg, dg_ref, step(BF) * np.abs(dg_ref) + np.abs(up) * (1.2 * err + f * np.abs(da)), what + " d_gate")
        close(du, du_ref, step(BF) * np.abs(du_ref) + np.abs(L.act(gate, act)[0]) * err + f * (np.abs(da) + err), what + " d_up")
        if a is not None:
            close(a, a_ref, step(BF) * np.abs(a_ref) + f * np.abs(up), what + " a")


@pytest.mark.parametrize("seed", range(30))
def test_random_logprobs(ctx, seed):
    r = random.Random(1000 + seed)
    V, dt = extent(r, 60000), r.choice([BF, F32])
    n = extent(r, max(2, 3_000_000 // V)) if r.random() < 0.7 else r.randint(1, 40)
    n = min(n, 1500)
    l = matrix(r, n, V, std=r.choice([0.1, 3.0, 20.0]), dtype=dt, aligned=r.random() < 0.4)
    if r.random() < 0.4:
        l[:, ::r.randint(2, 9)] = float("-inf")
    if r.random() < 0.3:
        l[:] = (l * 2).round() / 2                                    # many equal ones
    t = torch.tensor([r.randint(-1, V) for _ in range(n)], dtype=torch.int32, device=DEV)
    top = r.choice([0, 1, 8, 24, 25, 64])
    top = min(top, V)
    logp, ent, lse = (torch.empty(n, device=DEV) for _ in range(3))
    tv, ti = (torch.empty(n, top, device=DEV), torch.empty(n, top, dtype=torch.int32, device=DEV)) if top else (None, None)
    ctx.token_logprobs(l, t, logp, entropy=ent, lse=lse, top_values=tv, top_ids=ti)
    ref = L.logprobs(np64(l), t.cpu().numpy(), top)
    for got, want, extra in ((logp, ref[0], 0), (ent, ref[1], 2.0 ** -14), (lse, ref[2], 0)) + (((tv, ref[3], 0),) if top else ()):
        got, size = np64(got), np.abs(ref[2]) if want.ndim == 1 else np.abs(ref[2])[:, None]
        with np.errstate(invalid="ignore"):
            assert ((got == want) | (np.abs(got - want) <= 2.0 ** -18 + extra + 2.0 ** -22 * (size + np.abs(want)))).all(), (V, n, top)
    if top:
        assert (ti.cpu().numpy() == ref[4]).all(), (V, n, top)


def test_rows_behind_32_bit_offsets(ctx):
    """Outputs of more than 2^32 bytes and 2^31 numbers: their last rows are those of a call on these rows alone."""
    M, N, K = 270000, 8192, 8
    r = random.Random(1)
    x, w = matrix(r, 4096, K).repeat(66, 1)[:M].contiguous(), matrix(r, N, K)
    y = torch.empty(M, N, dtype=BF, device=DEV)
    z = torch.empty(M, N, dtype=BF, device=DEV)
    ctx.linear(x, w, y, activation="silu", z=z)
    y2, z2 = torch.empty(300, N, dtype=BF, device=DEV), torch.empty(300, N, dtype=BF, device=DEV)
    ctx.linear(x[-300:], w, y2, activation="silu", z=z2)
    assert torch.equal(y[-300:], y2) and torch.equal(z[-300:], z2)
    wd = matrix(r, K, N)
    ctx.linear_backward(x, wd, y, activation="silu", z=z, a=z)            # over the kept one
    a2 = torch.empty_like(z2)
    ctx.linear_backward(x[-300:], wd, y2, activation="silu", z=z2, a=a2)
    assert torch.equal(y[-300:], y2) and torch.equal(z[-300:], a2)
    q, s = torch.empty(M, N, dtype=torch.uint8, device=DEV), torch.empty(M, N // 128, dtype=torch.uint8, device=DEV)
    ctx.linear(x, w, y, z=q, z_scale=s)
    ctx.blockscale_dequantize(q, s, y)
    b2 = torch.empty(300, N, dtype=BF, device=DEV)
    ctx.blockscale_dequantize(q[-300:], s[-300:], b2)
    assert torch.equal(y[-300:], b2) and bool(((b2.float() - z2.float()).abs() <= 2.0 ** -3 * z2.float().abs().amax()).all())


def test_infinite_projections(ctx):
    """gelu and silu of +Inf are +Inf, in every form of the layer."""
    for M in (3, 200):
        x, w = torch.zeros(M, 8, dtype=BF, device=DEV), torch.zeros(64, 8, dtype=BF, device=DEV)
        x[:, 0], w[:, 0] = 3e38, 3e38
        for act in ("relu", "gelu", "gelu_tanh", "silu", "none"):
            y = torch.empty(M, 64, dtype=BF, device=DEV)
            ctx.linear(x, w, y, activation=act)
            assert bool((y == float("inf")).all()), act
