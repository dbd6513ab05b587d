"""GPU parity of the linear layers in bf16 and the gated feed-forward against the fp64 oracle.

Tolerances are arithmetic.  An output is rounded once (2^-8 of its size at most in bf16, 2^-24 in fp32).  A sum of K exact
products is off by at most K 2^-23 of the sum of their magnitudes (each addition cuts off less than 2^-23 of what is added
up so far).  Activations have slopes of at most 1.13 and second derivatives of at most 1.2; their fp32 forms are off by
2^-19 of their argument's size (the fast exponential and division by 2^-21 each, a few roundings)."""
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


def rows(seed, n, d, std=1.0, pad=0, dtype=BF, unit=8):
    """[n, d] of normal numbers with rows at multiples of `unit` elements; what lies between them is NaN."""
    g = torch.Generator().manual_seed(seed)
    pitch = -(-d // unit) * unit + pad
    t = torch.full((n, pitch), float("nan"), dtype=dtype, device=DEV)
    t[:, :d] = (torch.randn(n, d, generator=g) * std).to(dtype).to(DEV)
    return t[:, :d]


def hole(n, d, dtype=BF, pad=0, unit=8):
    """An output whose surroundings are looked at afterwards."""
    return torch.full((n + 2, -(-d // unit) * unit + pad), -77.0, dtype=dtype, device=DEV)


def untouched(whole, n, d):
    assert bool((whole[n:] == -77).all()) and bool((whole[:, d:] == -77).all()), "written beyond the matrix"


def bytes_for(n, d):
    """8 bits and scales, with something else between and behind the rows."""
    q = torch.full((n + 1, -(-d // 16) * 16 + 16), 0x55, dtype=torch.uint8, device=DEV)
    s = torch.full((n + 1, -(-(-(-d // 128)) // 4) * 4 + 4), 0x55, dtype=torch.uint8, device=DEV)
    return q, s


def widened(q, s, n, d):
    v = q[:n, :d].contiguous().view(torch.float8_e4m3fn)
    return B.widen(np64(v), s[:n, :-(-d // 128)].cpu().numpy().astype(np.int64) - 127, 1)


def check_bytes(q, s, n, d, ref, err, what):
    """What 8 bits stand for: half a step of 3 bits of fraction (2^-4), or of the smallest numbers (2^-10 of the scale), from
    a value off by err; the scale is that of a largest magnitude off by err."""
    nb = -(-d // 128)
    assert bool((q[n:] == 0x55).all()) and bool((q[:, d:] == 0x55).all()), what + ": bytes beyond the matrix"
    assert bool((s[n:] == 0x55).all()) and bool((s[:, nb:] == 0x55).all()), what + ": scales beyond the matrix"
    wide = lambda x: np.pad(x, ((0, 0), (0, -d % 128))).reshape(n, nb, 128)      # noqa: E731
    low, high = np.maximum(wide(np.abs(ref) - err), 0).max(2), wide(np.abs(ref) + err).max(2)
    e = s[:n, :nb].cpu().numpy().astype(np.int64) - 127
    least, most = np.where(low > 0, B.scale_exponent(low), -127), np.where(low > 0, B.scale_exponent(high), np.maximum(B.scale_exponent(high), 0))
    assert ((e >= least) & (e <= most)).all(), what + ": scale"
    scale = np.repeat(np.ldexp(1.0, e), 128, axis=1)[:, :d]
    off = np.abs(widened(q, s, n, d) - ref)
    assert (off <= 2.0 ** -4 * (np.abs(ref) + err) + 2.0 ** -10 * scale + err).all(), (what, off.max())


def rounding(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -24


def close(got, ref, tol, what=""):
    got = np64(got)
    assert got.shape == ref.shape, what
    off = ~(np.abs(got - ref) <= tol)
    assert not off.any(), f"{what}: {off.sum()} of {off.size}, worst {np.nanmax(np.abs(got - ref) / np.maximum(tol, 1e-300)):.3g} of the tolerance"


def sum_error(x, w, K):
    """Of x w^T: K 2^-23 of the sum of magnitudes."""
    return (K + 2) * 2.0 ** -23 * (np.abs(np64(x)) @ np.abs(np64(w)).T)


# few rows; one tile and several of one CTA, whole and ragged; CTA pairs (from 74 tiles of 256 x 256), whole and ragged
# (tiles as an earlier rule chose them: by today's, of 256 x 256 there are few here; test_gpu_tile_kernels.py names the kernel of each case)
SHAPES = [(1, 1, 1), (1, 8, 8), (3, 17, 40), (8, 33, 200), (9, 130, 129), (16, 300, 2050), (17, 64, 64), (33, 1, 9), (128, 128, 64), (129, 65, 72),
          (300, 257, 200), (140, 777, 1001), (1000, 512, 768), (2560, 2048, 128), (2500, 2001, 100), (18950, 100, 72)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(ctx, M, N, K):
    x, w = rows(1, M, K), rows(2, N, K, std=K ** -0.5, pad=8)
    g = torch.Generator().manual_seed(3)
    bias = torch.randn(N, generator=g).to(DEV)
    err = sum_error(x, w, K)
    for i, (dt, act, use_bias, res_pad, keep) in enumerate([(BF, "gelu", True, None, "bf16"), (BF, "silu", False, 0, None), (F32, "none", True, 3, None),
                                                            (F32, "gelu_tanh", False, 0, "bf16"), (BF, "relu", True, 1, "bytes"), (F32, "none", False, None, "bytes")]):
        residual = None if res_pad is None else rows(4 + i, M, N, std=2.0, dtype=dt, pad=res_pad, unit=1 if res_pad % 2 else 8)
        y = hole(M, N, dt, pad=i % 3, unit=1 if i in (2, 4) else 8)
        z = hole(M, N) if keep == "bf16" else None
        q, s = bytes_for(M, N) if keep == "bytes" else (None, None)
        kept = {"z": z[:M, :N]} if keep == "bf16" else {"z": q[:M, :N], "z_scale": s[:M, :-(-N // 128)]} if keep else {}
        ctx.linear(x, w, y[:M, :N], bias=bias if use_bias else None, activation=act, residual=residual, **kept)
        z_ref, y_ref = L.linear(np64(x), np64(w), np64(bias) if use_bias else None, act, None if residual is None else np64(residual))
        z_err = err + 2.0 ** -23 * (np.abs(z_ref) + (np.abs(np64(bias)) if use_bias else 0))
        size = np.abs(z_ref) + (0 if residual is None else np.abs(np64(residual)))
        what = f"{dt} {act} {keep}"
        close(y[:M, :N], y_ref, rounding(dt) * np.abs(y_ref) + 1.2 * z_err + (2.0 ** -19 if act != "none" else 2.0 ** -23) * size, what)
        untouched(y, M, N)
        if keep == "bf16":
            close(z[:M, :N], z_ref, rounding(BF) * np.abs(z_ref) + z_err * (1 + 2.0 ** -8), what + " z")
            untouched(z, M, N)
        elif keep == "bytes":
            check_bytes(q, s, M, N, z_ref, z_err, what)


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (2, 40, 17), (16, 130, 129), (33, 9, 1), (128, 64, 128), (129, 72, 65), (300, 200, 257), (140, 1001, 777),
                                   (1000, 768, 512), (2560, 128, 2048), (2500, 100, 2001), (18950, 72, 100), (130, 700, 300)])
def test_linear_backward(ctx, M, N, K):
    dy, w = rows(1, M, N, std=0.1), rows(2, N, K, std=N ** -0.5)
    dy_w = (N + 2) * 2.0 ** -23 * (np.abs(np64(dy)) @ np.abs(np64(w)))
    raw = np64(dy) @ np64(w)
    for i, (dt, act, kept, again, res_pad) in enumerate([(BF, "gelu", "bf16", True, None), (BF, "silu", "bytes", True, 0), (F32, "none", None, False, 1),
                                                         (F32, "gelu_tanh", "bf16", True, 0), (BF, "relu", "bf16", False, 3), (BF, "none", "bytes", True, None),
                                                         (BF, "none", None, False, None)]):
        residual = None if res_pad is None else rows(4 + i, M, K, std=0.1, dtype=dt, pad=res_pad, unit=1 if res_pad % 2 else 8)
        given, z_ref = {}, None
        if kept == "bf16":
            z = rows(20 + i, M, K)
            given, z_ref = {"z": z}, np64(z)
        elif kept == "bytes":
            q, s = bytes_for(M, K)
            ctx.blockscale_quantize(rows(20 + i, M, K), q[:M, :K], s[:M, :-(-K // 128)])
            given, z_ref = {"z": q[:M, :K], "z_scale": s[:M, :-(-K // 128)]}, widened(q, s, M, K)
        dx, a = hole(M, K, dt, pad=i % 3, unit=1 if i == 2 else 8), hole(M, K, pad=i % 2) if again else None
        ctx.linear_backward(dy, w, dx[:M, :K], activation=act, residual=residual, a=a[:M, :K] if again else None, **given)
        dx_ref, a_ref = L.linear_backward(np64(dy), np64(w), act, z_ref, None if residual is None else np64(residual))
        size = np.abs(raw) * (1 if z_ref is None else 1 + np.abs(z_ref)) + (0 if residual is None else np.abs(np64(residual)))
        what = f"{dt} {act} {kept}"
        close(dx[:M, :K], dx_ref, rounding(dt) * np.abs(dx_ref) + 1.2 * dy_w + (2.0 ** -19 if act != "none" else 2.0 ** -23) * size, what)
        untouched(dx, M, K)
        if again:
            close(a[:M, :K], a_ref, rounding(BF) * np.abs(a_ref) + 2.0 ** -19 * np.abs(z_ref), what + " a")
            untouched(a, M, K)


GATED_SHAPES = [(1, 1, 1), (2, 17, 40), (9, 130, 129), (16, 200, 300), (17, 64, 64), (128, 128, 64), (129, 72, 65), (300, 200, 257), (140, 1001, 777),
                (1000, 300, 640), (4700, 64, 512), (2500, 100, 1001), (18950, 72, 100)]


@pytest.mark.parametrize("M,d,f", GATED_SHAPES)
def test_gated_linear(ctx, M, d, f):
    x, wg, wu = rows(1, M, d), rows(2, f, d, std=d ** -0.5), rows(3, f, d, std=d ** -0.5, pad=16)
    eg, eu = sum_error(x, wg, d), sum_error(x, wu, d)
    for i, (act, keep) in enumerate([("silu", "bf16"), ("gelu", None), ("gelu_tanh", "bytes"), ("relu", "bytes"), ("none", None)]):
        a = hole(M, f, pad=i % 3)
        kept, outs = {}, []
        if keep == "bf16":
            outs = [hole(M, f), hole(M, f, pad=8)]
            kept = {"gate": outs[0][:M, :f], "up": outs[1][:M, :f]}
        elif keep:
            outs = [bytes_for(M, f), bytes_for(M, f)]
            nb = -(-f // 128)
            kept = {"gate": outs[0][0][:M, :f], "gate_scale": outs[0][1][:M, :nb], "up": outs[1][0][:M, :f], "up_scale": outs[1][1][:M, :nb]}
        ctx.gated_linear(x, wg, wu, a[:M, :f], activation=act, **kept)
        gate, up, a_ref = L.gated_linear(np64(x), np64(wg), np64(wu), act)
        h = np.abs(L.act(gate, act)[0])
        close(a[:M, :f], a_ref, rounding(BF) * np.abs(a_ref) + (1.2 * eg + 2.0 ** -19 * np.abs(gate)) * (np.abs(up) + eu) + h * eu, f"{act} {keep}")
        untouched(a, M, f)
        for o, ref, err in zip(outs, (gate, up), (eg, eu)):
            if keep == "bf16":
                close(o[:M, :f], ref, rounding(BF) * np.abs(ref) + err * (1 + 2.0 ** -8), "kept")
                untouched(o, M, f)
            else:
                check_bytes(*o, M, f, ref, err, f"{act} kept")


@pytest.mark.parametrize("M,d,f", GATED_SHAPES)
def test_gated_linear_backward(ctx, M, d, f):
    dy, w = rows(1, M, d, std=0.1), rows(2, d, f, std=f ** -0.5)
    err = (d + 2) * 2.0 ** -23 * (np.abs(np64(dy)) @ np.abs(np64(w)))
    da = np64(dy) @ np64(w)
    for i, (act, form, again) in enumerate([("silu", "bf16", True), ("gelu", "bytes", True), ("gelu_tanh", "bf16", False), ("relu", "bytes", False), ("none", "bf16", True)]):
        src = [rows(5 + i, M, f), rows(15 + i, M, f, pad=8)]
        if form == "bf16":
            given, (gate, up) = {}, (np64(t) for t in src)
        else:
            nb, both = -(-f // 128), [bytes_for(M, f), bytes_for(M, f)]
            for t, (q, s) in zip(src, both):
                ctx.blockscale_quantize(t, q[:M, :f], s[:M, :nb])
            src = [q[:M, :f] for q, _ in both]
            given = {"gate_scale": both[0][1][:M, :nb], "up_scale": both[1][1][:M, :nb]}
            gate, up = (widened(q, s, M, f) for q, s in both)
        outs = [hole(M, f, pad=(i + k) % 3) for k in range(3)]
        ctx.gated_linear_backward(dy, w, *src, outs[0][:M, :f], outs[1][:M, :f], activation=act, a=outs[2][:M, :f] if again else None, **given)
        dg_ref, du_ref, a_ref = L.gated_linear_backward(np64(dy), np64(w), gate, up, act)
        h = np.abs(L.act(gate, act)[0])
        fine = 2.0 ** -19 * (1 + np.abs(gate))
        close(outs[0][:M, :f], dg_ref, rounding(BF) * np.abs(dg_ref) + np.abs(up) * (1.2 * err + fine * np.abs(da)), f"{act} {form} d_gate")
        close(outs[1][:M, :f], du_ref, rounding(BF) * np.abs(du_ref) + h * err + fine * (np.abs(da) + err), f"{act} {form} d_up")
        for o in outs[:2] + outs[2:] * again:
            untouched(o, M, f)
        if again:
            close(outs[2][:M, :f], a_ref, rounding(BF) * np.abs(a_ref) + fine * np.abs(up), f"{act} {form} a")


@pytest.mark.parametrize("n,d", [(1, 1), (3, 17), (5, 128), (9, 200), (4, 1001), (700, 768), (33, 4100)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_blockscale_dequantize(ctx, n, d, dtype):
    nb = -(-d // 128)
    q, s = bytes_for(n, d)
    ctx.blockscale_quantize(rows(d, n, d, std=30.0, dtype=F32) * torch.exp2(torch.randint(-60, 60, (1, d), device=DEV).float()), q[:n, :d], s[:n, :nb])
    for unit, pad in ((8, 0), (8, 8), (1, 0), (1, 3)):
        x = hole(n, d, dtype, pad=pad, unit=unit)
        ctx.blockscale_dequantize(q[:n, :d], s[:n, :nb], x[:n, :d])
        assert (np64(x[:n, :d]) == widened(q, s, n, d)).all()
        untouched(x, n, d)
    s[0, 0] = 255                                          # NaN for all of the block, and for nothing else
    ctx.blockscale_dequantize(q[:n, :d], s[:n, :nb], x[:n, :d])
    bad = torch.isnan(x[:n, :d])
    assert bool(bad[0, :128].all()) and int(bad.sum()) == min(d, 128)
    s[:n, :nb] = 0                                         # the smallest scale
    x32 = torch.empty(n, d, device=DEV)
    ctx.blockscale_dequantize(q[:n, :d], s[:n, :nb], x32)
    assert (np64(x32) == widened(q, s, n, d)).all()


# ------------------------------------------------------------------------------------------ values that are no numbers
def test_infinities_and_nan_stay_in_their_rows(ctx):
    for M in (5, 200, 4800):
        d, f = 72, 512
        x, wg, wu = rows(1, M, d), rows(2, f, d), rows(3, f, d)
        x[1, 3], x[M - 1, 0] = float("nan"), float("inf")
        clean = x.clone()
        clean[1], clean[M - 1] = 0, 0
        outs = []
        for v in (x, clean):
            y, a = torch.empty(M, f, dtype=BF, device=DEV), torch.empty(M, f, dtype=BF, device=DEV)
            (qg, sg), (qu, su) = bytes_for(M, f), bytes_for(M, f)
            ctx.linear(v, wg, y, activation="relu")
            ctx.gated_linear(v, wg, wu, a, gate=qg[:M, :f], gate_scale=sg[:M, :4], up=qu[:M, :f], up_scale=su[:M, :4])
            back = torch.empty(M, f, dtype=F32, device=DEV)
            ctx.blockscale_dequantize(qu[:M, :f], su[:M, :4], back)
            outs.append((y, a, back))
        for got, ref in zip(*outs):
            assert not bool(torch.isfinite(got[1]).any())
            keep = torch.ones(M, dtype=torch.bool, device=DEV)
            keep[1] = keep[M - 1] = False
            assert torch.equal(got[keep], ref[keep])
        assert bool(torch.isnan(outs[0][0][1]).all())                            # relu lets NaN through
        assert bool(torch.isnan(outs[0][2][1]).all()) and bool(torch.isnan(outs[0][2][M - 1]).all())


# ------------------------------------------------------------------------------------------ outputs over inputs
@pytest.mark.parametrize("M,N,K", [(7, 96, 64), (300, 257, 200), (2560, 2048, 72)])
def test_outputs_over_elementwise_operands(ctx, M, N, K):
    x, w = rows(1, M, K), rows(2, N, K, std=K ** -0.5)
    for dt, pad in ((BF, 0), (F32, 0), (BF, 1)):
        r = rows(3, M, N, dtype=dt, pad=pad, unit=1 if pad else 8)
        want = torch.empty(M, N, dtype=dt, device=DEV)
        ctx.linear(x, w, want, activation="gelu", residual=r)
        ctx.linear(x, w, r, activation="gelu", residual=r)
        assert torch.equal(r, want)
    z, wb = rows(4, M, N), rows(5, K, N)
    dx, a = torch.empty(M, N, dtype=BF, device=DEV), torch.empty(M, N, dtype=BF, device=DEV)
    ctx.linear_backward(x, wb, dx, activation="silu", z=z, a=a)
    z2, dx2 = z.clone(memory_format=torch.preserve_format), torch.empty_like(dx)
    z2 = rows(4, M, N)
    ctx.linear_backward(x, wb, dx2, activation="silu", z=z2, a=z2)
    assert torch.equal(dx, dx2) and torch.equal(a, z2)
    z3 = rows(4, M, N)
    ctx.linear_backward(x, wb, z3, activation="silu", z=z3)
    assert torch.equal(dx, z3)
    gate, up = rows(6, M, N), rows(7, M, N)
    outs = [torch.empty(M, N, dtype=BF, device=DEV) for _ in range(3)]
    ctx.gated_linear_backward(x, wb, gate, up, outs[0], outs[1], a=outs[2])
    a2 = torch.empty_like(outs[2])
    ctx.gated_linear_backward(x, wb, gate, up, gate, up, a=a2)
    assert torch.equal(gate, outs[0]) and torch.equal(up, outs[1]) and torch.equal(a2, outs[2])
    gate, up = rows(6, M, N), rows(7, M, N)                                       # the other way round
    ctx.gated_linear_backward(x, wb, gate, up, up, gate)
    assert torch.equal(up, outs[0]) and torch.equal(gate, outs[1])


# ------------------------------------------------------------------------------------------ streams, graphs, repetition
def test_calls_on_two_streams_and_in_a_graph(ctx):
    M, d, f = 2500, 136, 1000
    x, wg, wu, wd, dy = rows(1, M, d), rows(2, f, d, std=0.1), rows(3, f, d, std=0.1), rows(4, d, f, std=0.1), rows(5, M, d)
    wgu = torch.cat([wg, wu])

    def buffers():
        e = lambda *s: torch.empty(*s, dtype=BF, device=DEV)      # noqa: E731
        return {"a": e(M, f), "y": e(M, d), "dgu": e(M, 2 * f), "b": e(M, f), "dx": e(M, d), "q": [bytes_for(M, f), bytes_for(M, f)]}

    def step(o, stream=None):
        nb = -(-f // 128)
        (qg, sg), (qu, su) = o["q"]
        k = {"gate_scale": sg[:M, :nb], "up_scale": su[:M, :nb]}
        ctx.gated_linear(x, wg, wu, o["a"], gate=qg[:M, :f], up=qu[:M, :f], stream=stream, **k)
        ctx.linear(o["a"], wd, o["y"], residual=x, stream=stream)
        ctx.gated_linear_backward(dy, wd, qg[:M, :f], qu[:M, :f], o["dgu"][:, :f], o["dgu"][:, f:], a=o["b"], stream=stream, **k)
        ctx.linear_backward(o["dgu"], wgu, o["dx"], stream=stream)
    first = buffers()
    step(first)
    torch.cuda.synchronize()
    sets, streams = [buffers(), buffers()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for o, s in zip(sets, streams):
            step(o, s)
    torch.cuda.synchronize()
    third = buffers()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step(third)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for o in sets + [third]:
        for k in ("a", "y", "dgu", "b", "dx"):
            assert torch.equal(o[k], first[k]), k
    del graph


def test_a_wait_that_runs_out_is_reported(ctx):
    """With a limit of a nanosecond the kernels leave through their time-out; the next call is right again.  The limit is held
    against a timer that ticks every microsecond: a sum over 8192 is one that certainly takes longer."""
    for M, d, f in ((2560, 8192, 2048), (300, 8192, 300)):
        dy, w, gate, up = rows(1, M, d), rows(2, d, f, std=0.1), rows(3, M, f), rows(4, M, f)
        outs = [torch.empty(M, f, dtype=BF, device=DEV) for _ in range(4)]
        ctx.gated_linear_backward(dy, w, gate, up, outs[0], outs[1])
        ctx.set_wait_limit(1)
        try:
            ctx.gated_linear_backward(dy, w, gate, up, outs[2], outs[3])
            torch.cuda.synchronize()
        finally:
            ctx.set_wait_limit(2_000_000_000)
        assert ctx.device_status() == A.ERR_TIMEOUT
        ctx.gated_linear_backward(dy, w, gate, up, outs[2], outs[3])
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
        assert ctx.device_status() == 0


def test_long_sums_into_fp32_are_rounded_to_nearest(ctx):
    """4096 terms a sum: the tensor cores' own sums are off by 4e-6 of the result's size; added up every 512 they are
    off by less than 1e-6 (512 terms' share, 5e-7)."""
    for M in (130, 2600):
        x, w = rows(1, M, 4096), rows(2, 2048, 4096, std=2.0 ** -6)
        ref = x.double() @ w.double().t()
        y = torch.empty(M, 2048, device=DEV)
        ctx.linear(x, w, y)
        assert (y.double() - ref).norm() <= 1e-6 * ref.norm()
        wb = rows(3, 4096, 2048, std=2.0 ** -6)
        ctx.linear_backward(x, wb, y)
        ref = x.double() @ wb.double()
        assert (y.double() - ref).norm() <= 1e-6 * ref.norm()
