"""GPU parity of the operators between the linear layers against the fp64 oracle.

Tolerances come from the arithmetic: an output in bf16 is rounded once (2^-8 of its size at most), sums and products
are fp32 (a few 2^-24 of the absolute terms that enter them)."""
import numpy as np
import pytest
import torch

import oracle.block_oracle as O
from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
MASK = (0.25, (7 << 40) + 5, (3 << 33) + 11)


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def rnd(seed, *shape, dtype=F32, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).to(DEV)


def np64(t):
    return t.detach().double().cpu().numpy()


def rounding(dtype):
    return 2.0 ** -8 if dtype == BF else 2.0 ** -24


def close(got, ref, tol, what=""):
    got = np64(got)
    assert got.shape == ref.shape, what
    off = np.abs(got - ref) > tol
    assert not off.any(), f"{what}: {off.sum()} of {off.size}, worst {np.max(np.abs(got - ref) / np.maximum(tol, 1e-300)):.3g} of the tolerance"


# ---------------------------------------------------------------------------------------------- norm
# widths around every boundary of the kernels' row split (8, 256, 512, 768, 1024, 2048, 3072.. are multiples of groups)
WIDTHS = [1, 7, 8, 16, 100, 255, 256, 264, 768, 776, 1001, 1024, 1032, 2048, 2050, 4096, 4104, 8192, 16384]
TYPES = [(BF, BF), (F32, F32), (BF, F32)]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("xt,st", TYPES)
def test_add_rmsnorm(ctx, d, xt, st):
    rows = 5 if d > 2000 else 37
    x, res = rnd(d, rows, d, dtype=xt), rnd(d + 1, rows, d, dtype=st, std=3.0)
    gain = rnd(d + 2, d, dtype=F32 if d % 2 else BF)
    for residual, mask, keep in ((res, MASK, True), (res, None, False), (None, None, False)):
        h = torch.full((rows, d), -9.0, dtype=st, device=DEV) if keep else None
        y = torch.full((rows, d), -9.0, dtype=xt, device=DEV)
        rstd = torch.full((rows,), -9.0, device=DEV)
        ctx.add_rmsnorm(x, gain, residual=residual, h=h, y=y, rstd=rstd, eps=1e-6, dropout=mask)
        torch.cuda.synchronize()
        h_ref, y_ref, r_ref = O.add_rmsnorm(np64(x), np64(gain), None if residual is None else np64(residual), 1e-6, mask)
        if keep:
            close(h, h_ref, rounding(st) * np.abs(h_ref) + 2.0 ** -22 * (np.abs(np64(x)) * 2 + np.abs(np64(res))), "h")
        close(rstd, r_ref, 2.0 ** -19 * r_ref, "rstd")
        size = (np.abs(np64(x)) * 2 + (0 if residual is None else np.abs(np64(residual)))) * r_ref[:, None] * np.abs(np64(gain))
        close(y, y_ref, rounding(xt) * np.abs(y_ref) + 2.0 ** -19 * size, "y")


@pytest.mark.parametrize("B,T,d", [(1, 1, 8), (3, 5, 8), (1, 1, 1024), (2, 19, 100), (5, 33, 768), (4, 9, 1001), (2, 70, 1032), (3, 17, 2050),
                                   (2, 11, 4096), (1, 9, 8192), (2, 3, 16384), (700, 1, 64), (2, 3000, 72),
                                   (1, 5000, 776), (2, 2100, 1024), (5, 40, 128), (3, 70, 60), (9, 33, 130),
                                   # several rows of a block off the 16-byte grid, one ahead of the other where two fit
                                   (1, 7003, 1001), (2, 12011, 101), (1, 48007, 63), (2, 9001, 255), (1, 2503, 4095), (1, 4001, 2049)])
@pytest.mark.parametrize("xt,st", TYPES)
def test_add_rmsnorm_backward(ctx, B, T, d, xt, st):
    h = rnd(1, B, T, d, dtype=st, std=2.0)
    dy, dh_res = rnd(2, B, T, d, dtype=xt), rnd(3, B, T, d, dtype=st)
    gain = rnd(4, d, dtype=BF if d % 3 else F32)
    rstd = torch.rsqrt(h.float().square().mean(-1) + 1e-6)
    dh, dx = torch.full_like(h, -9.0), torch.full_like(dy, -9.0)
    n, S = torch.full((B,), 3.0, device=DEV), torch.full((d,), 5.0, device=DEV)
    args = [np64(v) for v in (dy, h, rstd, gain)]
    dh_ref, dx_ref, n_ref, S_ref = O.add_rmsnorm_backward(*args, np64(dh_res), MASK)
    hat = args[1] * args[2][..., None]
    u = np.abs(args[0] * args[3])
    size = np.abs(np64(dh_res)) + args[2][..., None] * (u + np.abs(hat) * np.mean(u * np.abs(hat), -1, keepdims=True))
    terms = np.abs(args[0] * hat)
    g, g_abs = np.sum(args[0] * hat, 1), terms.sum(1)
    eps_g = (T + 40) * 2.0 ** -23                     # at most T additions and two roundings a term
    n_tol = np.sum(2 * np.abs(g) * eps_g * g_abs + (eps_g * g_abs) ** 2, -1) + (d / 32 + 40) * 2.0 ** -23 * n_ref
    S_tol = (T + B + 80) * 2.0 ** -23 * g_abs.sum(0)
    for accumulate in (False, True):
        ctx.add_rmsnorm_backward(dy, h, rstd, gain, dh, dh_residual=dh_res, dx=dx, dropout=MASK, per_sample_sqnorm=n, grad_sum=S,
                                 accumulate_norms=accumulate, accumulate_sum=accumulate)
        torch.cuda.synchronize()
        k = 2 if accumulate else 1
        close(dh, dh_ref, rounding(st) * np.abs(dh_ref) + 2.0 ** -19 * size, "dh")
        close(dx, dx_ref, rounding(xt) * np.abs(dx_ref) + 2.0 ** -18 * size, "dx")
        close(n, k * n_ref, k * n_tol + 2.0 ** -22 * n_ref, "n")
        close(S, k * S_ref, k * S_tol + 2.0 ** -22 * np.abs(S_ref), "S")
    # without the gain's gradient, the residual's gradient and the mask; in place over dy's partner
    dh2 = torch.full_like(h, -9.0)
    ctx.add_rmsnorm_backward(dy, h, rstd, gain, dh2)
    only = torch.full((B,), -1.0, device=DEV)
    ctx.add_rmsnorm_backward(dy, h, rstd, gain, dh2, per_sample_sqnorm=only)
    torch.cuda.synchronize()
    plain = O.add_rmsnorm_backward(*args)[0]
    close(dh2, plain, rounding(st) * np.abs(plain) + 2.0 ** -19 * size, "dh alone")
    close(only, n_ref, n_tol + 2.0 ** -22 * n_ref, "norms alone")


def test_norm_gradient_is_that_of_the_forward_call_by_differences(ctx):
    """The derivative of <dy, y> + <dh_res, h> in random directions, from the forward kernel in fp32 with a step of
    2^-5: the truncation of the central difference is of order step^2 and shrinks by 4 from step 2^-4 to 2^-5, so
    the two are combined (Richardson) and what is left is of order step^4 and fp32 rounding / step."""
    B, T, d = 2, 3, 256
    x, res, dy, dh_res = (rnd(i, B, T, d).double() for i in range(4))
    gain = rnd(9, d).double()
    rstd, h = torch.empty(B, T, device=DEV), torch.empty(B, T, d, device=DEV)
    y = torch.empty_like(h)

    def loss(x, res, gain):
        ctx.add_rmsnorm(x.float(), gain.float(), residual=res.float(), h=h, y=y, rstd=rstd, eps=1e-6, dropout=MASK)
        return ((y.double() * dy).sum() + (h.double() * dh_res).sum()).item()
    loss(x, res, gain)
    dh, dx, S, n = torch.empty_like(h), torch.empty_like(h), torch.empty(d, device=DEV), torch.empty(B, device=DEV)
    ctx.add_rmsnorm_backward(dy.float(), h.clone(), rstd.clone(), gain.float(), dh, dh_residual=dh_res.float(), dx=dx, dropout=MASK,
                             per_sample_sqnorm=n, grad_sum=S)
    for seed in range(3):
        v = [rnd(50 + 3 * seed + i, *t.shape).double() for i, t in enumerate((x, res, gain))]
        slope = sum((g.double() * w).sum().item() for g, w in zip((dx, dh, S), v))

        def central(step):
            return (loss(x + step * v[0], res + step * v[1], gain + step * v[2]) - loss(x - step * v[0], res - step * v[1], gain - step * v[2])) / (2 * step)
        fine, coarse = central(2.0 ** -5), central(2.0 ** -4)
        scale = sum((g.double().abs() * w.abs()).sum().item() for g, w in zip((dx, dh, S), v))
        assert abs((4 * fine - coarse) / 3 - slope) < 2e-3 * scale / np.sqrt(3 * B * T * d) * 10


@pytest.mark.parametrize("xt,st", TYPES)
def test_norm_backward_on_pitched_and_shifted_rows_in_place(ctx, xt, st):
    """Rows that start at every offset from the 16-byte grid, each operand at its own pitch and shift; the stream's
    gradient is written over the one that comes in, dx over dy, and what lies between the rows stays as it was."""
    B, T = 3, 900
    for d, pitch, shift in ((768, 777, 3), (101, 107, 1), (510, 515, 5), (1000, 1001, 0)):
        wide = {k: rnd(i, B * T, pitch + i, dtype=t) for i, (k, t) in enumerate((("dy", xt), ("h", st), ("res", st)))}
        dy, h, res = (wide[k][:, shift:shift + d].unflatten(0, (B, T)) for k in ("dy", "h", "res"))
        gain = rnd(9, d)
        rstd = torch.rsqrt(h.float().square().mean(-1) + 1e-6)
        args = [np64(v) for v in (dy, h, rstd, gain)]
        dh_ref, dx_ref, n_ref, S_ref = O.add_rmsnorm_backward(*args, np64(res), MASK)
        u, hat = np.abs(args[0] * args[3]), args[1] * args[2][..., None]
        size = np.abs(np64(res)) + args[2][..., None] * (u + np.abs(hat) * np.mean(u * np.abs(hat), -1, keepdims=True))
        before = {k: v.clone() for k, v in wide.items()}
        S = torch.empty(d, device=DEV)
        ctx.add_rmsnorm_backward(dy, h, rstd, gain, res, dh_residual=res, dx=dy, dropout=MASK, grad_sum=S)
        torch.cuda.synchronize()
        close(res, dh_ref, rounding(st) * np.abs(dh_ref) + 2.0 ** -19 * size, "dh")
        close(dy, dx_ref, rounding(xt) * np.abs(dx_ref) + 2.0 ** -18 * size, "dx")
        close(S, S_ref, (T + B + 80) * 2.0 ** -23 * np.abs(args[0] * hat).sum((0, 1)) + 2.0 ** -22 * np.abs(S_ref), "S")
        assert torch.equal(wide["h"], before["h"])
        for k in ("dy", "res"):
            assert torch.equal(wide[k][:, :shift], before[k][:, :shift]) and torch.equal(wide[k][:, shift + d:], before[k][:, shift + d:])


def test_norm_on_pitched_and_shifted_rows_in_place_and_on_another_stream(ctx):
    side = torch.cuda.Stream()
    for d, pitch, shift in ((768, 1000, 8), (768, 1001, 3), (100, 104, 1)):
        wide_x, wide_r = rnd(1, 20, pitch + 16, dtype=BF), rnd(2, 20, pitch + 16, dtype=F32)
        x, res = wide_x[:, shift:shift + d], wide_r[:, shift:shift + d]
        gain = rnd(3, d)
        y_wide = torch.full((20, pitch), 7.0, dtype=BF, device=DEV)
        h_ref, y_ref, r_ref = O.add_rmsnorm(np64(x), np64(gain), np64(res))
        before = wide_r.clone()
        torch.cuda.synchronize()
        ctx.add_rmsnorm(x, gain, residual=res, h=res, y=y_wide[:, :d], stream=side)      # h over the residual itself
        side.synchronize()
        close(res, h_ref, 2.0 ** -22 * (np.abs(np64(x)) + np.abs(h_ref) + 1), "h in place")
        close(y_wide[:, :d], y_ref, 2.0 ** -8 * np.abs(y_ref) + 2.0 ** -17, "y")
        assert (y_wide[:, d:] == 7).all()
        before[:, shift:shift + d] = res
        assert torch.equal(before, wide_r)                                                # nothing beside the rows
        dy, dh = rnd(4, 20, d, dtype=BF), res.clone()
        rs = torch.tensor(r_ref, dtype=F32, device=DEV)
        g_ref = O.add_rmsnorm_backward(np64(dy)[None], np64(dh)[None], np64(rs)[None], np64(gain), np64(x)[None])[0][0]
        run = x.float().clone()
        torch.cuda.synchronize()
        ctx.add_rmsnorm_backward(dy, dh, rs, gain, run, dh_residual=run, stream=side)     # the stream's gradient in place
        side.synchronize()
        close(run, g_ref, 2.0 ** -17 * (1 + np.abs(g_ref)), "dh in place")


def test_norm_of_zero_infinite_and_nan_rows(ctx):
    d = 300
    x = rnd(1, 6, d, dtype=BF)
    x[0] = 0
    x[1, 7] = float("inf")
    x[2, 299] = float("nan")
    x[3] = 1e-30
    x[4] = 3e18                                                   # squares near the top of fp32: their sum must not overflow a row beside
    gain = torch.ones(d, device=DEV)
    y, r = torch.empty_like(x), torch.empty(6, device=DEV)
    q, s = torch.zeros(6, 304, dtype=torch.uint8, device=DEV)[:, :d], torch.zeros(6, 4, dtype=torch.uint8, device=DEV)[:, :3]
    ctx.add_rmsnorm(x, gain, y=y, rstd=r, q=q, q_scale=s, eps=1e-6)
    torch.cuda.synchronize()
    assert (y[0] == 0).all() and (s[0] == 127).all() and (q[0] == 0).all()
    assert r[1] == 0 and torch.isnan(y[1, 7]) and (y[1, :7] == 0).all()
    assert s[1].tolist()[0] == 255 and s[1].tolist()[1:] == [127, 127]
    assert torch.isnan(y[2]).all() and (s[2] == 255).all()
    assert torch.allclose(y[3].float(), torch.full((d,), 1e-27, device=DEV), rtol=2.0 ** -7)
    assert torch.allclose(y[4].float(), torch.ones(d, device=DEV), rtol=2.0 ** -7)
    _, y_ref, _ = O.add_rmsnorm(np64(x[5]), np.ones(d), None, 1e-6)
    close(y[5], y_ref, 2.0 ** -8 * np.abs(y_ref) + 2.0 ** -19, "the row beside them")


# ------------------------------------------------------------------------------------------- dropout
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 5), (4, 8), (7, 24), (9, 100), (1, 100003), (301, 768), (64, 1001)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_dropout(ctx, shape, dtype):
    x, r = rnd(1, *shape, dtype=dtype), rnd(2, *shape, dtype=dtype)
    for p in (0.0, 0.1, 0.5, 1.0):
        for residual in (None, r):
            out = torch.full(shape, -9.0, dtype=dtype, device=DEV)
            ctx.dropout(x, out, p=p, seed=MASK[1], offset=MASK[2], residual=residual)
            torch.cuda.synchronize()
            ref = O.drop(np64(x), (p, MASK[1], MASK[2])) + (0 if residual is None else np64(r))
            if residual is None:
                assert np.array_equal(np64(out) == 0, (ref == 0) | (np64(x) == 0))
            close(out, ref, rounding(dtype) * np.abs(ref) + 2.0 ** -23 * (np.abs(np64(x)) * 2 + np.abs(np64(r))), f"p={p}")


def test_dropout_is_its_own_gradient_and_drops_nan_and_takes_pitched_rows(ctx):
    for cols, pitch, shift in ((100, 117, 3), (96, 104, 8), (96, 97, 0)):
        wide = rnd(1, 33, pitch + 8, dtype=BF)
        x = wide[:, shift:shift + cols]
        mask = O.keep_mask(33 * cols, *MASK).reshape(33, cols)
        x[torch.tensor(~mask, device=DEV)] = float("nan")             # only what is dropped
        out = torch.full((33, pitch), 7.0, dtype=BF, device=DEV)
        ctx.dropout(x, out[:, :cols], p=MASK[0], seed=MASK[1], offset=MASK[2])
        torch.cuda.synchronize()
        ref = O.drop(np.where(mask, np64(x), 0), MASK)
        close(out[:, :cols], ref, 2.0 ** -8 * np.abs(ref), "pitched")
        assert (out[:, cols:] == 7).all()
    # in place; the same mask as inside the norm's call
    x = rnd(5, 40, 264)
    y, h = torch.empty_like(x), torch.empty_like(x)
    ctx.add_rmsnorm(x, torch.ones(264, device=DEV), h=h, y=y, dropout=MASK)
    ctx.dropout(x, x, p=MASK[0], seed=MASK[1], offset=MASK[2])
    torch.cuda.synchronize()
    assert torch.equal(x, h)


# --------------------------------------------------------------------------------------------- rope
@pytest.mark.parametrize("D,R", [(64, 64), (64, 32), (80, 20), (96, 96), (128, 64), (6, 2), (5, 4), (256, 256), (36, 36)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope(ctx, D, R, interleaved, dtype):
    t = A.RopeTable(R, scaling="by_parts", factor=8.0, context=512, low=1.0, high=16.0, magnitude=1.2)
    w = O.rope_frequencies(R, 1e4, "by_parts", 8.0, 512, 1.0, 16.0)
    for B, T, Hq, Hk in ((1, 1, 1, 1), (3, 1, 8, 2), (2, 33, 3, 1)):
        qkv = rnd(D + B, B, T, Hq + 2 * Hk, D, dtype=dtype)
        q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hk]
        pos = torch.randint(0, 1 << 20, (B, T), generator=torch.Generator().manual_seed(3), dtype=torch.int32).to(DEV)
        for inverse in (False, True):
            oq = torch.full((B, Hq, T, D), -9.0, dtype=dtype, device=DEV).transpose(1, 2)      # heads outside tokens
            ok = torch.full((B, T, Hk, D), -9.0, dtype=dtype, device=DEV)
            ctx.rope([q, k], t, outs=[oq, ok], positions=pos, interleaved=interleaved, inverse=inverse)
            torch.cuda.synchronize()
            for x, o in ((q, oq), (k, ok)):
                ref = O.rope(np64(x), pos.cpu().numpy(), w, t.magnitude, interleaved, inverse)
                pair = np.abs(np64(x)).max(-1, keepdims=True) * 2
                # an angle off by 2^-24 of a turn and by the sine's two units in the last place
                tol = rounding(dtype) * np.abs(ref) + 2.0 ** -20 * 1.2 * pair
                tol[..., R:] = 0
                close(o, ref, tol, "rope")
    # in place, positions counted from a first one; the inverse brings the input back up to rounding and magnitude^2
    x = rnd(1, 2, 9, 4, D, dtype=dtype)
    y = x.clone()
    ctx.rope([y], t, first_position=-3, interleaved=interleaved)
    torch.cuda.synchronize()
    ref = O.rope(np64(x), np.arange(-3, 6)[None].repeat(2, 0), w, t.magnitude, interleaved)
    close(y, ref, rounding(dtype) * np.abs(ref) + 2.0 ** -20 * 4 * np.abs(np64(x)).max(), "in place")
    assert torch.equal(y[..., R:], x[..., R:])


def test_rope_at_positions_that_pass_2_to_31_turns(ctx):
    """Phases are exact whole numbers: far positions are as good as near ones."""
    t = A.RopeTable(64, base=10000.0)
    x = rnd(1, 1, 4, 2, 64)
    o = torch.empty_like(x)
    first = (1 << 40) + 12345
    ctx.rope([x], t, outs=[o], first_position=first)
    torch.cuda.synchronize()
    turns = t.turns_host.numpy().view(np.uint64)
    angle = np.array([[((first + i) * int(u) % (1 << 64)) / 2.0 ** 64 * 2 * np.pi for u in turns] for i in range(4)])
    a, b = np64(x)[0, :, :, :32], np64(x)[0, :, :, 32:]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    ref = np.concatenate([a * c - b * s, a * s + b * c], -1)[None]
    close(o, ref, 2.0 ** -20 * 2 * np.abs(np64(x)).max(), "far positions")


# -------------------------------------------------------------------------------------------- 8 bits
def pitched(rows, cols, unit, dtype=torch.uint8):
    return torch.zeros(rows, (cols + unit - 1) // unit * unit + unit, dtype=dtype, device=DEV)[:, :cols]


def values(q):
    return q.view(torch.float8_e4m3fn).double().cpu().numpy() if q.is_contiguous() else q.contiguous().view(torch.float8_e4m3fn).double().cpu().numpy()


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (5, 768), (33, 1000), (2, 2049), (100, 136)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantise_rows_exactly(ctx, rows, cols, dtype):
    x = (rnd(1, rows, cols) * torch.exp(rnd(2, rows, cols) * 3)).to(dtype)
    x[0, 0] = 0
    if cols > 130:
        x[-1, 128:] = 0                                    # a block of zeros
    q, s = pitched(rows, cols, 16), pitched(rows, (cols + 127) // 128, 4)
    ctx.blockscale_quantize(x, q, s)
    torch.cuda.synchronize()
    v, e = O.quantise(np64(x), 1)
    assert np.array_equal(s.cpu().numpy(), e + 127) and np.array_equal(values(q), v)


def test_quantise_extremes(ctx):
    x = torch.zeros(8, 128, device=DEV)
    x[0, 3], x[1, 3], x[2, 3] = 448.0, 448.00003, 3.4e38
    x[3, 3], x[4, 3] = 1e-45, 2.0 ** -120
    x[5, 3], x[6, 3], x[7, 3] = float("inf"), float("-inf"), float("nan")
    x[:, 4] = 1e-3
    q, s = pitched(8, 128, 16), pitched(8, 1, 4)
    ctx.blockscale_quantize(x, q, s)
    torch.cuda.synchronize()
    v, e = O.quantise(np64(x[:5]), 1)
    assert np.array_equal(s[:5].cpu().numpy(), e + 127) and np.array_equal(values(q[:5]), v)
    assert (s[5:] == 255).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (128, 128), (130, 257), (768, 100), (33, 1000), (257, 512)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantise_weights_exactly(ctx, rows, cols, dtype):
    W = (rnd(1, rows, cols) * torch.exp(rnd(2, rows, cols) * 2)).to(dtype)
    q, qt = pitched(rows, cols, 16), pitched(cols, rows, 16)
    s = torch.zeros((rows + 127) // 128, (cols + 127) // 128, dtype=torch.uint8, device=DEV)
    ctx.blockscale_quantize_weight(W, q, s, q_t=qt)
    torch.cuda.synchronize()
    v, e = O.quantise(np64(W), 128)
    assert np.array_equal(s.cpu().numpy(), e + 127) and np.array_equal(values(q), v) and np.array_equal(values(qt), v.T)


@pytest.mark.parametrize("d", [1, 60, 64, 128, 100, 136, 768, 1000, 1001, 2048, 4104])
def test_norm_to_8_bits(ctx, d):
    x, res, gain = rnd(1, 9, d, dtype=BF), rnd(2, 9, d, dtype=BF, std=2.0), torch.exp(rnd(3, d))
    q, s = pitched(9, d, 16), pitched(9, (d + 127) // 128, 4)
    ctx.add_rmsnorm(x, gain, residual=res, q=q, q_scale=s, eps=1e-6)
    torch.cuda.synchronize()
    _, y, _ = O.add_rmsnorm(np64(x), np64(gain), np64(res), 1e-6)
    e = s.cpu().numpy().astype(int) - 127
    amax = np.abs(np.pad(y, ((0, 0), (0, -d % 128))).reshape(9, -1, 128)).max(-1)
    near = 1e-5 * amax                                      # fp32 and 64 bits may disagree on which side of a power of two a block is
    assert np.all((e >= O.scale_exponent(amax - near)) & (e <= O.scale_exponent(amax + near)))
    step = np.repeat(2.0 ** e, 128, 1)[:, :d]
    got = O.widen(values(q), e, 1)
    assert np.all(np.abs(got - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * step + 1e-5 * np.abs(y))


MATMULS = [(1, 1, 1), (1, 128, 128), (3, 5, 7), (2, 200, 33), (5, 2048, 640), (8, 300, 1100), (9, 256, 128), (17, 1000, 520), (64, 512, 2048),
           (100, 96, 4096), (128, 128, 512), (129, 257, 130), (257, 384, 768), (300, 1001, 1000), (512, 768, 2304), (1000, 2304, 768), (4, 4096, 16),
           (2600, 2304, 768), (5003, 1000, 1100), (2305, 2050, 130), (20000, 129, 640)]


@pytest.mark.parametrize("M,N,K", MATMULS)
@pytest.mark.parametrize("transposed", [False, True])
def test_blockscale_matmul(ctx, M, N, K, transposed):
    """Against 64 bits on the same 8-bit numbers.  The tensor cores add K in steps of 32; a step may lose up to
    2^-21 of the absolute terms so far."""
    x = rnd(1, M, K) * torch.exp(rnd(2, M, K))
    W = rnd(3, N, K) * torch.exp(rnd(4, N, K))
    a, sa = pitched(M, K, 16), pitched(M, (K + 127) // 128, 4)
    ctx.blockscale_quantize(x, a, sa)
    w = W.t().contiguous() if transposed else W
    b, bt = pitched(*w.shape, 16), pitched(w.shape[1], w.shape[0], 16)
    sb = torch.zeros((w.shape[0] + 127) // 128, (w.shape[1] + 127) // 128, dtype=torch.uint8, device=DEV)
    ctx.blockscale_quantize_weight(w, b, sb, q_t=bt)
    bias = rnd(5, N) if M % 2 else None
    torch.cuda.synchronize()
    av = O.widen(values(a), sa.cpu().numpy().astype(int) - 127, 1)
    bv = O.widen(values(b), sb.cpu().numpy().astype(int) - 127, 128)
    bv = bv.T if transposed else bv
    ref = av @ bv.T + (0 if bias is None else np64(bias))
    size = np.abs(av) @ np.abs(bv).T
    for dtype in (F32, BF):
        for pad in (0, 8, 3):
            wide = torch.full((M, N + pad), 7.0, dtype=dtype, device=DEV)
            ctx.blockscale_matmul(a, sa, bt if transposed else b, sb, wide[:, :N], scale_transposed=transposed, bias=bias)
            torch.cuda.synchronize()
            assert ctx.device_status() == 0
            close(wide[:, :N], ref, rounding(dtype) * np.abs(ref) + (K / 32 + 8) * 2.0 ** -21 * size + 2.0 ** -23 * np.abs(ref), f"{dtype} pitch {N + pad}")
            assert (wide[:, N:] == 7).all()


@pytest.mark.parametrize("M,N,K", [(1, 64, 256), (7, 130, 384), (150, 140, 300), (700, 520, 1024)])
def test_matmul_of_whole_numbers_is_exact(ctx, M, N, K):
    """Small whole numbers under scales of 1: every sum fits fp32, nothing may be lost."""
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-8, 9, (M, K), generator=g).float().to(DEV)
    w = torch.randint(-8, 9, (N, K), generator=g).float().to(DEV)
    a, b = pitched(M, K, 16), pitched(N, K, 16)
    a.copy_(x.to(torch.float8_e4m3fn).view(torch.uint8))
    b.copy_(w.to(torch.float8_e4m3fn).view(torch.uint8))
    sa = pitched(M, (K + 127) // 128, 4)
    sa.copy_(127 + torch.arange(M, device=DEV)[:, None] % 3)
    sb = (127 + torch.arange((N + 127) // 128, device=DEV)[:, None] - torch.arange((K + 127) // 128, device=DEV)).to(torch.uint8)
    out = torch.empty(M, N, device=DEV)
    ctx.blockscale_matmul(a, sa, b, sb, out)
    torch.cuda.synchronize()
    ref = O.widen(np64(x), sa.cpu().numpy().astype(int) - 127, 1) @ O.widen(np64(w), sb.cpu().numpy().astype(int) - 127, 128).T
    assert np.array_equal(np64(out), ref)


@pytest.mark.parametrize("M,N,K", [(1, 40, 1), (5, 130, 129), (200, 300, 1001), (2600, 2304, 135), (3, 64, 2060)])
def test_what_lies_between_the_rows_is_not_looked_at(ctx, M, N, K):
    """The bytes between a row's end and the next row, and the scale bytes there, may hold anything (NaN here)."""
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-8, 9, (M, K), generator=g).float().to(DEV)
    w = torch.randint(-8, 9, (N, K), generator=g).float().to(DEV)
    kb = (K + 127) // 128
    full = [torch.full((r, (c + 15) // 16 * 16 + 16), 0x7F, dtype=torch.uint8, device=DEV) for r, c in ((M, K), (N, K))]
    a, b = full[0][:, :K], full[1][:, :K]
    a.copy_(x.to(torch.float8_e4m3fn).view(torch.uint8))
    b.copy_(w.to(torch.float8_e4m3fn).view(torch.uint8))
    sa = torch.full((M, (kb + 3) // 4 * 4 + 4), 255, dtype=torch.uint8, device=DEV)[:, :kb]
    sa.fill_(127)
    sb = torch.full(((N + 127) // 128, kb + 3), 255, dtype=torch.uint8, device=DEV)[:, :kb]
    sb.fill_(127)
    out = torch.empty(M, N, device=DEV)
    ctx.blockscale_matmul(a, sa, b, sb, out)
    torch.cuda.synchronize()
    assert np.array_equal(np64(out), np64(x) @ np64(w).T)


@pytest.mark.parametrize("M", [2, 40, 300])
def test_matmul_propagates_nan_blocks_only_where_they_are(ctx, M):
    N, K = 256, 384
    x, W = rnd(1, M, K, dtype=BF), rnd(2, N, K)
    x[1, 200] = float("inf")
    a, sa, b = pitched(M, K, 16), pitched(M, 3, 4), pitched(N, K, 16)
    sb = torch.zeros(2, 3, dtype=torch.uint8, device=DEV)
    ctx.blockscale_quantize(x, a, sa)
    ctx.blockscale_quantize_weight(W, b, sb)
    out = torch.zeros(M, N, device=DEV)
    ctx.blockscale_matmul(a, sa, b, sb, out)
    torch.cuda.synchronize()
    assert torch.isnan(out[1]).all() and torch.isfinite(out[torch.arange(M, device=DEV) != 1]).all()


@pytest.mark.parametrize("M,N,K", [(300, 256, 16384), (2600, 2304, 16384)])      # waits enough that the clock moves in one of them
def test_matmul_wait_that_runs_out_is_reported_and_the_context_stays_usable(ctx, M, N, K):
    x, W = rnd(1, M, K, dtype=BF), rnd(2, N, K)
    a, sa, b = pitched(M, K, 16), pitched(M, K // 128, 4), pitched(N, K, 16)
    sb = torch.zeros(N // 128, K // 128, dtype=torch.uint8, device=DEV)
    ctx.blockscale_quantize(x, a, sa)
    ctx.blockscale_quantize_weight(W, b, sb)
    out, again = torch.zeros(M, N, device=DEV), torch.zeros(M, N, device=DEV)
    ctx.blockscale_matmul(a, sa, b, sb, out)
    ctx.set_wait_limit(1)
    ctx.blockscale_matmul(a, sa, b, sb, again)
    assert ctx.device_status() == A.ERR_TIMEOUT
    ctx.set_wait_limit(2_000_000_000)
    ctx.blockscale_matmul(a, sa, b, sb, again)
    assert ctx.device_status() == 0 and torch.equal(out, again)


# ------------------------------------------------------------------------------------------ refusals
def test_refusals_launch_nothing(ctx):
    x, g = rnd(1, 4, 64, dtype=BF), rnd(2, 64)
    y, r = torch.empty_like(x), torch.empty(4, device=DEV)
    t = A.RopeTable(32)
    heads = rnd(3, 1, 4, 2, 64, dtype=BF)
    q, s = pitched(4, 64, 16), pitched(4, 1, 4)
    b, sb = pitched(8, 64, 16), torch.zeros(1, 1, dtype=torch.uint8, device=DEV)
    out = torch.empty(4, 8, device=DEV)
    before = ctx.launch_count
    I, U, L, W = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED, A.ERR_ALIGNMENT, A.ERR_WORKSPACE
    odd = torch.zeros(4, 72, dtype=torch.uint8, device=DEV)
    cases = [
        (I, lambda: ctx.add_rmsnorm(x, g)),                                                        # no output
        (I, lambda: ctx.add_rmsnorm(x, g[:60], y=y)),
        (I, lambda: ctx.add_rmsnorm(x.t(), g, y=y)),
        (I, lambda: ctx.add_rmsnorm(x, g, y=y, eps=-1.0)),
        (I, lambda: ctx.add_rmsnorm(x, g, y=y, eps=float("nan"))),
        (I, lambda: ctx.add_rmsnorm(x, g, y=y, dropout=(1.5, 0, 0))),
        (I, lambda: ctx.add_rmsnorm(x, g, y=y, dropout=(float("nan"), 0, 0))),
        (I, lambda: ctx.add_rmsnorm(x, g, y=y, dropout=(0.5, -1, 0))),
        (I, lambda: ctx.add_rmsnorm(x, g, y=y, q=q)),
        (I, lambda: ctx.add_rmsnorm(x[:0], g, y=y[:0])),
        (U, lambda: ctx.add_rmsnorm(x.half(), g, y=y.half())),
        (U, lambda: ctx.add_rmsnorm(x.float(), g, residual=x, y=y.float())),                       # F32 onto a BF16 stream
        (U, lambda: ctx.add_rmsnorm(torch.zeros(1, 16392, device=DEV), torch.zeros(16392, device=DEV), y=torch.zeros(1, 16392, device=DEV))),
        (L, lambda: ctx.add_rmsnorm(x, g, q=odd[:, :64], q_scale=s)),
        (I, lambda: ctx.add_rmsnorm_backward(x, x, r[:3], g, y)),
        (W, lambda: ctx.add_rmsnorm_backward(x, x, r, g, y, grad_sum=torch.empty(64, device=DEV), workspace=torch.empty(16, dtype=torch.uint8, device=DEV))),
        (I, lambda: ctx.dropout(x, y, p=-0.1, seed=0)),
        (I, lambda: ctx.dropout(x, y[:3], p=0.1, seed=0)),
        (U, lambda: ctx.dropout(x.double(), y.double(), p=0.1, seed=0)),
        (I, lambda: ctx.rope([heads], A.RopeTable(128))),                                          # wider than a head
        (I, lambda: ctx.rope([heads[0]], t)),
        (I, lambda: ctx.rope([heads], t, positions=torch.zeros(1, 3, dtype=torch.int32, device=DEV))),
        (I, lambda: ctx.rope([heads], t, positions=torch.zeros(1, 4, dtype=torch.int64, device=DEV))),
        (I, lambda: ctx.rope([heads], t, outs=[heads[:, :, :1].expand(1, 4, 2, 64)])),             # outputs fall on one another
        (U, lambda: ctx.rope([heads] * 5, t)),
        (U, lambda: ctx.rope([heads.half()], t)),
        (L, lambda: ctx.blockscale_quantize(x, odd[:, :64], s)),
        (L, lambda: ctx.blockscale_quantize(x, q, torch.zeros(4, 5, dtype=torch.uint8, device=DEV)[:, :1])),
        (I, lambda: ctx.blockscale_quantize(x, q, torch.zeros(4, 2, dtype=torch.uint8, device=DEV))),
        (U, lambda: ctx.blockscale_quantize(x.half(), q, s)),
        (I, lambda: ctx.blockscale_matmul(q, s, b[:, :32], sb, out)),
        (I, lambda: ctx.blockscale_matmul(q, s, b, sb, out[:, :7])),
        (I, lambda: ctx.blockscale_matmul(q, s, b, sb.expand(2, 1), out)),
        (U, lambda: ctx.blockscale_matmul(q, s, b, sb, out.half())),
        (L, lambda: ctx.blockscale_matmul(q, s, torch.zeros(8, 72, dtype=torch.uint8, device=DEV)[:, :64], sb, out)),
        (I, lambda: ctx.dropout(x.cpu(), y, p=0.1, seed=0)),
    ]
    for k, (status, call) in enumerate(cases):
        with pytest.raises(A.AdlocoError) as e:
            call()
        assert e.value.status == status, (k, e.value)
    assert ctx.launch_count == before


def test_null_pointers_and_empty_sizes_are_argument_errors(ctx):
    import ctypes as C
    lib, h = ctx.lib, ctx.h
    before = ctx.launch_count
    buf = C.c_void_p(torch.zeros(1024, device=DEV).data_ptr())
    zeros = C.create_string_buffer(256)          # an argument struct of nothing
    assert lib.adloco_add_rmsnorm(h, None, None) == A.ERR_INVALID_ARG and lib.adloco_add_rmsnorm(h, zeros, None) == A.ERR_INVALID_ARG
    assert lib.adloco_add_rmsnorm_backward(h, zeros, None) == A.ERR_INVALID_ARG
    assert lib.adloco_blockscale_matmul(h, zeros, None) == A.ERR_INVALID_ARG
    assert lib.adloco_dropout(None, 0, 1, 1, buf, 1, None, 0, buf, 1, 0.5, 0, 0, None) == A.ERR_INVALID_ARG
    assert lib.adloco_dropout(h, 0, 0, 1, buf, 1, None, 0, buf, 1, 0.5, 0, 0, None) == A.ERR_INVALID_ARG
    assert lib.adloco_rope(h, 0, None, 1, 1, 1, 8, 8, buf, 1.0, None, 0, 0, 0, 0, None) == A.ERR_INVALID_ARG
    assert lib.adloco_blockscale_quantize(h, 0, 1, 0, buf, 0, buf, 16, buf, 4, None) == A.ERR_INVALID_ARG
    assert lib.adloco_blockscale_quantize_weight(h, 0, 1, 1, None, 1, buf, 16, None, 0, buf, 4, None) == A.ERR_INVALID_ARG
    assert lib.adloco_add_rmsnorm_backward_workspace(None, 1, 1, 1) == 0
    assert ctx.launch_count == before
