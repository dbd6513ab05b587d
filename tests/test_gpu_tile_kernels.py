"""The tile kernels of the linear layers that large calls launch, against the fp64 oracle: every epilogue, what is kept in both
forms, both output types.  Which kernel ran is asserted, so that another rule for the tiles cannot leave one of them untested.
Tolerances as in test_gpu_layers.py."""
import numpy as np
import pytest
import torch

import oracle.layer_oracle as L
from kernels_run import kernels_of
from paper_2508_18182_b200 import binding as A
from test_gpu_layers import bytes_for, check_bytes, close, hole, np64, rounding, rows, sum_error, untouched, widened

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
KINDS = {"linear": "0", "linear_backward": "1", "gated": "2", "gated_backward": "3"}
# sums as the tensor cores leave them, added up for what goes to 8 bits, and for fp32 outputs
PLAIN, SUMMED, SUMMED_F32 = "0", "1", "2"


@pytest.fixture(scope="module")
def ctx():
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the shapes are worked out for 148 SMs")
    c = A.Context(0)
    yield c
    assert c.device_status() == 0
    c.close()


def ran(call, kind, pair, columns, sums, in8, blocks=None):
    want = [KINDS[kind], "true" if pair else "false", str(columns), sums, "true" if in8 else "false"]
    found = kernels_of(call)
    assert [f[:2] for f in found] == [("dense_tile_kernel", want)]
    assert blocks is None or found[0][2] == blocks


# Of M x N outputs and K terms: pairs of CTAs with 256 x 256 (ragged in every direction), pairs with 256 x 128, single CTAs with 128 x 128,
# with 128 x 64 and K shared by two of them, and with 128 x 64 alone; NARROW ends in the first half of a tile
PAIRS, NARROW, HALVES, SOLO, SHARED, SINGLE = (2300, 2001, 1100), (2300, 1900, 1100), (1665, 777, 1001), (100, 9601, 1000), (300, 401, 2100), (300, 401, 200)
BLOCKS = {SHARED: 42, SINGLE: 21}


def expected(shape, dtype, to8):
    """(pair, columns) of a linear call; 256 columns are not for sums that go to 8 bits beside a bf16 output."""
    if shape in (PAIRS, NARROW):
        return (True, 128) if to8 and dtype == BF else (True, 256)
    return {HALVES: (True, 128), SOLO: (False, 128), SHARED: (False, 64), SINGLE: (False, 64)}[shape]


LINEAR = [(PAIRS, BF, "gelu", True, 0, "bf16"), (PAIRS, BF, "silu", False, 1, None), (PAIRS, F32, "gelu_tanh", True, 3, "bf16"), (PAIRS, F32, "relu", True, 0, "bytes"),
          (PAIRS, BF, "gelu", True, 0, "bytes"), (PAIRS, BF, "none", True, 8, None), (PAIRS, F32, "none", False, 1, None),
          (NARROW, F32, "gelu", True, 0, "bytes"), (NARROW, BF, "gelu", True, 0, "bytes"),
          (SHARED, BF, "gelu", True, 0, "bf16"), (SHARED, BF, "silu", True, 1, None), (SHARED, F32, "gelu_tanh", True, 0, None), (SHARED, F32, "none", False, 3, "bf16"),
          (SINGLE, BF, "gelu", True, 0, "bf16"), (SINGLE, F32, "none", True, 0, None), (HALVES, BF, "gelu", True, 1, "bf16"), (HALVES, F32, "silu", True, 0, None),
          (HALVES, F32, "silu", False, 0, "bytes"), (HALVES, BF, "none", False, 0, "bytes"), (SOLO, BF, "relu", True, 0, "bf16"), (SOLO, F32, "gelu_tanh", True, 0, "bytes"),
          (SOLO, BF, "gelu", True, 1, "bytes")]


@pytest.mark.parametrize("shape,dtype,act,use_bias,res_pad,keep", LINEAR)
def test_linear(ctx, shape, dtype, act, use_bias, res_pad, keep):
    M, N, K = shape
    x, w = rows(1, M, K), rows(2, N, K, std=K ** -0.5, pad=8)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(3)).to(DEV) if use_bias else None
    residual = rows(4, M, N, std=2.0, dtype=dtype, pad=res_pad, unit=1 if res_pad % 2 else 8)
    y, z = hole(M, N, dtype, pad=3), hole(M, N) if keep == "bf16" else None
    q, s = bytes_for(M, N) if keep == "bytes" else (None, None)
    kept = {"z": z[:M, :N]} if keep == "bf16" else {"z": q[:M, :N], "z_scale": s[:M, :-(-N // 128)]} if keep else {}
    ran(lambda: ctx.linear(x, w, y[:M, :N], bias=bias, activation=act, residual=residual, **kept), "linear", *expected(shape, dtype, keep == "bytes"),
        SUMMED_F32 if dtype == F32 else SUMMED if keep == "bytes" else PLAIN, False, BLOCKS.get(shape))
    z_ref, y_ref = L.linear(np64(x), np64(w), np64(bias) if use_bias else None, act, np64(residual))
    z_err = sum_error(x, w, K) + 2.0 ** -23 * (np.abs(z_ref) + (np.abs(np64(bias)) if use_bias else 0))
    close(y[:M, :N], y_ref, rounding(dtype) * np.abs(y_ref) + 1.2 * z_err + (2.0 ** -19 if act != "none" else 2.0 ** -23) * (np.abs(z_ref) + np.abs(np64(residual))))
    untouched(y, M, N)
    if keep == "bf16":
        close(z[:M, :N], z_ref, rounding(BF) * np.abs(z_ref) + z_err * (1 + 2.0 ** -8), "z")
        untouched(z, M, N)
    elif keep == "bytes":
        check_bytes(q, s, M, N, z_ref, z_err, "z")


BACK = [(shape, dtype, act, kept, again, res_pad)
        for shape in (PAIRS, HALVES, SOLO, SHARED)
        for dtype, act, kept, again, res_pad in ((BF, "gelu", "bf16", True, 0), (BF, "silu", "bytes", True, 1), (F32, "gelu_tanh", "bytes", True, 0), (F32, "silu", "bf16", False, 3),
                                                 (F32, "none", None, False, 0), (BF, "relu", "bytes", False, None), (BF, "none", None, False, 1))]


@pytest.mark.parametrize("shape,dtype,act,kept,again,res_pad", BACK)
def test_linear_backward(ctx, shape, dtype, act, kept, again, res_pad):
    M, K, N = shape                                          # outputs M x K, sums over N
    dy, w = rows(1, M, N, std=0.1), rows(2, N, K, std=N ** -0.5)
    residual = None if res_pad is None else rows(4, M, K, std=0.1, dtype=dtype, pad=res_pad, unit=1 if res_pad % 2 else 8)
    given, z_ref = {}, None
    if kept == "bf16":
        z = rows(20, M, K)
        given, z_ref = {"z": z}, np64(z)
    elif kept == "bytes":
        q, s = bytes_for(M, K)
        ctx.blockscale_quantize(rows(20, M, K), q[:M, :K], s[:M, :-(-K // 128)])
        given, z_ref = {"z": q[:M, :K], "z_scale": s[:M, :-(-K // 128)]}, widened(q, s, M, K)
    dx, a = hole(M, K, dtype, pad=3), hole(M, K, pad=1) if again else None
    ran(lambda: ctx.linear_backward(dy, w, dx[:M, :K], activation=act, residual=residual, a=a[:M, :K] if again else None, **given), "linear_backward",
        *expected(shape, dtype, False), SUMMED_F32 if dtype == F32 else PLAIN, kept == "bytes",
        None if shape == SHARED and dtype == F32 else BLOCKS.get(shape))      # (fp32 beside z and a leaves no room for the join)
    dx_ref, a_ref = L.linear_backward(np64(dy), np64(w), act, z_ref, None if residual is None else np64(residual))
    raw, err = np64(dy) @ np64(w), (N + 2) * 2.0 ** -23 * (np.abs(np64(dy)) @ np.abs(np64(w)))
    size = np.abs(raw) * (1 if z_ref is None else 1 + np.abs(z_ref)) + (0 if residual is None else np.abs(np64(residual)))
    close(dx[:M, :K], dx_ref, rounding(dtype) * np.abs(dx_ref) + 1.2 * err + (2.0 ** -19 if act != "none" else 2.0 ** -23) * size)
    untouched(dx, M, K)
    if again:
        close(a[:M, :K], a_ref, rounding(BF) * np.abs(a_ref) + 2.0 ** -19 * np.abs(z_ref), "a")
        untouched(a, M, K)


GATED_PAIRS, GATED_NARROW = (2300, 1100, 2001), (2300, 1100, 1940)      # M, d, f
GATED_HALVES, GATED_SINGLE = (300, 2100, 401), (100, 1280, 9601)      # the latter: more tiles than pairs of SMs


@pytest.mark.parametrize("shape,pair,columns,act,keep", [(GATED_PAIRS, True, 256, "silu", "bf16"), (GATED_PAIRS, True, 256, "gelu", None), (GATED_PAIRS, True, 256, "gelu_tanh", "bytes"),
                                                         (GATED_PAIRS, True, 256, "silu", "bytes"), (GATED_HALVES, True, 128, "silu", "bf16"), (GATED_HALVES, True, 128, "gelu", None),
                                                         (GATED_HALVES, True, 256, "silu", "bytes"), (GATED_NARROW, True, 256, "gelu", "bytes"), (GATED_SINGLE, False, 256, "gelu", "bytes"), (GATED_SINGLE, False, 128, "silu", "bf16")])
def test_gated_linear(ctx, shape, pair, columns, act, keep):
    M, d, f = shape
    x, wg, wu = rows(1, M, d), rows(2, f, d, std=d ** -0.5), rows(3, f, d, std=d ** -0.5, pad=16)
    eg, eu = sum_error(x, wg, d), sum_error(x, wu, d)
    a, kept, outs, nb = hole(M, f, pad=1), {}, [], -(-f // 128)
    if keep == "bf16":
        outs = [hole(M, f), hole(M, f, pad=8)]
        kept = {"gate": outs[0][:M, :f], "up": outs[1][:M, :f]}
    elif keep:
        outs = [bytes_for(M, f), bytes_for(M, f)]
        kept = {"gate": outs[0][0][:M, :f], "gate_scale": outs[0][1][:M, :nb], "up": outs[1][0][:M, :f], "up_scale": outs[1][1][:M, :nb]}
    ran(lambda: ctx.gated_linear(x, wg, wu, a[:M, :f], activation=act, **kept), "gated", pair, columns, SUMMED if keep == "bytes" else PLAIN, False)
    gate, up, a_ref = L.gated_linear(np64(x), np64(wg), np64(wu), act)
    h = np.abs(L.act(gate, act)[0])
    close(a[:M, :f], a_ref, rounding(BF) * np.abs(a_ref) + (1.2 * eg + 2.0 ** -19 * np.abs(gate)) * (np.abs(up) + eu) + h * eu)
    untouched(a, M, f)
    for o, ref, err in zip(outs, (gate, up), (eg, eu)):
        if keep == "bf16":
            close(o[:M, :f], ref, rounding(BF) * np.abs(ref) + err * (1 + 2.0 ** -8), "kept")
            untouched(o, M, f)
        else:
            check_bytes(*o, M, f, ref, err, "kept")


@pytest.mark.parametrize("act,form,again", [("silu", "bf16", True), ("silu", "bytes", True), ("gelu", "bytes", True), ("gelu_tanh", "bf16", False), ("gelu", "bf16", True),
                                            ("none", "bytes", False), ("relu", "bf16", True)])
@pytest.mark.parametrize("shape,pair,columns", [(GATED_PAIRS, True, 256), (GATED_HALVES, False, 64), (GATED_SINGLE, False, 128)])
def test_gated_linear_backward(ctx, shape, pair, columns, act, form, again):
    M, d, f = shape
    dy, w = rows(1, M, d, std=0.1), rows(2, d, f, std=f ** -0.5)
    err = (d + 2) * 2.0 ** -23 * (np.abs(np64(dy)) @ np.abs(np64(w)))
    da = np64(dy) @ np64(w)
    src, given = [rows(5, M, f), rows(15, M, f, pad=8)], {}
    if form == "bf16":
        gate, up = (np64(t) for t in src)
    else:
        nb, both = -(-f // 128), [bytes_for(M, f), bytes_for(M, f)]
        for t, (q, s) in zip(src, both):
            ctx.blockscale_quantize(t, q[:M, :f], s[:M, :nb])
        src = [q[:M, :f] for q, _ in both]
        given = {"gate_scale": both[0][1][:M, :nb], "up_scale": both[1][1][:M, :nb]}
        gate, up = (widened(q, s, M, f) for q, s in both)
    outs = [hole(M, f, pad=k) for k in range(3)]
    ran(lambda: ctx.gated_linear_backward(dy, w, *src, outs[0][:M, :f], outs[1][:M, :f], activation=act, a=outs[2][:M, :f] if again else None, **given),
        "gated_backward", pair, columns, PLAIN, form == "bytes")
    dg_ref, du_ref, a_ref = L.gated_linear_backward(np64(dy), np64(w), gate, up, act)
    h, fine = np.abs(L.act(gate, act)[0]), 2.0 ** -19 * (1 + np.abs(gate))
    close(outs[0][:M, :f], dg_ref, rounding(BF) * np.abs(dg_ref) + np.abs(up) * (1.2 * err + fine * np.abs(da)), "d_gate")
    close(outs[1][:M, :f], du_ref, rounding(BF) * np.abs(du_ref) + h * err + fine * (np.abs(da) + err), "d_up")
    if again:
        close(outs[2][:M, :f], a_ref, rounding(BF) * np.abs(a_ref) + fine * np.abs(up), "a")
    for o in outs[:2] + outs[2:] * again:
        untouched(o, M, f)
