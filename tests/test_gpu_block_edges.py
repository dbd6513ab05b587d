"""GPU tests of the operators between the linear layers at the places where they could go wrong: what only few shapes,
types or callers reach.  Oracle and tolerances as in test_gpu_block_ops.py; whole numbers small enough that every sum
fits fp32 are compared for equality."""
import threading
import time

import numpy as np
import pytest
import torch

import oracle.block_oracle as O
import test_gpu_block_ops as parity
from paper_2508_18182_b200 import binding as A
from test_gpu_block_ops import BF, DEV, F32, MASK, TYPES, close, np64, pitched, rnd, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def whole(seed, *shape, share=1.0, top=1, dtype=F32):
    """Whole numbers of -top .. top, `share` of them kept."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(-top, top + 1, shape, generator=g).float()
    return (x * (torch.rand(shape, generator=g) < share)).to(dtype).to(DEV)


# ------------------------------------------------------------------------------- norm, the gain's gradient
@pytest.mark.parametrize("d", [224, 256, 229, 776])
def test_norms_of_one_long_sample_with_more_blocks_than_columns(ctx, d):
    """One sample of many chunks: its norm is added up by a cluster of eight blocks of 128 columns, some without any.
    dy and h are small whole numbers under rstd = 1, so the gain's gradient and its squared norm are exact."""
    T = 592 * 16
    dy, h = whole(1, 1, T, d, share=0.01), whole(2, 1, T, d)
    g = (np64(dy) * np64(h)).sum(1)
    n_ref = np.sum(g * g)
    assert n_ref < 2 ** 24
    rstd, gain, dh = torch.ones(1, T, device=DEV), torch.ones(d, device=DEV), torch.empty_like(h)
    n, S = torch.zeros(40, 1, device=DEV), torch.zeros(40, d, device=DEV)
    for i in range(40):
        ctx.add_rmsnorm_backward(dy, h, rstd, gain, dh, per_sample_sqnorm=n[i], grad_sum=S[i] if i % 2 else None)
    torch.cuda.synchronize()
    assert (np64(n) == n_ref).all() and (np64(S[1::2]) == g).all()


# ------------------------------------------------------------------------------------ launches that overlap
@pytest.mark.parametrize("M,N,K", [(1, 2048, 1024), (12, 512, 2048), (40, 300, 512), (2600, 2304, 256)])
def test_every_operand_may_be_written_by_the_call_before(ctx, M, N, K):
    """Operands are overwritten in place between products, nothing waits: each product has the values of its turn."""
    x, w = [whole(i, M, K, top=8) for i in range(4)], [whole(9 + i, N, K, top=8) for i in range(4)]
    a, sa, b, sb = pitched(M, K, 16), pitched(M, K // 128, 4), pitched(N, K, 16), torch.zeros(-(-N // 128), K // 128, dtype=torch.uint8, device=DEV)
    bias, zero, out = torch.zeros(1, N, device=DEV), [whole(20 + i, 1, N, top=8) for i in range(4)], torch.zeros(24, M, N, device=DEV)
    torch.cuda.synchronize()
    for i in range(24):
        ctx.blockscale_quantize_weight(w[i % 3], b, sb)
        ctx.blockscale_quantize(x[i % 4], a, sa)
        ctx.dropout(zero[i // 6], bias, p=0.0, seed=0)
        ctx.blockscale_matmul(a, sa, b, sb, out[i], bias=bias[0])
    torch.cuda.synchronize()
    for i in range(24):
        ref = x[i % 4].double() @ w[i % 3].double().t() + zero[i // 6].double()
        assert torch.equal(out[i].double(), ref), i


def test_gain_and_turns_may_be_written_by_the_call_before(ctx):
    x, gains = whole(1, 64, 256, top=3), [whole(2 + i, 1, 256, top=5) for i in range(3)]
    gain, out, ones = torch.zeros(1, 256, device=DEV), torch.zeros(30, 64, 256, device=DEV), torch.ones(64, device=DEV)
    dh = torch.zeros(30, 64, 256, device=DEV)
    tables, table = [A.RopeTable(64, base=10.0 ** (2 + i)) for i in range(3)], A.RopeTable(64)
    heads, turned, ref = rnd(5, 1, 8, 2, 64), torch.zeros(30, 1, 8, 2, 64, device=DEV), torch.zeros(3, 1, 8, 2, 64, device=DEV)
    for i in range(3):
        ctx.rope([heads], tables[i], outs=[ref[i]])
    torch.cuda.synchronize()
    for i in range(30):
        ctx.dropout(gains[i % 3], gain, p=0.0, seed=0)
        ctx.add_rmsnorm(x, gain[0], y=out[i], eps=0.5)
        ctx.dropout(gains[(i + 1) % 3], gain, p=0.0, seed=0)
        ctx.add_rmsnorm_backward(x, x, ones, gain[0], dh[i])
    for i in range(30):
        table.turns.copy_(tables[i % 3].turns)
        ctx.rope([heads], table, outs=[turned[i]])
    torch.cuda.synchronize()
    for i in range(30):
        r = torch.rsqrt(x.double().square().mean(-1, keepdim=True) + 0.5)
        assert torch.allclose(out[i].double(), x.double() * r * gains[i % 3].double(), rtol=2.0 ** -19, atol=0)
        g = gains[(i + 1) % 3].double()
        u = x.double() * g
        exact = u - x.double() * (u * x.double()).mean(-1, keepdim=True)
        assert torch.allclose(dh[i].double(), exact, rtol=2.0 ** -19, atol=2.0 ** -19 * 200)
        assert torch.equal(turned[i], ref[i % 3])

# --------------------------------------------------------------------------------- residual beside dropout
@pytest.mark.parametrize("p", [0.0, 0.05, 0.1, 0.25, 0.3, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("xt", [F32, BF])
def test_residual_is_returned_as_it_is_where_the_branch_is_dropped(ctx, p, xt):
    """An fp32 residual: bit for bit where the mask drops; elsewhere r + x s is formed by two fused operations with s held as
    a sum of two fp32 numbers, so it is off by the rounding of either (2^-24 of the result, nearly) and by 2^-45 of x s.
    Inf and NaN count where they are kept and nowhere else."""
    rows, d = 50, 1000
    mask = (p, 77, 5)
    x, r = rnd(1, rows, d, dtype=xt, std=2.0), rnd(2, rows, d, std=0.7)
    kept = O.keep_mask(rows * d, *mask).reshape(rows, d)
    s = 65536 / max(65536 - round(p * 65536), 1)
    near = torch.tensor(kept, device=DEV) & (rnd(3, rows, d) > 0)           # the residual cancels the branch, nearly
    r[near] = (x.double() * -s * (1 + 2.0 ** -18 * rnd(4, rows, d).double())).float()[near]
    x[0, ::3], x[1, ::3], x[2, ::3] = float("inf"), float("-inf"), float("nan")
    r[3, ::5], r[4, ::5] = float("inf"), float("-inf")
    x[5], r[5] = 1e38, -3e38                                                # x s may lie outside fp32, the sum does not
    gain, out, h, y = torch.ones(d, device=DEV), torch.empty(rows, d, device=DEV), torch.empty(rows, d, device=DEV), torch.empty_like(x)
    ctx.add_rmsnorm(x, gain, residual=r, h=h, y=y, dropout=mask)
    results = [h]
    if xt == F32:
        ctx.dropout(x, out, p=p, seed=77, offset=5, residual=r)
        wide = torch.zeros(rows, d + 3, device=DEV)[:, :d]                 # rows off the 16-byte grid: element by element
        ctx.dropout(x, wide, p=p, seed=77, offset=5, residual=r)
        off = torch.zeros(rows, d + 3, device=DEV)[:, 1:d + 1]
        ctx.add_rmsnorm(x, gain, residual=r, h=off, y=y, dropout=mask)
        results += [out, wide, off]
    torch.cuda.synchronize()
    dropped = torch.tensor(~kept, device=DEV)
    x64, r64 = np64(x), np64(r)
    with np.errstate(all="ignore"):
        ref = r64 + np.where(kept, x64 * s, 0.0)
        ref = np.where(np.abs(ref) > 3.4028235677973366e38, np.sign(ref) * np.inf, ref)
    finite = np.isfinite(ref)
    tol = (2.0 ** -23 * np.abs(ref) + 2.0 ** -45 * s * np.where(kept, np.abs(x64), 0.0)) * (1 + 2.0 ** -20) + 2.0 ** -149
    for got in results:
        assert torch.equal(got[dropped], r[dropped])
        g = np64(got)
        assert np.array_equal(g[~finite], ref[~finite], equal_nan=True)
        assert (np.abs(g[finite] - ref[finite]) <= tol[finite]).all()

# ------------------------------------------------------------------------------------------------- rotary
def test_rope_refuses_outputs_that_fall_on_one_another(ctx):
    t = A.RopeTable(64)
    x = rnd(1, 3, 4, 5, 64)
    flat = torch.empty(1 << 16, device=DEV)
    before = ctx.launch_count
    # strides of sample, token and head in heads of 64
    for b, n, h in ((100, 1, 1), (100, 4, 1), (100, 1, 3), (8, 5, 1), (12, 3, 10), (61, 6, 2), (0, 5, 1)):
        with pytest.raises(A.AdlocoError) as e:
            ctx.rope([x], t, outs=[flat.as_strided(x.shape, (b * 64, n * 64, h * 64, 1))])
        assert e.value.status == A.ERR_INVALID_ARG, (b, n, h)
    with pytest.raises(A.AdlocoError) as e:                     # heads of which two share their last and first element
        ctx.rope([x], t, outs=[flat.as_strided(x.shape, (2000, 320, 63, 1))])
    assert e.value.status == A.ERR_INVALID_ARG and ctx.launch_count == before


@pytest.mark.parametrize("b,n,h", [(20, 5, 1), (5, 15, 1), (4, 1, 12), (1, 3, 12), (1, 15, 3), (60, 3, 13), (7, 21, 4), (24, 6, 25), (1, 6, 15), (1, 9, 12)])
def test_rope_writes_wherever_the_outputs_lie_apart(ctx, b, n, h):
    """Any order of the dimensions, also strides that do not nest."""
    shape = (3, 4, 5, 64)
    places = {b * i + n * j + h * k for i in range(3) for j in range(4) for k in range(5)}
    assert len(places) == 60
    t = A.RopeTable(64)
    x = rnd(1, *shape)
    dense = torch.empty_like(x)
    ctx.rope([x], t, outs=[dense])
    flat = torch.full((1 << 14,), 7.0, device=DEV)
    out = flat.as_strided(shape, (b * 64, n * 64, h * 64, 1))
    ctx.rope([x], t, outs=[out])
    torch.cuda.synchronize()
    assert torch.equal(out, dense)
    rest = torch.ones(256, dtype=torch.bool, device=DEV)
    rest[torch.tensor(sorted(places), device=DEV)] = False
    assert (flat.view(256, 64)[rest] == 7).all()


def test_rope_in_place_needs_the_strides_of_the_input(ctx):
    """The same memory in another order is neither in place nor apart."""
    t = A.RopeTable(32)
    buf = rnd(1, 2, 6, 4, 64)
    kept, before = buf.clone(), ctx.launch_count
    for out in (buf.view(2, 4, 6, 64).transpose(1, 2), buf.view(-1).as_strided(buf.shape, (64, 512, 128, 1))):
        with pytest.raises(A.AdlocoError) as e:
            ctx.rope([buf], t, outs=[out])
        assert e.value.status == A.ERR_INVALID_ARG
    assert ctx.launch_count == before and torch.equal(buf, kept)
    # strides of extents of one are not looked at
    one, ref = rnd(2, 1, 1, 4, 64), torch.empty(1, 1, 4, 64, device=DEV)
    ctx.rope([one], t, outs=[ref], first_position=9)
    ctx.rope([one], t, outs=[one.as_strided((1, 1, 4, 64), (7, 9, 64, 1))], first_position=9)
    torch.cuda.synchronize()
    assert torch.equal(one, ref)

# --------------------------------------------------------------------------------------------- the binding
@pytest.mark.parametrize("shape", [(96,), (7, 96), (3, 7, 96), (2, 5, 3, 96)])
def test_norm_backward_takes_its_workspace_for_any_shape_and_stream(ctx, shape):
    """A tensor of three dimensions is samples of rows; any other one is one sample.  With a stream and without."""
    dy, h, gain = rnd(1, *shape), rnd(2, *shape), rnd(3, 96)
    rstd = torch.rsqrt(h.square().mean(-1) + 1e-6)
    B = shape[0] if len(shape) == 3 else 1
    args = [np64(v).reshape(B, -1, 96) for v in (dy, h)] + [np64(rstd).reshape(B, -1), np64(gain)]
    dh_ref, _, n_ref, S_ref = O.add_rmsnorm_backward(*args)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, side):
        dh, n, S = torch.zeros_like(h), torch.zeros(B, device=DEV), torch.zeros(96, device=DEV)
        torch.cuda.synchronize()
        ctx.add_rmsnorm_backward(dy, h, rstd, gain, dh, per_sample_sqnorm=n, grad_sum=S, stream=stream)
        torch.cuda.synchronize()
        assert np.allclose(np64(dh), dh_ref.reshape(shape), rtol=1e-4, atol=1e-5) and np.allclose(np64(n), n_ref, rtol=1e-4)
        assert np.allclose(np64(S), S_ref, rtol=1e-4, atol=1e-4)
    for bad in (dy.reshape(-1)[0], None, dy.cpu(), dy[..., :0]):
        with pytest.raises(A.AdlocoError) as e:
            ctx.add_rmsnorm_backward(bad, h, rstd, gain, dh, grad_sum=S, stream=side)
        assert e.value.status == A.ERR_INVALID_ARG


def test_flags_without_a_truth_value_are_argument_errors(ctx):
    x, gain, r = rnd(1, 2, 4, 64), rnd(2, 64), torch.ones(2, 4, device=DEV)
    n, S = torch.zeros(2, device=DEV), torch.zeros(64, device=DEV)
    q, s, b, sb = pitched(32, 64, 16), pitched(32, 1, 4), pitched(64, 64, 16), torch.full((1, 1), 127, dtype=torch.uint8, device=DEV)
    heads, table, out = rnd(3, 1, 4, 2, 64), A.RopeTable(64), torch.zeros(32, 64, device=DEV)
    neither = torch.tensor([1, 2])
    before = ctx.launch_count
    for call in (lambda: ctx.add_rmsnorm_backward(x, x, r, gain, torch.empty_like(x), per_sample_sqnorm=n, accumulate_norms=neither),
                 lambda: ctx.add_rmsnorm_backward(x, x, r, gain, torch.empty_like(x), grad_sum=S, accumulate_sum=neither),
                 lambda: ctx.rope([heads], table, interleaved=neither),
                 lambda: ctx.rope([heads], table, inverse=neither),
                 lambda: ctx.blockscale_matmul(q, s, b, sb, out, scale_transposed=neither)):
        with pytest.raises(A.AdlocoError) as e:
            call()
        assert e.value.status == A.ERR_INVALID_ARG
    assert ctx.launch_count == before


def test_other_threads_run_while_a_call_waits_for_room_in_the_launch_queue(ctx):
    """Behind a kernel of about half a second the queue fills up and a call waits; a thread that wakes every few
    milliseconds goes on meanwhile."""
    x = torch.zeros(1, 64, device=DEV)
    ctx.dropout(x, x, p=0.5, seed=1)
    torch.cuda.synchronize()
    stop, wakes = threading.Event(), [time.perf_counter()]

    def tick():
        while not stop.wait(0.002):
            wakes.append(time.perf_counter())
    thread = threading.Thread(target=tick)
    thread.start()
    torch.cuda._sleep(1_000_000_000)
    longest = 0.0
    for _ in range(6000):
        t0 = time.perf_counter()
        ctx.dropout(x, x, p=0.5, seed=1)
        longest = max(longest, time.perf_counter() - t0)
        if longest > 0.1:
            break
    t_end = time.perf_counter()
    time.sleep(0.01)
    stop.set()
    thread.join()
    torch.cuda.synchronize()
    if longest <= 0.1:
        pytest.skip("the launch queue took every call")
    gaps = np.diff([w for w in wakes if w <= t_end] + [t_end])
    assert gaps.max() < 0.5 * longest, (gaps.max(), longest)


# ------------------------------------------------------------------------------------------- widths of a row
# one at least of every instantiation that the other file's widths leave out: on the 16-byte grid 512 (two groups a lane, going
# back), 2560 and 2824 (three groups of 128 threads) and what lies between its widths above 4096; off the grid two, three and
# four groups of 128 threads and both forms of 512
@pytest.mark.parametrize("d", [512, 520, 1100, 1500, 2560, 2824, 3001, 3500, 4097, 5001, 5120, 8191, 8200, 9001, 12288, 12001, 16383])
@pytest.mark.parametrize("xt,st", TYPES)
def test_norm_of_every_width_forward(ctx, d, xt, st):
    parity.test_add_rmsnorm(ctx, d, xt, st)


@pytest.mark.parametrize("B,T,d", [(3, 41, 512), (2, 300, 520), (2, 33, 1100), (1, 2500, 1300), (2, 35, 1500), (2, 29, 2560), (1, 1300, 2824), (2, 27, 3001),
                                   (2, 25, 3500), (3, 1, 4097), (2, 700, 4097), (1, 900, 5001), (2, 17, 5120), (2, 13, 8191), (2, 11, 8200),
                                   (1, 700, 9001), (3, 10, 9001), (2, 9, 12288), (1, 500, 12001), (2, 7, 16383), (1, 1, 16383), (300, 1, 5001)])
@pytest.mark.parametrize("xt,st", TYPES)
def test_norm_of_every_width_backward(ctx, B, T, d, xt, st):
    parity.test_add_rmsnorm_backward(ctx, B, T, d, xt, st)


@pytest.mark.parametrize("d", [512, 1100, 2560, 3500, 5001, 8192, 12001])
def test_norm_of_every_width_to_8_bits(ctx, d):
    parity.test_norm_to_8_bits(ctx, d)


# ------------------------------------------------------------------------------------- offsets beyond 32 bits
def far_rows(buffer, at, rows, cols, pitch):
    return buffer[at:].as_strided((rows, cols), (pitch, 1))


def test_rows_that_lie_more_than_32_bits_apart(ctx):
    """Three rows, 2^31 elements from one to the next: every operator finds them, on and off the 16-byte grid."""
    pitch, d = (1 << 31) + 8, 776
    big = torch.empty(2 * pitch + (1 << 16), dtype=BF, device=DEV)
    near = [rnd(i, 3, d, dtype=BF) for i in range(4)]
    gain, mask = rnd(9, d), (0.25, 3, 4)
    for shift in (0, 1):
        x, r, y, h, u, dh = (far_rows(big, 1024 * i + shift, 3, d, pitch) for i in range(6))
        x.copy_(near[0]), r.copy_(near[1]), u.copy_(near[2])
        rstd, ref = torch.empty(3, device=DEV), [torch.empty(3, d, dtype=BF, device=DEV) for _ in range(3)]
        ctx.add_rmsnorm(x, gain, residual=r, h=h, y=y, rstd=rstd, dropout=mask)
        ctx.add_rmsnorm(near[0], gain, residual=near[1], h=ref[0], y=ref[1], dropout=mask)
        torch.cuda.synchronize()
        assert torch.equal(h, ref[0]) and torch.equal(y, ref[1])
        S, S_ref = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        ctx.add_rmsnorm_backward(u, h, rstd, gain, dh, grad_sum=S)
        ctx.add_rmsnorm_backward(near[2], ref[0], rstd, gain, ref[2], grad_sum=S_ref)
        torch.cuda.synchronize()
        assert torch.equal(dh, ref[2]) and torch.allclose(S, S_ref, rtol=2.0 ** -20, atol=2.0 ** -18)
        ctx.dropout(x, y, p=0.25, seed=3, offset=4, residual=r)
        ctx.dropout(near[0], ref[0], p=0.25, seed=3, offset=4, residual=near[1])
        torch.cuda.synchronize()
        assert torch.equal(y, ref[0])
        q, s, q_ref, s_ref = pitched(3, d, 16), pitched(3, 7, 4), pitched(3, d, 16), pitched(3, 7, 4)
        ctx.blockscale_quantize(x, q, s)
        ctx.blockscale_quantize(near[0], q_ref, s_ref)
        torch.cuda.synchronize()
        assert torch.equal(q, q_ref) and torch.equal(s, s_ref)
    # heads: samples and tokens 2^31 elements apart
    table, heads = A.RopeTable(64), rnd(5, 3, 1, 2, 64, dtype=BF)
    ref = torch.empty_like(heads)
    ctx.rope([heads], table, outs=[ref], first_position=7)
    for strides in ((pitch, 128, 64, 1), (1 << 33, pitch, 64, 1)):
        shape = (3, 1, 2, 64) if strides[0] == pitch else (1, 3, 2, 64)
        a, o = big.as_strided(shape, strides), big[4096:].as_strided(shape, strides)
        a.copy_(heads.view(shape))
        pos = torch.full(shape[:2], 7, dtype=torch.int32, device=DEV)
        ctx.rope([a], table, outs=[o], positions=pos)
        torch.cuda.synchronize()
        assert torch.equal(o, ref.view(shape))


@pytest.mark.parametrize("M", [3, 40])
def test_products_whose_operands_pass_32_bits(ctx, M):
    """A's and the output's rows 2^27 (40 rows) or 2^31 (3 rows) apart, B's 2^25."""
    N, K, far = 130, 300, (1 << 31 if M == 3 else 1 << 27) + 16
    a_flat, o_flat = torch.empty((M - 1) * far + 512, dtype=torch.uint8, device=DEV), torch.empty((M - 1) * far + 512, dtype=BF, device=DEV)
    b_flat = torch.empty((N - 1) * ((1 << 25) + 16) + 512, dtype=torch.uint8, device=DEV)
    a, b, out = a_flat.as_strided((M, K), (far, 1)), b_flat.as_strided((N, K), ((1 << 25) + 16, 1)), o_flat.as_strided((M, N), (far, 1))
    x, w = whole(1, M, K, top=8), whole(2, N, K, top=8)
    sa, sb = pitched(M, 3, 4), torch.zeros(2, 3, dtype=torch.uint8, device=DEV)
    ctx.blockscale_quantize(x, a, sa)
    ctx.blockscale_quantize_weight(w, b, sb)
    ctx.blockscale_matmul(a, sa, b, sb, out)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0 and torch.equal(out, (x @ w.t()).to(BF))


def test_the_same_memory_with_another_pitch_is_refused(ctx):
    """An output over its input is in place only where their rows are the same ones."""
    flat = rnd(1, 4, 256)
    tight, spaced = flat.view(-1).as_strided((4, 64), (64, 1)), flat[:, :64]
    x, gain, rstd, kept, before = rnd(2, 4, 64), rnd(3, 64), torch.ones(4, device=DEV), flat.clone(), ctx.launch_count
    for call in (lambda: ctx.add_rmsnorm(x, gain, residual=tight, h=spaced, y=torch.empty_like(x)),
                 lambda: ctx.add_rmsnorm_backward(x, x, rstd, gain, spaced, dh_residual=tight),
                 lambda: ctx.add_rmsnorm_backward(tight, x, rstd, gain, torch.empty_like(x), dx=spaced),
                 lambda: ctx.dropout(tight, spaced, p=0.5, seed=1),
                 lambda: ctx.dropout(x, spaced, p=0.5, seed=1, residual=tight)):
        with pytest.raises(A.AdlocoError) as e:
            call()
        assert e.value.status == A.ERR_INVALID_ARG
    assert ctx.launch_count == before and torch.equal(flat, kept)
