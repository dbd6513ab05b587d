"""GPU parity of the log-probabilities of given tokens, their entropy and best alternatives, and their gradient against the
fp64 oracle.

Tolerances are arithmetic: sums of exponentials are fp32 sums of positive terms that are right to 2^-20 each (the difference
to the maximum is rounded to 2^-24 of at most 60 before a term stops counting, the fast exponential is right to 2^-22), so
log-sums are right to 2^-18 + 2^-23 of their size; the entropy's terms are weighted by up to that difference."""
import numpy as np
import pytest
import torch

import oracle.layer_oracle as L
from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def np64(t):
    return t.detach().double().cpu().numpy()


def logits_of(seed, n, V, dtype, std=3.0, pitch=None, shift=0):
    g = torch.Generator().manual_seed(seed)
    pitch = V if pitch is None else pitch
    whole = torch.full((n * pitch + shift + 8,), 99.0, dtype=dtype, device=DEV)
    t = whole[shift:shift + n * pitch].view(n, pitch)[:, :V]
    t.copy_((torch.randn(n, V, generator=g) * std).to(dtype))
    return t


def targets_of(seed, n, V):
    t = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    t[::5] = -1
    if n > 3:
        t[3] = V                                             # the first number that is no token
    return t.to(DEV)


def run(ctx, l, t, top, stream=None):
    n = l.shape[0]
    o = {k: torch.full((n,), -9.0, device=DEV) for k in ("logp", "entropy", "lse")}
    if top:
        o["top_values"], o["top_ids"] = torch.full((n, top), -9.0, device=DEV), torch.full((n, top), -9, dtype=torch.int32, device=DEV)
    ctx.token_logprobs(l, t, o["logp"], entropy=o["entropy"], lse=o["lse"], top_values=o.get("top_values"), top_ids=o.get("top_ids"), stream=stream)
    return o


def check(o, l, t, top):
    ref = L.logprobs(np64(l), t.cpu().numpy(), top)
    size = np.abs(ref[2])
    for name, want, extra in (("logp", ref[0], 0), ("entropy", ref[1], 2.0 ** -14), ("lse", ref[2], 0), ("top_values", ref[3], 0)):
        if name not in o:
            continue
        got, s = np64(o[name]), (size if want.ndim == 1 else size[:, None])
        with np.errstate(invalid="ignore", over="ignore"):
            want = np.where(np.abs(want) > np.finfo(np.float32).max, want.astype(np.float32), want)      # beyond fp32: an infinity
            off = ~((got == want) | (np.isnan(got) & np.isnan(want)) | (np.abs(got - want) <= 2.0 ** -18 + extra + 2.0 ** -22 * (s + np.abs(want))))
        assert not off.any(), (name, got[off][:4], want[off][:4])
    if top:
        usable = ~np.isnan(ref[2])
        assert (o["top_ids"].cpu().numpy()[usable] == ref[4][usable]).all()
        ids = o["top_ids"].cpu().numpy()
        assert ((ids >= 0) & (ids < l.shape[1])).all() and all(len(set(r)) == top for r in ids)


# a warp a row (to 512), 128 threads (to 4096), a block, and a cluster (few rows from 16384 on)
# (as an earlier rule had it: now a warp a row to 512, a block of 256 threads, and a cluster; test_gpu_token_logprobs_forms.py names the
# kernel of each case and has the many rows that take a warp each up to 12288)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 31, 100, 257, 512, 513, 1000, 4095, 4096, 4097, 9999, 16383, 16384, 50257, 131072])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_logprobs(ctx, V, dtype):
    for n, top, pitch, shift in ((1, 0, None, 0), (5, min(V, 5), None, 0), (7, min(V, 64), V + 3, 1), (75, min(V, 20), None, 3)):
        if n * V > 2_000_000:
            n = 38
        l, t = logits_of(V + n, n, V, dtype, pitch=pitch, shift=shift), targets_of(n, n, V)
        check(run(ctx, l, t, top), l, t, top)


@pytest.mark.parametrize("V", [40, 700, 6000, 20000])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_with_masks_ties_and_no_numbers(ctx, V, dtype):
    lowest = torch.finfo(dtype).min
    l = logits_of(1, 24, V, dtype)
    l[0] = -INF                                              # nothing is left
    l[1] = lowest                                            # the same with the type's lowest number: all are equal
    l[2, 1:] = -INF                                          # one token is left
    l[3, :V // 2] = -INF
    l[4, ::2] = lowest
    l[5, V // 3] = NAN
    l[6, V - 1] = INF
    l[7] = 2.5                                               # all are equal
    l[8] = torch.arange(V, device=DEV).to(dtype) / 8         # ascending, with ties in bf16
    l[9] = -torch.arange(V, device=DEV).to(dtype) / 8
    l[10] = torch.where(torch.arange(V, device=DEV) % 7 == 3, 4.0, -4.0).to(dtype)
    l[11] = 0.0
    l[11, ::2] = -0.0                                        # equal to 0
    l[12] = NAN
    l[13, :] = 1e4
    l[13, 5] = 2e4
    l[14] = torch.finfo(dtype).max
    l[15, 3] = torch.finfo(dtype).max
    l[16, :2] = torch.tensor([lowest, torch.finfo(dtype).max], dtype=dtype, device=DEV)
    l[17, :] = lowest
    l[17, 9] = -INF
    t = targets_of(2, 24, V)
    t[:18] = torch.tensor([1, 1, 0, V - 1, 1, 1, 1, 7, V - 1, 0, 3, 0, 0, 5, 2, 3, 1, 9], dtype=torch.int32, device=DEV)
    for top in (1, 7, 40):
        for rows in (slice(None), slice(0, 9), slice(9, 18)):         # many rows, and few
            check(run(ctx, l[rows], t[rows], top), l[rows], t[rows], top)


@pytest.mark.parametrize("V", [1, 9, 100, 2047, 2049, 8192, 50257])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_backward(ctx, V, dtype):
    for n, pitch, shift, with_entropy in ((1, None, 0, True), (13, None, 0, False), (9, V + 5, 1, True)):
        l, t = logits_of(V, n, V, dtype, std=2.0, pitch=pitch, shift=shift), targets_of(n, n, V)
        o = run(ctx, l, t, 0)
        g = torch.Generator().manual_seed(4)
        d_logp, d_ent = torch.randn(n, generator=g).to(DEV), torch.randn(n, generator=g).to(DEV)
        given = {"entropy": o["entropy"], "d_entropy": d_ent} if with_entropy else {}
        ref = L.logprobs_backward(np64(l), t.cpu().numpy(), np64(o["lse"]), np64(d_logp), *((np64(o["entropy"]), np64(d_ent)) if with_entropy else ()))
        logp = np64(l) - np64(o["lse"])[:, None]
        p = np.exp(logp)
        size = p * (np.abs(np64(d_logp))[:, None] + (np.abs(np64(d_ent))[:, None] * (np.abs(logp) + np.abs(np64(o["entropy"]))[:, None]) if with_entropy else 0))
        round_off = 2.0 ** -8 if dtype == BF else 2.0 ** -24
        tol = round_off * np.abs(ref) + size * (2.0 ** -20 + 2.0 ** -23 * np.abs(logp)) + 2.0 ** -23 * np.abs(np64(d_logp))[:, None] * (p > 0.4) + 1e-37
        for place in ("apart", "other alignment", "in place"):
            if place == "in place":
                got = l.clone() if pitch is None else l
                src = got
            else:
                src, off = l, 0 if place == "apart" else 1
                got = torch.full((n * V + 1,), 7.0, dtype=dtype, device=DEV)[off:off + n * V].view(n, V)
            ctx.token_logprobs_backward(src, t, o["lse"], d_logp, got, **given)
            bad = ~(np.abs(np64(got) - ref) <= tol)
            assert not bad.any(), (place, np64(got)[bad][:4], ref[bad][:4])


def test_backward_of_rows_that_take_no_part(ctx):
    for V in (40, 3000):
        l = logits_of(1, 6, V, F32)
        l[0] = -INF
        l[1] = NAN
        l[2, 3] = INF
        t = torch.tensor([1, -1, -1, 2, -1, 0], dtype=torch.int32, device=DEV)
        o = run(ctx, l, t, 0)
        d = torch.ones(6, device=DEV)
        zero = torch.zeros(6, device=DEV)
        for given in ({}, {"entropy": o["entropy"], "d_entropy": zero}):
            got = torch.full((6, V), 5.0, device=DEV)
            ctx.token_logprobs_backward(l, t, o["lse"], d, got, **given)
            assert bool((got[[0, 1, 2, 4]] == 0).all()) and bool(torch.isfinite(got).all()) and bool((got[3] != 0).any())


def test_gradient_against_differences(ctx):
    V, n = 50, 3
    l, t = logits_of(3, n, V, F32, std=1.0), torch.tensor([4, 0, 49], dtype=torch.int32, device=DEV)
    dl, dh = torch.tensor([1.0, -0.5, 2.0], device=DEV), torch.tensor([0.3, 1.0, -1.0], device=DEV)
    o = run(ctx, l, t, 0)
    got = torch.empty_like(l)
    ctx.token_logprobs_backward(l, t, o["lse"], dl, got, entropy=o["entropy"], d_entropy=dh)
    h = 2.0 ** -5
    for j in range(V):
        both = []
        for s in (h, -h):
            v = l.clone()
            v[:, j] += s
            q = run(ctx, v, t, 0)
            both.append((dl * q["logp"] + dh * q["entropy"]).double())
        # off by h^2 / 6 of a third derivative (at most 3 here) and by 2^-17 of the values over 2 h
        assert bool(((both[0] - both[1]) / (2 * h) - got[:, j].double()).abs().max() < 3 * h * h + 2.0 ** -17 * 3 / (2 * h))


def test_rows_behind_32_bit_offsets(ctx):
    """The last rows of a matrix of more than 2^32 bytes, and of more than 2^31 numbers."""
    V, n = 50000, 43100
    l = torch.empty(n, V, dtype=BF, device=DEV)
    tail = logits_of(5, 4, V, BF)
    l[:-4].zero_()
    l[-4:] = tail
    t = torch.zeros(n, dtype=torch.int32, device=DEV)
    o = run(ctx, l, t, 3)
    want = run(ctx, tail, t[:4], 3)
    for k in o:
        assert torch.allclose(o[k][-4:].double(), want[k].double(), rtol=1e-5), k
    assert torch.allclose(o["logp"][:-4], torch.full((n - 4,), -float(np.log(V)), device=DEV), rtol=1e-5)
    ctx.token_logprobs_backward(l, t, o["lse"], torch.ones(n, device=DEV), l)
    d = torch.empty_like(tail)
    ctx.token_logprobs_backward(tail, t[:4], o["lse"][-4:].contiguous(), torch.ones(4, device=DEV), d)
    assert torch.equal(l[-4:], d)


def test_results_do_not_change_from_run_to_run_or_in_a_graph(ctx):
    for n, V in ((3, 40000), (300, 5000), (400, 300)):
        l, t = logits_of(7, n, V, BF), targets_of(7, n, V)
        first = run(ctx, l, t, 9)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
            again = run(ctx, l, t, 9)
        for _ in range(3):
            for v in again.values():
                v.fill_(-1)
            graph.replay()
            torch.cuda.synchronize()
            for k in first:
                assert torch.equal(first[k], again[k]), k
        del graph
