"""What the linear layers keep in 8 bits is the rounding of well-rounded sums.

A number of 8 bits changes by a whole step, 2^-4 of its size, when its sum falls on the other side of a border between two
of them.  A sum off by e does so with a probability of |e| over the distance of the borders around it.  The sums are claimed to be
off by at most 1e-6 of their size in the norm (every 512 terms are added up to nearest; the tensor cores' own sums of 8192
terms are off by 8e-6), so that over all numbers the expected changes are at most
    1e-6 rms(sums) * the sum of 1 / distance,
and a count of rare independent events stays within six of its standard deviations."""
import numpy as np
import pytest
import torch

import oracle.block_oracle as B
from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    assert c.device_status() == 0
    c.close()


def np64(t):
    return t.detach().double().cpu().numpy()


def normal(seed, n, d, std=1.0):
    return (torch.randn(n, d, generator=torch.Generator().manual_seed(seed)) * std).to(BF).to(DEV)


def bytes_for(n, d):
    return (torch.zeros(n, -(-d // 16) * 16, dtype=torch.uint8, device=DEV)[:, :d],
            torch.zeros(n, -(-d // 512) * 4, dtype=torch.uint8, device=DEV)[:, :-(-d // 128)])


def check(q, s, exact):
    n, d = exact.shape
    got = B.widen(np64(q.contiguous().view(torch.float8_e4m3fn)), s.cpu().numpy().astype(np.int64) - 127, 1)
    blocks = np.pad(np.abs(exact), ((0, 0), (0, -d % 128))).reshape(n, -1, 128)
    scale = np.repeat(np.ldexp(1.0, B.scale_exponent(blocks.max(2))), 128, axis=1)[:, :d]
    # the numbers of 8 bits at an exact sum: steps of an eighth of its power of two, of 2^-9 of the scale at least
    step = np.maximum(np.ldexp(1.0, np.floor(np.log2(np.maximum(np.abs(exact), 1e-300))).astype(np.int64) - 3), 2.0 ** -9 * scale)
    want = np.rint(exact / step) * step
    expected = (1e-6 * np.sqrt((exact ** 2).mean()) / step).sum()
    changed = int((got != want).sum())
    assert changed <= expected + 6 * np.sqrt(expected), (changed, expected, exact.size)


@pytest.mark.parametrize("M,N", [(8, 500), (300, 1000), (2300, 1100)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_linear(ctx, M, N, dtype):
    x, w = normal(1, M, 8192), normal(2, N, 8192, 8192 ** -0.5)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(3)).to(DEV)
    q, s = bytes_for(M, N)
    ctx.linear(x, w, torch.empty(M, N, dtype=dtype, device=DEV), bias=bias, activation="gelu", z=q, z_scale=s)
    check(q, s, np64(x.double() @ w.double().t() + bias.double()))


@pytest.mark.parametrize("M,f", [(8, 500), (300, 1000), (2300, 1100)])
def test_gated_linear(ctx, M, f):
    x, wg, wu = normal(1, M, 8192), normal(2, f, 8192, 8192 ** -0.5), normal(3, f, 8192, 8192 ** -0.5)
    (qg, sg), (qu, su) = bytes_for(M, f), bytes_for(M, f)
    ctx.gated_linear(x, wg, wu, torch.empty(M, f, dtype=BF, device=DEV), gate=qg, up=qu, gate_scale=sg, up_scale=su)
    check(qg, sg, np64(x.double() @ wg.double().t()))
    check(qu, su, np64(x.double() @ wu.double().t()))
