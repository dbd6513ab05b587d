"""Activations and their derivatives where numbers end: the limits at the infinities and at sizes whose square is none, in the
forward and in the backward calls alike."""
import pytest
import torch

from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")
# z, value, derivative (relu, gelu, gelu_tanh and silu are alike there)
POINTS = [(INF, INF, 1.0), (-INF, 0.0, 0.0), (1e20, 1e20, 1.0), (-1e20, 0.0, 0.0), (3e38, 3e38, 1.0), (-3e38, 0.0, 0.0), (250.0, 250.0, 1.0),
          (-250.0, 0.0, 0.0), (190.0, 190.0, 1.0), (-190.0, 0.0, 0.0), (NAN, NAN, NAN)]


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def same(got, want):
    return bool(((got == want) | (torch.isnan(got) & torch.isnan(want))).all())


def points(M):
    z = torch.tensor([p[0] for p in POINTS], dtype=F32).to(BF)
    value, slope = (torch.tensor([p[i] for p in POINTS], dtype=F32) for i in (1, 2))
    value = torch.where(torch.isfinite(z.float()) & (value != 0), z.float(), value)          # as bf16 holds them
    return [t.to(DEV).repeat(M, 1) for t in (z, value, slope)]


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M", [3, 200, 2600])
def test_forward(ctx, act, M):
    """z = x w: one number of each row of w meets the one that is not 0 of x."""
    z, value, _ = points(M)
    n = z.shape[1]
    x, w = torch.zeros(M, 8, dtype=BF, device=DEV), torch.zeros(n, 8, dtype=BF, device=DEV)
    x[:, 0], w[:, 0] = 1, z[0]
    for dtype in (BF, F32):
        y = torch.empty(M, n, dtype=dtype, device=DEV)
        ctx.linear(x, w, y, activation=act)
        assert same(y.float(), value), (act, y[0])


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M", [3, 200, 2600])
def test_backward(ctx, act, M):
    z, value, slope = points(M)
    n = z.shape[1]
    z = torch.nn.functional.pad(z, (0, -n % 8))[:, :n]
    dy, w = torch.zeros(M, 8, dtype=BF, device=DEV), torch.zeros(8, n + -n % 8, dtype=BF, device=DEV)[:, :n]
    dy[:, 0], w[0] = 1, 2
    for dtype in (BF, F32):
        dx, a = torch.empty(M, n, dtype=dtype, device=DEV), torch.empty(M, n, dtype=BF, device=DEV)
        ctx.linear_backward(dy, w, dx, activation=act, z=z, a=a)
        assert same(a.float(), value) and same(dx.float(), 2 * slope), (act, a[0], dx[0])


@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M", [3, 200, 2600])
def test_gated_backward(ctx, act, M):
    z, value, slope = points(M)
    n = z.shape[1]
    z = torch.nn.functional.pad(z, (0, -n % 8))[:, :n]
    up = torch.ones(M, n + -n % 8, dtype=BF, device=DEV)[:, :n]
    dy, w = torch.zeros(M, 8, dtype=BF, device=DEV), torch.zeros(8, n + -n % 8, dtype=BF, device=DEV)[:, :n]
    dy[:, 0], w[0] = 1, 1
    dg, du, a = (torch.empty(M, n, dtype=BF, device=DEV) for _ in range(3))
    ctx.gated_linear_backward(dy, w, z, up, dg, du, activation=act, a=a)
    assert same(a.float(), value) and same(du.float(), value) and same(dg.float(), slope), (act, a[0], du[0], dg[0])
