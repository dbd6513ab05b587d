"""Up to 16 rows into fp32: every 512 terms are added up to nearest, whatever the width says about the warps of a block."""
import pytest
import torch

from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


# a block's warps share K: eight of them, and (for many blocks an SM) two, which then have 8192 terms each; K with a ragged end
@pytest.mark.parametrize("K,N", [(16384, 2048), (16384, 36000), (4096, 36000), (16390, 36000)])
@pytest.mark.parametrize("M", [1, 8, 16, 17])
def test_long_sums(ctx, M, K, N):
    """Off by less than 1e-6 of the result's size (512 terms' share of what the tensor cores cut off, 5e-7)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(M + K + N)
    pitch = -(-K // 8) * 8
    x = torch.randn(M, pitch, generator=g, device=DEV).bfloat16()[:, :K]
    w = (torch.randn(N, pitch, generator=g, device=DEV) * 2.0 ** -7).bfloat16()[:, :K]
    y = torch.empty(M, N, device=DEV)
    ctx.linear(x, w, y)
    off, size = 0.0, 0.0
    for i in range(0, N, 4096):
        ref = x.double() @ w[i:i + 4096].double().t()
        off += float((y[:, i:i + 4096].double() - ref).square().sum())
        size += float(ref.square().sum())
    assert off <= 1e-12 * size, (off / size) ** 0.5
