"""Which tiles the linear layers take: those that the rule rates best among the ones that there is shared memory for."""
import pytest
import torch

from kernels_run import kernels_of
from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the rule is worked through for 148 SMs")
    c = A.Context(0)
    yield c
    c.close()


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def ran(call):
    found = kernels_of(call)
    assert len(found) == 1, found
    return found[0]


# rows, d, f -> a pair of CTAs, columns of the tile (of both projections)
@pytest.mark.parametrize("M,d,f,pair,columns", [(256, 4096, 1024, "true", "128"), (64, 4096, 512, "true", "128"), (17, 2048, 2048, "true", "128"),
                                                (128, 1024, 1024, "true", "128"), (4096, 2048, 5632, "true", "256")])
def test_gated_linear(ctx, M, d, f, pair, columns):
    x, w, a = z(M, d), z(f, d), z(M, f)
    name, args, _ = ran(lambda: ctx.gated_linear(x, w, w, a))
    assert name == "dense_tile_kernel" and args[1:3] == [pair, columns], args


# few tiles of 64 columns: two blocks a tile while they all run at once, both have eight blocks of K, and their join has room
@pytest.mark.parametrize("M,K,N,share", [(64, 4096, 1024, 2), (256, 2048, 1024, 2), (32, 8192, 512, 2), (256, 900, 1024, 1)])
def test_few_tiles(ctx, M, K, N, share):
    pitch = -(-K // 8) * 8
    x, w, y = z(M, pitch)[:, :K], z(N, pitch)[:, :K], z(M, N)
    name, args, blocks = ran(lambda: ctx.linear(x, w, y))
    assert name == "dense_tile_kernel" and args[1:3] == ["false", "64"], args
    assert blocks == share * -(-M // 128) * -(-N // 64)


def test_no_room_for_two_shares_of_a_tile(ctx):
    """fp32 residual and output beside z and a kept in bf16 take 12 KB a warp: the tiles are those that are best without."""
    M, N, K = 64, 4096, 1024
    dy, w, z_, a, r = z(M, N), z(N, K), z(M, K), z(M, K), z(M, K, dtype=F32)
    name, args, blocks = ran(lambda: ctx.linear_backward(dy, w, r, activation="gelu", z=z_, a=a, residual=r))
    assert name == "dense_tile_kernel" and args[1:3] == ["false", "64"] and blocks == 16, (args, blocks)
