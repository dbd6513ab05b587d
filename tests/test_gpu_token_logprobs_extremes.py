"""The loss at the ends of the numbers' range, in every form of its kernel (a warp, a block, a cluster a row)."""
import pytest
import torch

from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def run(ctx, l, t, top):
    n = l.shape[0]
    o = [torch.full((n,), -9.0, device=DEV) for _ in range(3)]
    o += [torch.full((n, top), -9.0, device=DEV), torch.full((n, top), -9, dtype=torch.int32, device=DEV)]
    ctx.token_logprobs(l, t, o[0], entropy=o[1], lse=o[2], top_values=o[3], top_ids=o[4])
    return o


# rows, V, from where on all is the lowest number: behind what a thread's first 16 bytes hold, and behind its first four pieces
@pytest.mark.parametrize("n,V,start", [(3, 500, 256), (40, 6000, 2048), (40, 50257, 2048), (40, 50257, 8192), (2, 50257, 4096), (1200, 3000, 256), (1200, 3000, 1024)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_largest_number_and_then_the_lowest(ctx, n, V, start, dtype):
    """One token has all the probability: entropy 0 and log-probability 0 exactly, all others have -Inf (beyond fp32)."""
    ends = torch.finfo(dtype)
    l = torch.zeros(n, V, dtype=dtype, device=DEV)
    l[:, start:] = ends.min
    l[:, 0] = ends.max
    l[n // 2, 0] = ends.max / 2                              # still further than 1e30 from all others
    t = torch.zeros(n, dtype=torch.int32, device=DEV)
    t[0] = V - 1
    logp, entropy, lse, values, ids = run(ctx, l, t, 3)
    assert bool((entropy == 0).all())
    assert torch.equal(lse, l[:, 0].float())
    assert bool((logp[1:] == 0).all()) and float(logp[0]) == -INF
    assert bool((ids == torch.arange(3, dtype=torch.int32, device=DEV)).all())
    assert bool((values[:, 0] == 0).all())


@pytest.mark.parametrize("n,V", [(3, 500), (40, 6000), (2, 50257), (1200, 3000)])
def test_groups_of_the_lowest_number_behind_usual_ones(ctx, n, V):
    """Masked by the type's lowest number: as by -Inf."""
    g = torch.Generator().manual_seed(V)
    l = torch.randn(n, V, generator=g).to(BF).to(DEV)
    l[:, V // 3:] = torch.finfo(BF).min
    t = torch.randint(0, V // 3, (n,), generator=g, dtype=torch.int32).to(DEV)
    got = run(ctx, l, t, 5)
    l[:, V // 3:] = -INF
    for a, b in zip(got, run(ctx, l, t, 5)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n,V", [(3, 500), (40, 6000), (2, 50257), (1200, 3000)])
def test_a_number_added_to_all_logits_changes_no_log_probability(ctx, n, V):
    """Multiples of 2^-6 below 2^15 are fp32 numbers and so are their differences: all but lse is the same to the last bit."""
    g = torch.Generator().manual_seed(V)
    l = torch.randint(-300, 300, (n, V), generator=g).float().div(64).to(DEV)
    t = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).to(DEV)
    first = run(ctx, l, t, 5)
    for shift in (2.0 ** 14, -(2.0 ** 14)):
        other = run(ctx, l + shift, t, 5)
        for i in (0, 1, 3, 4):
            assert torch.equal(first[i], other[i]), i
        assert bool(((other[2].double() - shift - first[2].double()).abs() <= 2.0 ** -9).all())
