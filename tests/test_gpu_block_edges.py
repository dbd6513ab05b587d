"""GPU tests of the operators between the linear layers at the places where they could go wrong: what only few shapes,
types or callers reach.  Oracle and tolerances as in test_gpu_block_ops.py; whole numbers small enough that every sum
fits fp32 are compared for equality."""
import numpy as np
import pytest
import torch

import oracle.block_oracle as O
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
