"""The forms of the log-probabilities' kernel against the fp64 oracle, the one that ran named: a warp a row where there are rows for
many warps and the row's maxima of 32 lanes bound the best tokens, a block a row, a cluster a row; and calls that leave outputs
out.  Tolerances as in test_gpu_token_logprobs.py."""
import pytest
import torch

from kernels_run import kernels_of
from paper_2508_18182_b200 import binding as A
from test_gpu_token_logprobs import check, logits_of, targets_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def warp_rows():
    """As many rows as give every SM eight, and an odd number of them."""
    return 8 * torch.cuda.get_device_properties(0).multi_processor_count + 1


def outputs(n, top, names=("logp", "entropy", "lse")):
    o = {k: torch.full((n,), -9.0, device=DEV) for k in names}
    if top:
        o["top_values"], o["top_ids"] = torch.full((n, top), -9.0, device=DEV), torch.full((n, top), -9, dtype=torch.int32, device=DEV)
    return o


def call(ctx, l, t, o):
    ctx.token_logprobs(l, t if "logp" in o else None, o.get("logp"), entropy=o.get("entropy"), lse=o.get("lse"), top_values=o.get("top_values"), top_ids=o.get("top_ids"))


def ran(ctx, l, t, o, dtype, threads, cluster=False):
    found = kernels_of(lambda: call(ctx, l, t, o))
    want = ["__nv_bfloat16" if dtype == BF else "float", str(threads), "true" if cluster else "false", "true" if "entropy" in o else "false"]
    assert [f[:2] for f in found] == [("logprob_kernel", want)], found


@pytest.mark.parametrize("V,top,threads", [(513, 0, 32), (513, 24, 32), (513, 25, 256), (4097, 1, 32), (4097, 24, 32), (12288, 8, 32), (12289, 8, 256), (3000, 8, 32)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_rows(ctx, V, top, threads, dtype):
    n = warp_rows()
    for pitch, shift in ((None, 0), (V + 3, 1)):
        l, t = logits_of(V + top, n, V, dtype, pitch=pitch, shift=shift), targets_of(n, n, V)
        o = outputs(n, top)
        ran(ctx, l, t, o, dtype, threads)
        check(o, l, t, top)


@pytest.mark.parametrize("V", [700, 6000])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_rows_with_masks_ties_and_no_numbers(ctx, V, dtype):
    n, ends = warp_rows(), torch.finfo(dtype)
    at = torch.arange(V, device=DEV)
    l, t = logits_of(1, n, V, dtype), targets_of(2, n, V)
    kinds = [lambda r: r.fill_(-INF), lambda r: r.fill_(ends.min), lambda r: r[1:].fill_(-INF), lambda r: r[:V // 2].fill_(-INF), lambda r: r[::2].fill_(ends.min),
             lambda r: r[V // 3].fill_(NAN), lambda r: r[V - 1].fill_(INF), lambda r: r.fill_(2.5), lambda r: r.copy_((at / 8).to(dtype)), lambda r: r.copy_((-at / 8).to(dtype)),
             lambda r: r.copy_(torch.where(at % 7 == 3, 4.0, -4.0).to(dtype)), lambda r: r.copy_(torch.where(at % 2 == 0, -0.0, 0.0).to(dtype)), lambda r: r.fill_(NAN),
             lambda r: r.fill_(ends.max), lambda r: r[3].fill_(ends.max), lambda r: r[9].fill_(-INF)]
    for i, kind in enumerate(kinds):                         # rows of one block and rows far apart
        kind(l[i])
        kind(l[n - 3 - 5 * i])
    for top in (1, 7, 24):
        o = outputs(n, top)
        ran(ctx, l, t, o, dtype, 32)
        check(o, l, t, top)


@pytest.mark.parametrize("n,V,threads,cluster", [(0, 3000, 32, False), (40, 3000, 256, False), (3, 20000, 512, True), (5, 300, 32, False)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_outputs_left_out(ctx, n, V, threads, cluster, dtype):
    n = n or warp_rows()
    l, t = logits_of(V, n, V, dtype), targets_of(n, n, V)
    for names, top in ((("logp",), 0), (("lse",), 0), (("logp", "lse"), 6), (("entropy",), 0), ((), 3), (("logp", "entropy"), 1)):
        o = outputs(n, top, names)
        ran(ctx, l, t, o, dtype, threads, cluster)
        check(o, l, t, top)
