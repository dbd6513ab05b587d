"""Outputs that would race with one another or with an operand are refused before any launch."""
import pytest
import torch

from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def refused(ctx, f, *args, **kw):
    before = ctx.launch_count
    with pytest.raises(A.AdlocoError) as e:
        f(*args, **kw)
    assert e.value.status == A.ERR_INVALID_ARG, e.value
    assert ctx.launch_count == before


def test_scales(ctx):
    M, f = 32, 256
    x, wg, wu, a = z(M, 16), z(f, 16), z(f, 16), z(M, f)
    q, p, s, t = z(M, f, dtype=U8), z(M, f, dtype=U8), z(M, 4, dtype=U8)[:, :2], z(M, 4, dtype=U8)[:, :2]
    refused(ctx, ctx.gated_linear, x, wg, wu, a, gate=q, up=p, gate_scale=s, up_scale=s)              # one buffer for both
    refused(ctx, ctx.gated_linear, x, wg, wu, a, gate=q, up=q, gate_scale=s, up_scale=t)
    over = a.view(U8)[:, :4].as_strided((M, 2), (2 * f, 1))
    refused(ctx, ctx.gated_linear, x, wg, wu, a, gate=q, up=p, gate_scale=over, up_scale=t)           # or in another output
    refused(ctx, ctx.linear, x, wg, a, z=q, z_scale=over)
    refused(ctx, ctx.linear, x, wg, a, z=q, z_scale=q[:, :2])
    refused(ctx, ctx.linear, x, wg, a, z=q, z_scale=x.view(U8)[:, :2])                                # or in an operand
    both = z(M, 8, dtype=U8)                                                                          # columns of one matrix are apart
    ctx.gated_linear(x, wg, wu, a, gate=q, up=p, gate_scale=both[:, :2], up_scale=both[:, 4:6])
    dy, wd = z(M, 16), z(16, f)
    dg, du = z(M, f), z(M, f)
    refused(ctx, ctx.gated_linear_backward, dy, wd, q, p, dg, du, gate_scale=dg.view(U8)[:, :2], up_scale=t)
    arena = z(3 * M * f, dtype=U8)
    q = arena[:M * f].view(M, f)
    refused(ctx, ctx.blockscale_dequantize, q, s, arena[M * f - 512:3 * M * f - 512].view(BF).view(M, f))
    ctx.blockscale_dequantize(q, s, arena[M * f:].view(BF).view(M, f))


def test_parts_of_one_another(ctx):
    M, N = 40, 64
    x, w, whole = z(M, 16), z(N, 16), z(M + 1, 2 * N)
    y, below, beside, shifted = whole[:M, :N], whole[1:, :N], whole[:M, N:], whole[:M, 8:N + 8]
    refused(ctx, ctx.linear, x, w, y, z=below)
    refused(ctx, ctx.linear, x, w, y, z=shifted)
    refused(ctx, ctx.linear, x, w, y, residual=below)
    refused(ctx, ctx.linear, x, w, y, residual=shifted)
    refused(ctx, ctx.linear, x, w, y, bias=whole.view(F32)[3, :N])
    ctx.linear(x, w, y, z=beside, residual=y)
    ctx.linear(x, w, y, residual=beside)
    dy, v = z(M, 16), z(16, N)
    refused(ctx, ctx.linear_backward, dy, v, y, activation="gelu", z=below)
    refused(ctx, ctx.linear_backward, dy, v, y, activation="gelu", z=beside, a=shifted)
    refused(ctx, ctx.linear_backward, dy, v, y, activation="gelu", z=beside, a=below)
    ctx.linear_backward(dy, v, y, activation="gelu", z=beside, a=beside)
    ctx.gated_linear_backward(dy, v, z(M, N), z(M, N), y, beside)


def test_loss(ctx):
    n, V = 12, 100
    l, t = z(n, V, dtype=F32), z(n, dtype=torch.int32)
    v = lambda: z(n, dtype=F32)      # noqa: E731
    refused(ctx, ctx.token_logprobs, l, t, t.view(F32))
    refused(ctx, ctx.token_logprobs, l, t, l[3, :n])
    one = z(2 * n, dtype=F32)
    refused(ctx, ctx.token_logprobs, l, t, one[:n], lse=one[1:n + 1])
    ctx.token_logprobs(l, t, one[:n], lse=one[n:])
    top = z(n, 2, dtype=F32)
    refused(ctx, ctx.token_logprobs, l, t, top.view(-1)[4:4 + n], top_values=top, top_ids=z(n, 2, dtype=torch.int32))
    d = z(n, V, dtype=F32)
    lse, g, e, de = v(), v(), v(), v()
    refused(ctx, ctx.token_logprobs_backward, l, t, d[2, :n], g, d)
    refused(ctx, ctx.token_logprobs_backward, l, t, lse, d[2, 5:n + 5], d)
    refused(ctx, ctx.token_logprobs_backward, l, t, lse, g, d, entropy=d[0, :n], d_entropy=de)
    refused(ctx, ctx.token_logprobs_backward, l, t, lse, g, d, entropy=e, d_entropy=d[n - 1, :n])
    refused(ctx, ctx.token_logprobs_backward, l, d[1, :n].view(torch.int32), lse, g, d)
    both = z(n + 1, V, dtype=F32)
    refused(ctx, ctx.token_logprobs_backward, both[1:], t, lse, g, both[:n])                          # another row's logits
    ctx.token_logprobs_backward(l, t, lse, g, l)
