"""What the linear layers, the restoring of 8 bits and the loss refuse, before any launch."""
import pytest
import torch

from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    c = A.Context(0)
    yield c
    c.close()


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def refused(ctx, status, f, *args, **kw):
    before = ctx.launch_count
    with pytest.raises(A.AdlocoError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value
    assert ctx.launch_count == before


def test_linear(ctx):
    x, w, y = z(4, 16), z(24, 16), z(4, 24)
    bad, align, types = A.ERR_INVALID_ARG, A.ERR_ALIGNMENT, A.ERR_UNSUPPORTED
    refused(ctx, bad, ctx.linear, x.float(), w, y)
    refused(ctx, bad, ctx.linear, x, w.half(), y)
    refused(ctx, types, ctx.linear, x, w, y.half())
    refused(ctx, bad, ctx.linear, x, z(24, 15), y)
    refused(ctx, bad, ctx.linear, x, w, z(4, 23))
    refused(ctx, bad, ctx.linear, x, w, z(5, 24))
    refused(ctx, align, ctx.linear, z(4, 15), z(24, 15), y)                   # rows that do not start at 16 bytes
    refused(ctx, align, ctx.linear, z(4, 24)[:, 1:17], w, y)
    refused(ctx, bad, ctx.linear, z(16, 4).t(), w, y)
    refused(ctx, bad, ctx.linear, x, w, y, activation="swish")
    refused(ctx, bad, ctx.linear, x, w, y, activation=3)
    refused(ctx, bad, ctx.linear, x, w, y, bias=z(24))
    refused(ctx, bad, ctx.linear, x, w, y, bias=z(23, dtype=F32))
    refused(ctx, bad, ctx.linear, x, w, y, residual=z(4, 24, dtype=F32))
    refused(ctx, bad, ctx.linear, x, w, y, z=y)
    refused(ctx, bad, ctx.linear, x, w, y, z_scale=z(4, 4, dtype=torch.uint8)[:, :1])
    refused(ctx, align, ctx.linear, x, w, y, z=z(4, 25)[:, :24])
    refused(ctx, align, ctx.linear, x, w, y, z=z(4, 24, dtype=torch.uint8), z_scale=z(4, 4, dtype=torch.uint8)[:, :1])
    refused(ctx, align, ctx.linear, x, w, y, z=z(4, 32, dtype=torch.uint8)[:, :24], z_scale=z(4, 1, dtype=torch.uint8))
    refused(ctx, bad, ctx.linear, z(4, 24), z(24, 24), None)
    square = z(4, 24)
    refused(ctx, bad, ctx.linear, square, z(24, 24), square)                  # over an operand of the product
    refused(ctx, bad, ctx.linear, x, w, z(4, 48)[:, :24], residual=None, z=None, stream="default")
    big = z(4, 48)
    refused(ctx, bad, ctx.linear, x, w, big.as_strided((4, 24), (40, 1)), residual=big.as_strided((4, 24), (48, 1)))      # over it with another pitch
    with pytest.raises(A.AdlocoError):
        ctx.linear(x.cpu(), w, y)


def test_linear_backward(ctx):
    dy, w, dx = z(4, 24), z(24, 16), z(4, 16)
    bad, align = A.ERR_INVALID_ARG, A.ERR_ALIGNMENT
    refused(ctx, bad, ctx.linear_backward, dy, z(23, 16), dx)
    refused(ctx, bad, ctx.linear_backward, dy, w, dx, activation="gelu")      # without z
    refused(ctx, bad, ctx.linear_backward, dy, w, dx, a=z(4, 16))
    refused(ctx, bad, ctx.linear_backward, dy, w, dx, activation="gelu", z=z(4, 16), a=z(4, 16, dtype=F32))
    refused(ctx, bad, ctx.linear_backward, dy, w, dx, activation="gelu", z=z(4, 16), a=dx)
    refused(ctx, align, ctx.linear_backward, dy, z(24, 17)[:, :16], dx)
    f32 = z(4, 16, dtype=F32)
    zz = f32.view(BF)[:, :16]
    refused(ctx, bad, ctx.linear_backward, dy, w, f32, activation="gelu", z=zz)      # fp32 over bf16


def test_gated(ctx):
    x, wg, wu, a = z(4, 16), z(24, 16), z(24, 16), z(4, 24)
    bad, align = A.ERR_INVALID_ARG, A.ERR_ALIGNMENT
    refused(ctx, bad, ctx.gated_linear, x, wg, z(23, 16), a)
    refused(ctx, bad, ctx.gated_linear, x, wg, wu, a.float())
    refused(ctx, bad, ctx.gated_linear, x, wg, wu, a, gate=z(4, 24))          # one without the other
    q, s = z(4, 32, dtype=torch.uint8)[:, :24], z(4, 4, dtype=torch.uint8)[:, :1]
    refused(ctx, bad, ctx.gated_linear, x, wg, wu, a, gate=z(4, 24), up=q, up_scale=s)
    refused(ctx, bad, ctx.gated_linear, x, wg, wu, a, gate=z(4, 24), up=a)
    refused(ctx, align, ctx.gated_linear, x, wg, wu, a, gate=z(4, 25)[:, :24], up=z(4, 24))
    dy, wd = z(4, 16), z(16, 24)
    args = (dy, wd, z(4, 24), z(4, 24), z(4, 24))
    refused(ctx, bad, ctx.gated_linear_backward, *args, None)
    refused(ctx, bad, ctx.gated_linear_backward, dy, wd, None, z(4, 24), z(4, 24), z(4, 24))
    refused(ctx, bad, ctx.gated_linear_backward, *args, args[4])              # two outputs in one place
    refused(ctx, bad, ctx.gated_linear_backward, *args, z(4, 24), gate_scale=s)
    refused(ctx, bad, ctx.gated_linear_backward, *args, z(4, 24), activation="gate")


def test_restore(ctx):
    q, s, x = z(4, 32, dtype=torch.uint8)[:, :24], z(4, 4, dtype=torch.uint8)[:, :1], z(4, 24)
    refused(ctx, A.ERR_UNSUPPORTED, ctx.blockscale_dequantize, q, s, x.half())
    refused(ctx, A.ERR_INVALID_ARG, ctx.blockscale_dequantize, q, s, z(4, 23))
    refused(ctx, A.ERR_ALIGNMENT, ctx.blockscale_dequantize, z(4, 24, dtype=torch.uint8), s, x)
    refused(ctx, A.ERR_INVALID_ARG, ctx.blockscale_dequantize, z(4, 32)[:, :24], s, x)


def test_logprobs(ctx):
    l, t = z(4, 10), z(4, dtype=torch.int32)
    v = lambda: z(4, dtype=F32)      # noqa: E731
    bad, types = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED
    refused(ctx, types, ctx.token_logprobs, l.half(), t, v())
    refused(ctx, bad, ctx.token_logprobs, l, t.long(), v())
    refused(ctx, bad, ctx.token_logprobs, l, None, v())
    refused(ctx, bad, ctx.token_logprobs, l, None, None)
    refused(ctx, bad, ctx.token_logprobs, l, t[:3], v())
    refused(ctx, bad, ctx.token_logprobs, l, t, v().bfloat16())
    refused(ctx, bad, ctx.token_logprobs, l, t, v(), top_values=z(4, 3, dtype=F32))
    refused(ctx, bad, ctx.token_logprobs, l, t, v(), top_values=z(4, 3, dtype=F32), top_ids=z(4, 3, dtype=torch.int64))
    refused(ctx, bad, ctx.token_logprobs, l, t, v(), top_values=z(4, 11, dtype=F32), top_ids=z(4, 11, dtype=torch.int32))
    refused(ctx, types, ctx.token_logprobs, z(4, 100), t, v(), top_values=z(4, 65, dtype=F32), top_ids=z(4, 65, dtype=torch.int32))
    one = v()
    refused(ctx, bad, ctx.token_logprobs, l, t, one, lse=one)                 # two outputs in one place
    refused(ctx, bad, ctx.token_logprobs_backward, l, t, v(), v(), z(4, 10, dtype=F32))
    refused(ctx, bad, ctx.token_logprobs_backward, l, t, v(), v(), z(4, 9))
    refused(ctx, bad, ctx.token_logprobs_backward, l, t, v(), v(), z(4, 10), entropy=v())
    refused(ctx, bad, ctx.token_logprobs_backward, l, t, None, v(), z(4, 10))
    wide = z(4, 30)
    refused(ctx, bad, ctx.token_logprobs_backward, wide.as_strided((4, 10), (30, 1)), t, v(), v(), wide.as_strided((4, 10), (20, 1)))
