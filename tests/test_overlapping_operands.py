"""Which operands may share memory, decided on the host: against the sets of bytes that two matrices cover.  The addresses are made
up and the context is an empty one, so this runs only where there is no device to launch on: a call that is not refused ends with the
CUDA error of the missing device."""
import ctypes as C
import random

import pytest
import torch

from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only without a device")
BASE = 1 << 32
FAR = 1 << 40


class LogprobsBackward(C.Structure):
    _fields_ = [("rows", C.c_int64), ("V", C.c_int64), ("logits", C.c_void_p), ("logits_stride", C.c_int64), ("targets", C.c_void_p), ("lse", C.c_void_p),
                ("d_logp", C.c_void_p), ("entropy", C.c_void_p), ("d_entropy", C.c_void_p), ("d_logits", C.c_void_p), ("d_logits_stride", C.c_int64),
                ("reserved", C.c_int32), ("dtype", C.c_int)]


class Logprobs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("V", C.c_int64), ("logits", C.c_void_p), ("logits_stride", C.c_int64), ("targets", C.c_void_p), ("logp", C.c_void_p),
                ("entropy", C.c_void_p), ("lse", C.c_void_p), ("top_values", C.c_void_p), ("top_ids", C.c_void_p), ("top", C.c_int32), ("dtype", C.c_int)]


@pytest.fixture(scope="module")
def lib():
    return A.load_library()


@pytest.fixture(scope="module")
def ctx():
    return C.create_string_buffer(1 << 20)


def covered(p, stride, cols, rows, bytes_):
    return {p + (r * stride + c) * bytes_ + b for r in range(rows) for c in range(cols) for b in range(bytes_)}


def back(lib, ctx, **changes):
    a = LogprobsBackward(rows=4, V=6, logits=BASE, logits_stride=6, targets=FAR, lse=FAR + 4096, d_logp=FAR + 8192, d_logits=FAR + 65536, d_logits_stride=6,
                         dtype=0)
    for k, v in changes.items():
        setattr(a, k, v)
    return lib.adloco_token_logprobs_backward(ctx, C.byref(a), None)


def test_layouts_against_the_bytes_that_they_cover(lib, ctx):
    r = random.Random(5)
    counts = [0, 0, 0]
    for _ in range(4000):
        rows, V = r.randint(1, 5), r.randint(1, 6)
        s = V + r.choice([0, 0, 1, 3, 8, V, 2 * V])
        t = s if r.random() < 0.7 else V + r.randint(0, 12)
        at = BASE + 4 * r.randint(-60, 60)
        mine, other = covered(at, t, V, rows, 4), covered(BASE, s, V, rows, 4)
        same = at == BASE and (rows == 1 or s == t)
        refused = back(lib, ctx, rows=rows, V=V, logits_stride=s, d_logits=at, d_logits_stride=t) == A.ERR_INVALID_ARG
        if mine & other and not same:
            assert refused, (rows, V, s, t, at - BASE)
            counts[0] += 1
        elif same or s == t or rows == 1 or max(mine) < min(other) or max(other) < min(mine):
            assert not refused, (rows, V, s, t, at - BASE)
            counts[1] += 1
        else:
            counts[2] += 1                                   # other pitches within one another's span: may be refused
    assert min(counts[:2]) > 500 and counts[2] < 600, counts


def test_a_row_that_lies_between_other_rows(lib, ctx):
    """The vectors are single rows: between two rows of the gradient they share nothing, over one of them they do."""
    for name in ("targets", "lse", "d_logp"):
        for off in range(0, 4 * 40, 4):
            vector = {BASE + off + i for i in range(4 * 4)}
            shares = bool(vector & covered(BASE, 10, 6, 4, 4))
            got = back(lib, ctx, d_logits=BASE, d_logits_stride=10, logits=FAR + (1 << 20), **{name: BASE + off})
            assert (got == A.ERR_INVALID_ARG) == shares, (name, off)


def test_the_loss(lib, ctx):
    def call(**changes):
        a = Logprobs(rows=4, V=6, logits=BASE, logits_stride=6, targets=FAR, logp=FAR + 4096, entropy=FAR + 8192, lse=FAR + 12288, top_values=FAR + 16384,
                     top_ids=FAR + 20480, top=2, dtype=0)
        for k, v in changes.items():
            setattr(a, k, v)
        return lib.adloco_token_logprobs(ctx, C.byref(a), None)
    assert call() != A.ERR_INVALID_ARG
    outs = ("logp", "entropy", "lse", "top_values", "top_ids")
    sizes = {"logp": 16, "entropy": 16, "lse": 16, "top_values": 32, "top_ids": 32, "targets": 16, "logits": 96}
    places = {"logits": BASE, "targets": FAR, "logp": FAR + 4096, "entropy": FAR + 8192, "lse": FAR + 12288, "top_values": FAR + 16384, "top_ids": FAR + 20480}
    for out in outs:
        for other, at in places.items():
            if other == out:
                continue
            for shift, shares in ((0, True), (4 - sizes[out], True), (-sizes[out], False), (sizes[other] - 4, True), (sizes[other], False)):
                assert (call(**{out: at + shift}) == A.ERR_INVALID_ARG) == shares, (out, other, shift)


def test_restoring(lib, ctx):
    def call(x, q=BASE, scale=BASE + (1 << 20)):
        return lib.adloco_blockscale_dequantize(ctx, 0, 4, 16, q, 16, scale, 4, x, 16, None)
    assert call(FAR) != A.ERR_INVALID_ARG
    for x in (BASE, BASE + 60, BASE - 252, BASE + (1 << 20), BASE + (1 << 20) + 12):
        assert call(x) == A.ERR_INVALID_ARG, x - BASE
    for x in (BASE + 64, BASE - 256, BASE + (1 << 20) + 16):
        assert call(x) != A.ERR_INVALID_ARG, x - BASE
