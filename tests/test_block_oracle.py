"""The oracle of the operators between the linear layers against known answers, closed forms and differences, and
the host function that makes rotary frequencies (no GPU)."""
import ctypes as C

import numpy as np
import pytest

import oracle.block_oracle as O
from paper_2508_18182_b200 import binding as A


@pytest.mark.parametrize("counter,key,answer", [      # the generator's published known answers
    ([0, 0, 0, 0], [0, 0], [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0], [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1])])
def test_generator_known_answers(counter, key, answer):
    assert O.philox(np.array([counter], dtype=np.uint64), key)[0].tolist() == answer


def test_mask_rate_and_independence_of_length():
    m = O.keep_mask(200000, 0.3, 123456789012345, 77)
    assert abs(1 - m.mean() - 0.3) < 5 * np.sqrt(0.3 * 0.7 / 200000)      # five standard deviations
    assert np.array_equal(m[:1003], O.keep_mask(1003, 0.3, 123456789012345, 77))
    assert O.keep_mask(100, 1.0, 1, 1).sum() == 0 and O.keep_mask(100, 0.0, 1, 1).all()
    assert not np.array_equal(m, O.keep_mask(200000, 0.3, 123456789012345, 78))


def test_norm_closed_forms():
    h, y, r = O.add_rmsnorm(np.array([[3.0, -3.0, 3.0, 3.0]]), np.array([1.0, 2.0, 0.5, 0.0]), eps=0.0)
    assert np.allclose(y, [[1.0, -2.0, 0.5, 0.0]]) and np.allclose(r, 1 / 3)
    h, y, r = O.add_rmsnorm(np.zeros((1, 4)), np.ones(4), residual=np.zeros((1, 4)), eps=1e-2)
    assert np.all(y == 0) and np.allclose(r, 10.0)


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(1)
    B, T, d = 2, 3, 7
    x, res, dy, dh_r = (rng.standard_normal((B, T, d)) for _ in range(4))
    gain, mask = rng.standard_normal(d), (0.25, 9, 4)

    def loss(x, res, gain):
        h, y, _ = O.add_rmsnorm(x, gain, res, dropout=mask)
        return np.sum(y * dy) + np.sum(h * dh_r)
    h, _, r = O.add_rmsnorm(x, gain, res, dropout=mask)
    dh, dx, n, S = O.add_rmsnorm_backward(dy, h, r, gain, dh_r, mask)
    step = 1e-6
    for arg, grad in ((0, dx), (1, dh), (2, S)):
        args = [x, res, gain]
        flat = args[arg].reshape(-1)
        for i in range(0, flat.size, 3):
            old = flat[i]
            flat[i] = old + step
            up = loss(*args)
            flat[i] = old - step
            down = loss(*args)
            flat[i] = old
            assert abs((up - down) / (2 * step) - grad.reshape(-1)[i]) < 1e-7 * max(1.0, np.abs(grad).max())
    hat = h * r[..., None]
    assert np.allclose(n, [sum(np.sum(dy[b, :, j] * hat[b, :, j]) ** 2 for j in range(d)) for b in range(B)])


def test_rotation_is_orthogonal_and_depends_on_differences_of_positions():
    rng = np.random.default_rng(2)
    w = O.rope_frequencies(8)
    q, k = rng.standard_normal((1, 1, 1, 10)), rng.standard_normal((1, 1, 1, 10))
    for inter in (False, True):
        turned = O.rope(q, [[1234567]], w, interleaved=inter)
        assert np.allclose(np.sum(turned ** 2), np.sum(q ** 2)) and np.array_equal(turned[..., 8:], q[..., 8:])
        assert np.allclose(O.rope(turned, [[1234567]], w, interleaved=inter, inverse=True), q)
        dots = [np.sum(O.rope(q, [[m]], w, interleaved=inter) * O.rope(k, [[m - 5]], w, interleaved=inter)) for m in (5, 1000)]
        assert np.allclose(dots[0], dots[1])


@pytest.mark.parametrize("R", [2, 10, 64, 96])
@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("by_parts", 8.0)])
def test_library_frequencies(R, scaling, factor):
    t = A.RopeTable(R, base=10000.0, scaling=scaling, factor=factor, context=4096, low=1.0, high=32.0, device="cpu")
    w = O.rope_frequencies(R, 10000.0, scaling, factor, 4096, 1.0, 32.0)
    turns = t.turns_host.numpy().view(np.uint64).astype(np.float64) / 2.0 ** 64
    # both sides come out of pow() and a few operations in 64 bits
    assert np.allclose(turns, w / (2 * np.pi), rtol=1e-14, atol=2.0 ** -64)


def test_library_frequencies_refuse_what_they_cannot_take():
    lib = A.load_library()
    buf = (C.c_uint64 * 64)()

    def call(R=64, base=1e4, scaling=0, factor=1.0, context=4096.0, low=1.0, high=32.0, out=buf):
        return lib.adloco_rope_frequencies(R, base, scaling, factor, context, low, high, out)
    assert call() == A.OK
    for bad in (dict(R=0), dict(R=3), dict(base=0.0), dict(base=float("inf")), dict(scaling=4), dict(scaling=-1), dict(out=None),
                dict(scaling=1, factor=0.0), dict(scaling=2, factor=float("nan")), dict(scaling=3, high=1.0), dict(scaling=3, context=0.0)):
        assert call(**bad) == A.ERR_INVALID_ARG, bad


def test_eight_bit_numbers():
    # every number of the format maps to itself; halves go to the even neighbour
    codes = np.arange(127)
    vals = np.where(codes < 8, codes * 2.0 ** -9, (1 + (codes % 8) / 8) * 2.0 ** (codes // 8 - 7.0))
    assert vals[-1] == 448 and np.array_equal(O.to_e4m3(vals), vals)
    mid = (vals[1:] + vals[:-1]) / 2
    assert np.array_equal(O.to_e4m3(mid), np.where(codes[:-1] % 2 == 0, vals[:-1], vals[1:]))
    # the scale is the smallest power of two that fits
    for amax in (448.0, 448.0001, 449.0, 1.0, 1.75, 1.7500001, 3e-39, 3e38, 0.0):
        e = int(O.scale_exponent(amax))
        assert amax <= 448 * 2.0 ** e and (amax == 0 or e == -127 or amax > 448 * 2.0 ** (e - 1))
    x = np.random.default_rng(0).standard_normal((5, 300)) * 7
    q, e = O.quantise(x, 1)
    assert e.shape == (5, 3) and np.abs(O.widen(q, e, 1) - x).max() <= 2.0 ** -4 * np.abs(x).max()
    assert np.all(np.abs(O.widen(q, e, 1) - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * np.repeat(2.0 ** e, 128, 1)[:, :300])


@pytest.mark.parametrize("rot_dim,kw", [(4, dict(base=1.0, scaling="ntk", factor=1e-200)), (8, dict(scaling="linear", factor=1e-320)),
                                        (8, dict(scaling="by_parts", factor=1e-320, context=1.0, low=10.0, high=20.0))])
def test_frequencies_that_leave_the_range_of_numbers_are_refused(rot_dim, kw):
    with pytest.raises(A.AdlocoError) as e:
        A.RopeTable(rot_dim, device="cpu", **kw)
    assert e.value.status == A.ERR_INVALID_ARG
    A.RopeTable(rot_dim, device="cpu", **{**kw, "factor": 4.0})
