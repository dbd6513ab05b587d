"""The fp64 oracle of the linear layers and the loss: closed forms, torch in 64 bits, differences (CPU)."""
import numpy as np
import pytest
import torch

import oracle.layer_oracle as L

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def test_activations_against_torch():
    z = torch.linspace(-9, 9, 721, dtype=torch.float64)
    F = torch.nn.functional
    for name, f in (("relu", F.relu), ("silu", F.silu), ("gelu", F.gelu), ("gelu_tanh", lambda t: F.gelu(t, approximate="tanh"))):
        assert np.allclose(L.act(z.numpy(), name)[0], f(z).numpy(), rtol=1e-13, atol=1e-15), name


@pytest.mark.parametrize("name", ACTS)
def test_slopes_against_differences(name):
    z = np.linspace(-6.03, 6.01, 401)
    h = 1e-5
    slope = (L.act(z + h, name)[0] - L.act(z - h, name)[0]) / (2 * h)      # off by h^2 f''' / 6
    assert np.allclose(L.act(z, name)[1], slope, atol=1e-9)


@pytest.mark.parametrize("name", ACTS)
def test_backward_passes_against_differences(name):
    r = np.random.default_rng(3)
    x, w1, w2, g = r.normal(size=(3, 5)), r.normal(size=(4, 5)), r.normal(size=(6, 4)), r.normal(size=(3, 6))
    wu, h = r.normal(size=(4, 5)), 1e-6

    def two(x):                                   # act(x w1^T) w2^T
        return (L.linear(L.linear(x, w1, activation=name)[1], w2)[1] * g).sum()

    def gated(x):
        return (L.linear(L.gated_linear(x, w1, wu, name)[2], w2)[1] * g).sum()
    z = L.linear(x, w1)[0]
    dz, a = L.linear_backward(g, w2, name, z)
    dx = L.linear_backward(dz, w1)[0]
    gate, up, b = L.gated_linear(x, w1, wu, name)
    dg, du, b2 = L.gated_linear_backward(g, w2, gate, up, name)
    dxg = L.linear_backward(du, wu, residual=L.linear_backward(dg, w1)[0])[0]
    assert np.allclose(a, L.act(z, name)[0]) and np.allclose(b, b2)
    for i in range(3):
        for j in range(5):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((two(x + e) - two(x - e)) / (2 * h) - dx[i, j]) < 1e-7
            assert abs((gated(x + e) - gated(x - e)) / (2 * h) - dxg[i, j]) < 1e-7


def test_logprobs_against_torch():
    g = torch.Generator().manual_seed(1)
    l = (torch.randn(7, 33, generator=g, dtype=torch.float64) * 3).requires_grad_(True)
    t = np.array([0, 32, 5, -1, 33, 7, 7])
    logp, entropy, lse, values, ids = L.logprobs(l.detach().numpy(), t, top=4)
    ls = torch.log_softmax(l, 1)
    H = -(ls.exp() * ls).sum(1)
    keep = torch.tensor([1.0, 1, 1, 0, 0, 1, 1], dtype=torch.float64)
    picked = ls[torch.arange(7), torch.tensor(t).clamp(0, 32)] * keep
    assert np.allclose(logp, picked.detach()) and np.allclose(entropy, H.detach()) and np.allclose(lse, torch.logsumexp(l, 1).detach())
    tv, ti = ls.detach().topk(4, 1)
    assert np.allclose(values, tv) and (ids == ti.numpy()).all()
    dl, dh = torch.randn(7, generator=g, dtype=torch.float64), torch.randn(7, generator=g, dtype=torch.float64)
    want, = torch.autograd.grad((picked * dl).sum() + (H * dh).sum(), l)
    got = L.logprobs_backward(l.detach().numpy(), t, lse, dl.numpy(), entropy, dh.numpy())
    assert np.allclose(got, want.numpy(), atol=1e-12)


def test_logprobs_of_odd_rows():
    inf, nan = np.inf, np.nan
    l = np.array([[-inf] * 4, [0.0, -inf, 0.0, -inf], [1.0, nan, 0.0, 2.0], [1.0, inf, 0.0, 2.0], [2.0, 2.0, 2.0, 2.0]])
    logp, entropy, lse, values, ids = L.logprobs(l, np.array([1, 1, 0, 0, 3]), top=3)
    assert lse[0] == -inf and logp[0] == -inf and entropy[0] == 0 and (values[0] == -inf).all() and (ids[0] == [0, 1, 2]).all()
    assert logp[1] == -inf and np.isclose(entropy[1], np.log(2)) and (ids[1] == [0, 2, 1]).all() and values[1, 2] == -inf
    for r in (2, 3):
        assert np.isnan([lse[r], logp[r], entropy[r]]).all() and np.isnan(values[r]).all()
    assert (ids[4] == [0, 1, 2]).all() and np.allclose(values[4], -np.log(4)) and np.isclose(entropy[4], np.log(4))
    d = L.logprobs_backward(l, np.array([1, -1, -1, -1, 3]), lse, np.ones(5))
    assert (d[:4] == 0).all() and np.allclose(d[4], [-0.25, -0.25, -0.25, 0.75])
