"""fp64 restatement of the linear layers with their epilogues, of the gated feed-forward, and of the loss; plain numpy,
no code shared with the CUDA path.  8-bit numbers are block_oracle's."""
import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, name):
    """Value and derivative."""
    z = np.asarray(z, dtype=np.float64)
    if name == "none":
        return z, np.ones_like(z)
    if name == "relu":
        return np.where(z > 0, z, 0.0), (z > 0).astype(np.float64)
    if name == "silu":
        h = np.exp(-np.logaddexp(0.0, -z))
        return z * h, h * (1 + z * (1 - h))
    if name == "gelu":
        h = 0.5 * (1 + _erf(z / math.sqrt(2.0)))
        return z * h, h + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = np.tanh(c * (z + 0.044715 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 0.134145 * z * z)


def linear(x, w, bias=None, activation="none", residual=None):
    """(z, y)"""
    z = np.asarray(x, dtype=np.float64) @ np.asarray(w, dtype=np.float64).T
    if bias is not None:
        z = z + bias
    y = act(z, activation)[0]
    return z, y if residual is None else y + residual


def linear_backward(dy, w, activation="none", z=None, residual=None):
    """(dx, a)"""
    dx = np.asarray(dy, dtype=np.float64) @ np.asarray(w, dtype=np.float64)
    a = None
    if z is not None:
        a, slope = act(z, activation)
        dx = dx * slope
    return dx if residual is None else dx + residual, a


def gated_linear(x, w_gate, w_up, activation="silu"):
    """(gate, up, a)"""
    x = np.asarray(x, dtype=np.float64)
    gate, up = x @ np.asarray(w_gate, dtype=np.float64).T, x @ np.asarray(w_up, dtype=np.float64).T
    return gate, up, act(gate, activation)[0] * up


def gated_linear_backward(dy, w_down, gate, up, activation="silu"):
    """(d_gate, d_up, a)"""
    da = np.asarray(dy, dtype=np.float64) @ np.asarray(w_down, dtype=np.float64)
    a, slope = act(gate, activation)
    return da * up * slope, da * a, a * up


# ------------------------------------------------------------------ the loss
def logprobs(logits, targets=None, top=0):
    """(logp, entropy, lse, top values, top ids); rows of nothing but -inf, and rows with NaN or +inf, as the library states."""
    l = np.asarray(logits, dtype=np.float64)
    n, V = l.shape
    bad = np.isnan(l).any(1) | (l == np.inf).any(1)
    none = (l == -np.inf).all(1)
    safe = np.where((bad | none)[:, None], 0.0, l)
    m = safe.max(1, keepdims=True)
    e = np.exp(safe - m)
    lse = m[:, 0] + np.log(e.sum(1))
    p = e / e.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        entropy = -np.where(p > 0, p * np.log(p), 0.0).sum(1)
    lse = np.where(bad, np.nan, np.where(none, -np.inf, lse))
    entropy = np.where(bad, np.nan, np.where(none, 0.0, entropy))
    logp = None
    if targets is not None:
        given = (targets >= 0) & (targets < V)
        at = l[np.arange(n), np.where(given, targets, 0)]
        with np.errstate(invalid="ignore"):
            logp = np.where(given, np.where(none, -np.inf, at - lse), 0.0)
    # the lower id first among equals: a stable sort of the negated row, NaN last
    order = np.argsort(-l, axis=1, kind="stable")[:, :top]
    with np.errstate(invalid="ignore"):
        values = np.where(none[:, None], -np.inf, np.take_along_axis(l, order, 1) - lse[:, None])
    return logp, entropy, lse, values, order


def logprobs_backward(logits, targets, lse, d_logp, entropy=None, d_entropy=None):
    l = np.asarray(logits, dtype=np.float64)
    n, V = l.shape
    given = (targets >= 0) & (targets < V)
    s = np.where(given, d_logp, 0.0)[:, None]
    c = np.zeros((n, 1)) if d_entropy is None else np.asarray(d_entropy, dtype=np.float64)[:, None]
    H = np.zeros((n, 1)) if entropy is None else np.asarray(entropy, dtype=np.float64)[:, None]
    with np.errstate(invalid="ignore", over="ignore"):
        logp = l - np.asarray(lse, dtype=np.float64)[:, None]
        p = np.exp(logp)
        hit = np.arange(V) == np.where(given, targets, -1)[:, None]
        d = s * (hit - p) - c * np.where(p == 0, 0.0, p * (logp + H))
    return np.where(((s == 0) & (c == 0)) | (np.asarray(lse)[:, None] == -np.inf), 0.0, d)
