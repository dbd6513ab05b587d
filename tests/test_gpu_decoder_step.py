"""The example's training step (examples/decoder_step.py) against torch's autograd on the same model in fp32.

8-bit rounding is 2^-4 of a value at most and about 2.6 % of it in the mean square; each product rounds two operands (3.7 %),
a gradient passes through up to a dozen products whose errors are independent and each only a part of the residual
stream's sum: the sums of gradients are held to 25 % in norm and to a cosine of 0.97, their squared norms to 40 %."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle.block_oracle as O
from paper_2508_18182_b200 import binding as A

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("decoder_step", os.path.join(ROOT, "examples", "decoder_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(m, model, tokens, targets, seed):
    """Per-sample gradients of the same model in fp32: {name: [B, ...]} and the loss."""
    B, T = tokens.shape
    d, H = model.d, model.H
    w = O.rope_frequencies(d // H)
    params = {"embed": model.embed, "gain": model.gain, "head": model.head.W}
    for i, b in enumerate(model.blocks):
        params.update({("gain1", i): b["gain1"], ("gain2", i): b["gain2"]} | {(n, i): b[n].W for n in ("qkv", "proj", "up", "down")})
    keep = [torch.tensor(O.keep_mask(B * T * d, model.p, seed, site).reshape(B, T, d), device=tokens.device) for site in range(2 * len(model.blocks))]
    scale = 65536 / (65536 - round(model.p * 65536))
    angle = torch.tensor(np.arange(T)[:, None] * w, device=tokens.device).float()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def norm(h, gain):
        return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * gain

    def turn(x):
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    grads, total = {}, 0.0
    with torch.enable_grad():
        for s in range(B):
            p = {k: v.detach().clone().requires_grad_(True) for k, v in params.items()}
            h = p["embed"][tokens[s].long()]
            for i in range(len(model.blocks)):
                qkv = (norm(h, p["gain1", i]) @ p["qkv", i].T).view(T, 3, H, d // H)
                mixed = m.attention(turn(qkv[:, 0])[None], turn(qkv[:, 1])[None], qkv[None, :, 2])[0].reshape(T, d)
                h = h + torch.where(keep[2 * i][s], mixed @ p["proj", i].T * scale, 0.0)
                out = torch.nn.functional.gelu(norm(h, p["gain2", i]) @ p["up", i].T) @ p["down", i].T
                h = h + torch.where(keep[2 * i + 1][s], out * scale, 0.0)
            loss = torch.nn.functional.cross_entropy(norm(h, p["gain"]) @ p["head"].T, targets[s].long(), reduction="sum") / T
            for k, g in zip(p, torch.autograd.grad(loss, list(p.values()))):
                grads.setdefault(k, []).append(g)
            total += loss.item()
    return {k: torch.stack(v) for k, v in grads.items()}, total


def test_step_matches_autograd():
    m = example()
    ctx = A.Context(0)
    with torch.no_grad():
        model = m.Decoder(ctx, seed=3)
        g = torch.Generator(device=ctx.device).manual_seed(5)
        tokens = torch.randint(0, model.vocab, (6, 48), generator=g, device=ctx.device, dtype=torch.int32)
        targets = torch.randint(0, model.vocab, (6, 48), generator=g, device=ctx.device, dtype=torch.int32)
        loss, norms = model.step(tokens, targets, seed=77)
        again, norms2 = model.step(tokens, targets, seed=77)
    assert ctx.device_status() == 0 and loss == again
    ref, ref_loss = reference(m, model, tokens, targets, 77)
    assert abs(loss.item() / ref_loss - 1) < 0.05
    got = dict(model.sums)
    for i, b in enumerate(model.blocks):
        got.update({(n, i): b[n].S for n in ("qkv", "proj", "up", "down")})
    got["head"] = model.head.S
    assert set(got) == set(ref)
    for k, S in got.items():
        r = ref[k].sum(0)
        off = (S - r).norm() / r.norm()
        cos = torch.nn.functional.cosine_similarity(S.flatten(), r.flatten(), dim=0)
        assert off < 0.25 and cos > 0.97, (k, off.item(), cos.item())
    n_ref = sum(v.flatten(1).square().sum(1) for v in ref.values())
    assert torch.all((norms / n_ref - 1).abs() < 0.4), (norms / n_ref).tolist()
    ctx.close()


def test_example_runs(capsys):
    m = example()
    try:
        m.main()
    finally:
        torch.set_grad_enabled(True)
    assert "next batch" in capsys.readouterr().out
