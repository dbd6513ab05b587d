"""The example's training step with the gated feed-forward and the library's loss against torch's autograd on the same model in
fp32: every gradient, and the per-sample norms.

The 8-bit products of the other layers set the tolerance, as for the step without a gate: sums of gradients are held to 25 %
in norm and to a cosine of 0.97, their squared norms to 40 %; the projections kept in 8 bits round two numbers of the
backward pass (2.6 % each in the mean square) where a bf16 product's operands would be rounded 16 times less."""
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
    angle = torch.tensor(np.arange(T)[:, None] * O.rope_frequencies(d // H), device=tokens.device).float()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    params = {"embed": model.embed, "gain": model.gain, "head": model.head.W}
    for i, b in enumerate(model.blocks):
        params |= {("gain1", i): b["gain1"], ("gain2", i): b["gain2"], ("qkv", i): b["qkv"].W, ("proj", i): b["proj"].W,
                   ("gate_up", i): b["ff"].W, ("down", i): b["ff"].W_down}
    keep = [torch.tensor(O.keep_mask(B * T * d, model.p, seed, site).reshape(B, T, d), device=tokens.device) for site in range(2 * len(model.blocks))]
    scale = 65536 / (65536 - round(model.p * 65536))

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
                gate, up = (norm(h, p["gain2", i]) @ p["gate_up", i].T).chunk(2, -1)
                h = h + torch.where(keep[2 * i + 1][s], (torch.nn.functional.silu(gate) * up) @ p["down", i].T * scale, 0.0)
            loss = torch.nn.functional.cross_entropy(norm(h, p["gain"]) @ p["head"].T, targets[s].long(), ignore_index=-1, reduction="sum") / T
            for k, g in zip(p, torch.autograd.grad(loss, list(p.values()))):
                grads.setdefault(k, []).append(g)
            total += loss.item()
    return {k: torch.stack(v) for k, v in grads.items()}, total


def test_step_matches_autograd():
    m = example()
    ctx = A.Context(0)
    with torch.no_grad():
        model = m.Decoder(ctx, seed=3, feed_forward="gated")
        g = torch.Generator(device=ctx.device).manual_seed(5)
        tokens = torch.randint(0, model.vocab, (6, 48), generator=g, device=ctx.device, dtype=torch.int32)
        targets = torch.randint(0, model.vocab, (6, 48), generator=g, device=ctx.device, dtype=torch.int32)
        targets[:, :5] = -1                                          # a prompt's tokens have no loss
        loss, norms = model.step(tokens, targets, seed=77)
        again, _ = model.step(tokens, targets, seed=77)
    assert ctx.device_status() == 0 and loss == again
    ref, ref_loss = reference(m, model, tokens, targets, 77)
    assert abs(loss.item() / ref_loss - 1) < 0.05
    got = dict(model.sums)
    for i, b in enumerate(model.blocks):
        got |= {("qkv", i): b["qkv"].S, ("proj", i): b["proj"].S, ("gate_up", i): b["ff"].S, ("down", i): b["ff"].S_down}
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
        m.main("gated")
    finally:
        torch.set_grad_enabled(True)
    assert "next batch" in capsys.readouterr().out
