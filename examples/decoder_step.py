"""One training step of a small decoder with the norm test, as a program that uses the library would write it.

The residual stream is fp32, branches and gradients are bf16, the linear layers run in 8 bits (weights quantised once a
step, activations and gradients in their passes); the weight gradients and every parameter's per-sample norms come from
the bf16 activations X and gradients Delta, so the batch-size decision does not see the 8-bit rounding of the weights'
gradient.  Attention and the activation function are plain torch: they are the program's own.

With feed_forward="gated" the feed-forward is the library's gated one in bf16, which keeps its two projections and its input in
8 bits until the backward pass, and the loss is the library's too.

    python examples/decoder_step.py            # a step and its batch-size decision on cuda:0
    python examples/decoder_step.py gated
"""
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_18182_b200 import binding as A

BF, F32 = torch.bfloat16, torch.float32


class Linear8:
    """y = x W^T in 8 bits.  quantise() after every update of W."""

    def __init__(self, ctx, W):
        self.ctx, self.W = ctx, W
        N, K = W.shape
        dev = W.device
        self.q = torch.zeros(N, -(-K // 16) * 16, dtype=torch.float8_e4m3fn, device=dev)[:, :K]
        self.q_t = torch.zeros(K, -(-N // 16) * 16, dtype=torch.float8_e4m3fn, device=dev)[:, :N]
        self.scale = torch.zeros(-(-N // 128), -(-K // 128), dtype=torch.uint8, device=dev)
        self.S = torch.zeros(N, K, device=dev)                       # sum of the per-sample gradients
        self.quantise()

    def quantise(self):
        self.ctx.blockscale_quantize_weight(self.W, self.q, self.scale, q_t=self.q_t)

    def forward(self, q8):
        out = torch.empty(q8[0].shape[0], self.W.shape[0], dtype=BF, device=self.W.device)
        self.ctx.blockscale_matmul(*q8, self.q, self.scale, out)
        return out

    def backward(self, x, dy, norms, B):
        """The input's gradient; adds the weight's sum and per-sample norms."""
        self.ctx.linear_sqnorm(x.view(B, -1, x.shape[-1]), dy.view(B, -1, dy.shape[-1]), norms, accumulate_norms=True, grad_sum=self.S)
        dx = torch.empty(dy.shape[0], self.W.shape[1], dtype=BF, device=dy.device)
        self.ctx.blockscale_matmul(*to_8_bits(self.ctx, dy), self.q_t, self.scale, dx, scale_transposed=True)
        return dx


class Gated:
    """The feed-forward silu(x Wg^T) * (x Wu^T) -> Wd in bf16; both projections' weights are one matrix [2 hidden, d]."""

    def __init__(self, ctx, W, W_down):
        self.ctx, self.W, self.W_down = ctx, W, W_down
        self.S, self.S_down = torch.zeros_like(W), torch.zeros_like(W_down)
        self.refresh()

    def refresh(self):
        """After every update of the weights."""
        self.w, self.w_down = self.W.to(BF), self.W_down.to(BF)

    def forward(self, x, q8):
        """The block's output, and what the backward pass needs: x (as the norm's 8 bits) and the projections in 8 bits."""
        n, f, dev = x.shape[0], self.w_down.shape[1], x.device
        a, out = torch.empty(n, f, dtype=BF, device=dev), torch.empty(n, self.w_down.shape[0], dtype=BF, device=dev)
        gate, up = bytes_for(n, f, dev), bytes_for(n, f, dev)
        self.ctx.gated_linear(x, self.w[:f], self.w[f:], a, gate=gate[0], gate_scale=gate[1], up=up[0], up_scale=up[1])
        self.ctx.linear(a, self.w_down, out)
        return out, (q8, gate, up)

    def backward(self, saved, dy, norms, B):
        """The input's gradient; adds the weights' sums and per-sample norms."""
        (q8, gate, up), n, f, dev = saved, dy.shape[0], self.w_down.shape[1], dy.device
        d_both, a, x = torch.empty(n, 2 * f, dtype=BF, device=dev), torch.empty(n, f, dtype=BF, device=dev), torch.empty(n, self.w.shape[1], dtype=BF, device=dev)
        self.ctx.gated_linear_backward(dy, self.w_down, gate[0], up[0], d_both[:, :f], d_both[:, f:], gate_scale=gate[1], up_scale=up[1], a=a)
        self.ctx.linear_sqnorm(a.view(B, -1, f), dy.view(B, -1, dy.shape[-1]), norms, accumulate_norms=True, grad_sum=self.S_down)
        self.ctx.blockscale_dequantize(*q8, x)
        self.ctx.linear_sqnorm(x.view(B, -1, x.shape[-1]), d_both.view(B, -1, 2 * f), norms, accumulate_norms=True, grad_sum=self.S)
        dx = torch.empty_like(x)
        self.ctx.linear_backward(d_both, self.w, dx)
        return dx


def bytes_for(rows, cols, dev):
    """An 8-bit matrix and its scales, with the pitches that the library asks for."""
    return (torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.float8_e4m3fn, device=dev)[:, :cols],
            torch.zeros(rows, -(-cols // 512) * 4, dtype=torch.uint8, device=dev)[:, :-(-cols // 128)])


def to_8_bits(ctx, x):
    q, s = bytes_for(*x.shape, x.device)
    ctx.blockscale_quantize(x, q, s)
    return q, s


def attention(q, k, v):
    """Causal softmax attention on [B, T, H, D] in fp32."""
    q, k, v = (t.float().transpose(1, 2) for t in (q, k, v))
    s = q @ k.transpose(2, 3) * q.shape[-1] ** -0.5
    s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), float("-inf"))
    return (torch.softmax(s, -1) @ v).transpose(1, 2)


class Decoder:
    def __init__(self, ctx, *, layers=2, d=128, heads=4, hidden=256, vocab=256, p=0.1, seed=0, feed_forward="gelu"):
        self.ctx, self.d, self.H, self.p, self.vocab, self.gated = ctx, d, heads, p, vocab, feed_forward == "gated"
        dev = ctx.device
        g = torch.Generator(device=dev).manual_seed(seed)

        def weight(n, k):
            return torch.randn(n, k, generator=g, device=dev) * k ** -0.5
        self.embed = torch.randn(vocab, d, generator=g, device=dev)
        self.blocks = [{"gain1": torch.ones(d, device=dev), "gain2": torch.ones(d, device=dev), "qkv": Linear8(ctx, weight(3 * d, d)),
                        "proj": Linear8(ctx, weight(d, d))} |
                       ({"ff": Gated(ctx, weight(2 * hidden, d), weight(d, hidden))} if self.gated else
                        {"up": Linear8(ctx, weight(hidden, d)), "down": Linear8(ctx, weight(d, hidden))})
                       for _ in range(layers)]
        self.gain = torch.ones(d, device=dev)
        self.head = Linear8(ctx, weight(vocab, d))
        self.table = A.RopeTable(d // heads, base=10000.0, device=dev)
        self.sums = {}                                               # gradient sums of the vectors and of the embedding

    def _norm(self, x, gain, stream, mask):
        """stream + drop(x), its norm in bf16 (for the weight's gradient) and in 8 bits (for the product)."""
        n, d = stream.shape
        h, y, rstd = torch.empty_like(stream), torch.empty(n, d, dtype=BF, device=stream.device), torch.empty(n, device=stream.device)
        q8 = bytes_for(n, d, stream.device)
        self.ctx.add_rmsnorm(x, gain, residual=stream, h=h, y=y, rstd=rstd, q=q8[0], q_scale=q8[1], dropout=mask)
        return h, y, rstd, q8

    def step(self, tokens, targets, seed):
        """Loss, per-sample squared gradient norms [B]; the gradient sums are in every Linear8.S and in self.sums."""
        ctx, d, H = self.ctx, self.d, self.H
        B, T = tokens.shape
        dev = tokens.device
        masks = [(self.p, seed, site) if self.p > 0 else None for site in range(2 * len(self.blocks))]
        # ---- forward
        stream = torch.zeros(B * T, d, device=dev)
        branch, mask, saved = self.embed[tokens.view(-1).long()].to(BF), None, []
        for i, b in enumerate(self.blocks):
            h1, y1, r1, q8 = self._norm(branch, b["gain1"], stream, mask)
            qkv = b["qkv"].forward(q8).view(B, T, 3, H, d // H)
            ctx.rope([qkv[:, :, 0], qkv[:, :, 1]], self.table)                       # in place, inside the packed product
            with torch.enable_grad():
                qkv.requires_grad_(True)
                mixed = attention(qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]).reshape(B * T, d).to(BF)
            a = b["proj"].forward(to_8_bits(ctx, mixed.detach()))
            h2, y2, r2, q8 = self._norm(a, b["gain2"], h1, masks[2 * i])
            if self.gated:
                branch, kept = b["ff"].forward(y2, q8)
                saved.append((mask, h1, y1, r1, qkv, mixed, h2, None, r2, kept, None))
            else:
                with torch.enable_grad():
                    u = b["up"].forward(q8).requires_grad_(True)
                    act = torch.nn.functional.gelu(u.float()).to(BF)
                saved.append((mask, h1, y1, r1, qkv, mixed, h2, y2, r2, u, act))
                branch = b["down"].forward(to_8_bits(ctx, act.detach()))
            stream, mask = h2, masks[2 * i + 1]
        h, y, r, q8 = self._norm(branch, self.gain, stream, mask)
        if self.gated:
            d_logits = self.head.forward(q8)                                         # the gradient takes the logits' place
            logp, lse = torch.empty(B * T, device=dev), torch.empty(B * T, device=dev)
            ctx.token_logprobs(d_logits, targets.view(-1), logp, lse=lse)
            loss = -logp.sum() / T                                                   # a sample: one sequence
            ctx.token_logprobs_backward(d_logits, targets.view(-1), lse, torch.full_like(logp, -1.0 / T), d_logits)
        else:
            with torch.enable_grad():
                logits = self.head.forward(q8).requires_grad_(True)
                loss = torch.nn.functional.cross_entropy(logits.float(), targets.view(-1).long(), reduction="sum") / T
            d_logits, = torch.autograd.grad(loss, logits)
        # ---- backward
        norms = torch.zeros(B, device=dev)
        dy = self.head.backward(y, d_logits, norms, B)
        d_stream, d_branch = self._norm_back(dy, h, r, self.gain, None, mask, norms, B, "gain")
        for i in reversed(range(len(self.blocks))):
            b, (mask, h1, y1, r1, qkv, mixed, h2, y2, r2, u, act) = self.blocks[i], saved[i]
            if self.gated:
                dy = b["ff"].backward(u, d_branch, norms, B)
            else:
                d_act = b["down"].backward(act.detach(), d_branch, norms, B)
                d_u, = torch.autograd.grad(act, u, d_act)
                dy = b["up"].backward(y2, d_u, norms, B)
            d_stream, d_branch = self._norm_back(dy, h2, r2, b["gain2"], d_stream, masks[2 * i], norms, B, ("gain2", i))
            d_mixed = b["proj"].backward(mixed.detach(), d_branch, norms, B)
            d_qkv, = torch.autograd.grad(mixed, qkv, d_mixed)
            d_qkv = d_qkv.contiguous()
            ctx.rope([d_qkv[:, :, 0], d_qkv[:, :, 1]], self.table, inverse=True)
            dy = b["qkv"].backward(y1, d_qkv.view(B * T, 3 * d), norms, B)
            d_stream, d_branch = self._norm_back(dy, h1, r1, b["gain1"], d_stream, mask, norms, B, ("gain1", i))
        self.sums["embed"] = torch.zeros(self.vocab, d, device=dev)
        ctx.embedding_sqnorm(tokens, d_branch.view(B, T, d), self.vocab, norms, accumulate_norms=True, grad_sum=self.sums["embed"])
        return loss.detach(), norms

    def _norm_back(self, dy, h, rstd, gain, d_stream, mask, norms, B, name):
        S = torch.empty_like(gain)
        dh, dx = torch.empty_like(h), torch.empty_like(dy)
        shape = (B, -1, dy.shape[-1])
        self.ctx.add_rmsnorm_backward(dy.view(shape), h.view(shape), rstd, gain, dh.view(shape), dx=dx.view(shape), dropout=mask,
                                      dh_residual=None if d_stream is None else d_stream.view(shape),
                                      per_sample_sqnorm=norms, accumulate_norms=True, grad_sum=S)
        self.sums[name] = S
        return dh, dx

    def gradient_sums(self):
        feed_forward = [x for b in self.blocks for x in ((b["ff"].S, b["ff"].S_down) if self.gated else (b["up"].S, b["down"].S))]
        return [x for b in self.blocks for x in (b["qkv"].S, b["proj"].S)] + feed_forward + [self.head.S] + list(self.sums.values())


def main(feed_forward="gelu"):
    torch.set_grad_enabled(False)
    ctx = A.Context(0)
    model = Decoder(ctx, feed_forward=feed_forward)
    g = torch.Generator(device=ctx.device).manual_seed(1)
    tokens = torch.randint(0, model.vocab, (8, 64), generator=g, device=ctx.device, dtype=torch.int32)
    loss, norms = model.step(tokens, tokens.roll(-1, 1), seed=1)
    acc = A.Accumulator(ctx, model.gradient_sums())
    acc.accumulate(per_sample_sqnorm=norms)
    result = acc.finalize(A.make_params(0.5, b_cur=8, b_max=32))
    print(f"loss per sequence {loss.item() / 8:.3f}, mean squared norm of a sample's gradient {result.sum_sqnorm / 8:.4g}, "
          f"statistic {result.stat:.3g}: next batch {result.b_req}")
    acc.close()
    ctx.close()


if __name__ == "__main__":
    main(*sys.argv[1:2])
