"""Scoring recordings, and training, serving and continuing with a small token model, with the token operators (one MI355X).

  python examples/score_tokens.py

1. A WaveNet's teacher-forced logits of some recordings become log probabilities, entropies and alternatives.
2. A token model (the embeddings of the last two classes, added, an RMS norm, an output product) is trained on the same
   recordings: embed -> norm and product (plain torch, with its backward) -> log_probs, then log_probs_grad and
   embed_grad for the gradients of the logits and of the table.
3. The trained model is served in 8 bits: embed -> norm_quant -> matmul_quant -> log_probs.
4. It is served in 4 bits, and continues recordings: embed -> norm_mx -> matmul_mx -> adjust_logits (what came often lately is
   less likely, and only neighbouring classes are allowed) -> log_probs.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import workloads as W  # noqa: E402
from paper_1611_09482_amd import binding, ops  # noqa: E402

CLASSES = 256


def recordings(streams: int, length: int, seed: int = 0):
    """8-bit mu-law classes of a few tones in noise, int32 [streams][length]."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t = torch.arange(length, device="cuda", dtype=torch.float32)
    r = torch.rand((streams, 3, 3), generator=gen, device="cuda")
    x = (0.25 * r[:, :, :1] * torch.sin(t * (0.01 + 0.3 * r[:, :, 1:2]) + 6.2832 * r[:, :, 2:])).sum(1)
    x = (x + 0.01 * torch.randn((streams, length), generator=gen, device="cuda")).clamp(-1, 1)
    y = torch.sign(x) * torch.log1p(255 * x.abs()) / math.log(256.0)
    return ((y + 1) * 127.5 + 0.5).to(torch.int32).clamp(0, 255).contiguous()


def score_wavenet(classes, top: int = 3):
    """Log probabilities of recordings under a (random) WaveNet: its logits go into log_probs as they come."""
    cfg = W.ModelConfig(W.GATED, W.F32, 32, (1, 2, 4, 8, 16, 32), skip_channels=256, head_channels=256)
    model = binding.from_model(cfg, W.make_weights(cfg, 1), max_batch=classes.shape[0])
    before = torch.cat([torch.full_like(classes[:, :1], cfg.seed_input), classes[:, :-1]], 1).contiguous()
    logits = model.teacher_forced_parallel(before)
    return ops.log_probs(logits, classes, top=top)


class TokenModel:
    """logits = W norm(E[now] + E[before] / 2): table E and product W [classes][channels], gain [channels]."""

    def __init__(self, channels: int = 128, seed: int = 0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.table = 0.5 * torch.randn((CLASSES, channels), generator=gen, device="cuda")
        self.product = torch.randn((CLASSES, channels), generator=gen, device="cuda") / math.sqrt(channels)
        self.gain = torch.ones(channels, device="cuda")
        self.eps = 1e-6
        self.optimizer = torch.optim.Adam([self.table, self.product], lr=0.02)

    def train_step(self, now, before, after):
        """One step on the mean negative log probability of `after`; returns it (a tensor)."""
        h = ops.embed(self.table, now).requires_grad_()
        r = ops.embed(self.table, before, scale=0.5).requires_grad_()
        w = self.product.detach().requires_grad_()
        s = h + r
        y = s * torch.rsqrt((s * s).mean(-1, keepdim=True) + self.eps) * self.gain
        logits = y @ w.t()
        scores = ops.log_probs(logits.detach(), after)
        g = torch.full_like(scores.logp, -1.0 / after.numel())
        logits.backward(ops.log_probs_grad(logits.detach(), after, scores.lse, None, g))
        self.table.grad = ops.embed_grad(h.grad, now, CLASSES) + ops.embed_grad(r.grad, before, CLASSES, scale=0.5)
        self.product.grad = w.grad
        self.optimizer.step()
        return -scores.logp.mean()

    def score(self, now, before, after):
        """Negative log probability per token in float32."""
        s = ops.embed(self.table, now) + ops.embed(self.table, before, scale=0.5)
        y = s * torch.rsqrt((s * s).mean(-1, keepdim=True) + self.eps) * self.gain
        return -ops.log_probs(y @ self.product.t(), after).logp

    def serve(self):
        """The model in 8 bits: a function of (now, before, after) that returns LogProbs with 3 alternatives."""
        q = ops.quant_rows(self.product)

        def score(now, before, after):
            x = ops.norm_quant(ops.embed(self.table, now), self.gain, residual=ops.embed(self.table, before, scale=0.5),
                               eps=self.eps)
            return ops.log_probs(ops.matmul_quant(x.q, x.scale, q.q, q.scale, dtype=torch.float32), after, top=3)
        return score


    def serve_four_bits(self):
        """The model in 4 bits: a function of (now, before) that returns its logits."""
        q = ops.quant_mx(self.product)

        def logits(now, before):
            x = ops.norm_mx(ops.embed(self.table, now), self.gain, residual=ops.embed(self.table, before, scale=0.5),
                            eps=self.eps)
            return ops.matmul_mx(x.q, x.scale, q.q, q.scale, row_scale=x.row_scale, dtype=torch.float32)
        return logits


def neighbours(now, reach: int = 16):
    """Grammar of quiet sound, a row of bits each: the next class lies at most `reach` from this one."""
    at = torch.arange(CLASSES, device="cuda")
    near = ((at - now[:, None]).abs() <= reach).view(-1, CLASSES // 32, 32).long()
    return (near << torch.arange(32, device="cuda")).sum(2).to(torch.int32)


def continue_recordings(logits, start, steps: int, frequency: float = 0.02):
    """The most likely continuation of int32 [streams][prompt] under requests: [streams][prompt + steps]."""
    streams, prompt = start.shape
    tokens = torch.cat([start, torch.full((streams, steps), -1, dtype=torch.int32, device="cuda")], 1)
    prompts = torch.full((streams,), prompt, dtype=torch.int32, device="cuda")
    often = torch.full((streams,), frequency, device="cuda")
    none = torch.full((streams,), -1, dtype=torch.int32, device="cuda")
    for t in range(prompt, prompt + steps):
        now, before = tokens[:, t - 1].contiguous(), tokens[:, t - 2].contiguous()
        z = logits(now, before)
        ops.adjust_logits(z, tokens, torch.full_like(prompts, t), prompts=prompts, frequency=often, allowed=neighbours(now), out=z)
        tokens[:, t] = ops.log_probs(z, none, top=1).top_ids[:, 0]
    return tokens


def main(streams: int = 32, length: int = 2000, steps: int = 200):
    classes = recordings(streams, length)
    wavenet = score_wavenet(classes)
    print(f"WaveNet (random weights): {-wavenet.logp.mean().item() / math.log(2):.3f} bits per sample, "
          f"entropy {wavenet.entropy.mean().item() / math.log(2):.3f}, best of the last step: "
          f"{wavenet.top_ids[0, -1].tolist()}", flush=True)
    before, now, after = (classes[:, i:length - 2 + i].reshape(-1).contiguous() for i in range(3))
    model = TokenModel()
    first = model.score(now, before, after).mean().item()
    for i in range(steps):
        loss = model.train_step(now, before, after)
        if i % 50 == 49:
            print(f"step {i + 1}: {loss.item() / math.log(2):.3f} bits per sample", flush=True)
    full = model.score(now, before, after).mean().item()
    served = model.serve()(now, before, after)
    eight = -served.logp.mean().item()
    hit = (served.top_ids == after[:, None]).any(1).float().mean().item()
    print(f"token model: {first / math.log(2):.3f} bits before, {full / math.log(2):.3f} after training, "
          f"{eight / math.log(2):.3f} in 8 bits; the class is among the first three {100 * hit:.0f}% of the time", flush=True)
    logits = model.serve_four_bits()
    four = -ops.log_probs(logits(now, before), after).logp.mean().item()
    more = continue_recordings(logits, classes[:, :64], 64)
    jumps = (more[:, 64:] - more[:, 63:-1]).abs().max().item()
    print(f"in 4 bits: {four / math.log(2):.3f} bits; recordings continued by 64 samples, no step larger than {jumps}", flush=True)
    return first, full, eight


if __name__ == "__main__":
    main()
