"""The output head from training to serving: a head is trained against tokens and a teacher's top logits in one pass over the vocabulary per step,
without logits in memory, then held in microscaled 4-bit floating point and asked for the next tokens.

    python examples/output_head.py [--tokens 512] [--hidden 256] [--vocab 8000] [--steps 60]

Synthetic data: hidden states around one of `classes` directions, each with a token that goes with it; the teacher knows the direction and a few
tokens near it.  Weights are kept in fp32 beside the bf16 copy that the kernels read, as a training loop does.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2603_05168_amd as sbn  # noqa: E402

DEV = "cuda"


class Data:
    def __init__(self, tokens, hidden, vocab, top=8, classes=64, seed=0):
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.tokens, self.top, self.vocab = tokens, top, vocab
        self.directions = torch.randn(classes, hidden, generator=self.g, device=DEV)
        self.words = torch.randperm(vocab, generator=self.g, device=DEV)[:classes * top].view(classes, top)

    def batch(self):
        at = torch.randint(0, len(self.directions), (self.tokens,), generator=self.g, device=DEV)
        H = self.directions[at] + 0.7 * torch.randn(self.tokens, self.directions.shape[1], generator=self.g, device=DEV)
        targets = self.words[at, 0].clone()
        targets[torch.rand(self.tokens, generator=self.g, device=DEV) < 0.1] = -100   # not part of the answer
        logits = 6.0 - torch.arange(self.top, device=DEV).float() + 0.1 * torch.randn(self.tokens, self.top, generator=self.g, device=DEV)
        return H.bfloat16(), targets, self.words[at].contiguous(), logits


class Head:
    """Weights, gradients, and the workspace of both passes."""

    def __init__(self, tokens, hidden, vocab, top, tau=2.0):
        self.master = torch.randn(vocab, hidden, device=DEV) * 0.02
        self.W, self.dW = self.master.bfloat16(), torch.empty(vocab, hidden, dtype=torch.bfloat16, device=DEV)
        self.dH = torch.empty(tokens, hidden, dtype=torch.bfloat16, device=DEV)
        self.ce, self.kd, self.lse = torch.empty(tokens, device=DEV), torch.empty(tokens, device=DEV), torch.empty(2, tokens, device=DEV)
        self.tau = tau
        self.ws = sbn.new_workspace(sbn.sbn_head_workspace_bytes(tokens, hidden, vocab, top))

    def step(self, H, targets, top_idx, top_logits, lr, weight_kd=0.5):
        """One step; dH is what the blocks below would go on with."""
        kept = (targets >= 0).float()
        d_ce = (1 - weight_kd) * kept / kept.sum().clamp(min=1)
        d_kd = torch.full_like(self.kd, weight_kd / len(H))
        sbn.sbn_head_distill(H, self.W, top_idx, top_logits, self.tau, self.kd, self.lse, self.ws, targets=targets, ce=self.ce)
        sbn.sbn_head_distill_backward(H, self.W, top_idx, top_logits, self.tau, self.lse, d_kd, self.ws, targets=targets, d_ce=d_ce, dH=self.dH, dW=self.dW)
        loss = (self.ce * d_ce).sum() + (self.kd * d_kd).sum()
        self.master -= lr * self.dW
        self.W.copy_(self.master)
        return loss

    def to_mxfp4(self):
        """Codes and scales of the weights, once per checkpoint."""
        codes, scales = (torch.empty(n, dtype=torch.uint8, device=DEV) for n in sbn.sbn_mxfp4_bytes(*self.W.shape))
        sbn.sbn_mxfp4_quantize(self.W, codes, scales)
        return codes, scales


def evaluate(H, W, targets):
    """Mean cross entropy of the tokens that have a target, no gradients."""
    ce, lse = torch.empty(len(H), device=DEV), torch.empty(len(H), device=DEV)
    ws = sbn.new_workspace(sbn.sbn_head_workspace_bytes(len(H), H.shape[1], len(W), backward=False))
    sbn.sbn_head_cross_entropy(H, W, targets, ce, lse, ws)
    return (ce.sum() / (targets >= 0).sum().clamp(min=1)).item()


def serve(H, codes, scales, vocab):
    """Next tokens of a decode batch from the 4-bit head."""
    logits = torch.empty(len(H), vocab, device=DEV)
    sbn.sbn_mxfp4_linear(H, codes, scales, logits, sbn.new_workspace(sbn.sbn_mxfp4_workspace_bytes(*H.shape)))
    return logits.argmax(1), logits


def main(tokens=512, hidden=256, vocab=8000, steps=60, lr=0.3, quiet=False):
    data = Data(tokens, hidden, vocab)
    head = Head(tokens, hidden, vocab, data.top)
    H, targets, _, _ = data.batch()
    before = evaluate(H, head.W, targets)
    for step in range(steps):
        loss = head.step(*data.batch(), lr)
        if not quiet and (step + 1) % max(1, steps // 6) == 0:
            print(f"step {step + 1}: loss {loss.item():.4f}", flush=True)
    after = evaluate(H, head.W, targets)
    codes, scales = head.to_mxfp4()
    kept = targets >= 0
    tokens_4bit, logits = serve(H[kept][:64].contiguous(), codes, scales, vocab)
    agree = (tokens_4bit == targets[kept][:64]).float().mean().item()
    size = (codes.numel() + scales.numel()) / (head.W.numel() * 2)
    if not quiet:
        print(f"cross entropy {before:.3f} -> {after:.3f}; 4-bit head of {size:.2f} of its bf16 bytes: {100 * agree:.0f} % of the tokens")
    return before, after, agree


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("tokens", 512), ("hidden", 256), ("vocab", 8000), ("steps", 60)):
        parser.add_argument(f"--{name}", type=int, default=default)
    parser.add_argument("--lr", type=float, default=0.3)
    main(**vars(parser.parse_args()))
