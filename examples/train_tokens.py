"""Trains a small encoder to fill in masked tokens of synthetic sequences, with the library's operators around the
matrix products and the optimizer step: dropout behind the embedding, the residual stream's addition, dropout and
root-mean-square norm in one pass behind each layer, the cross entropy of the tied output layer over the masked
tokens alone, and the Sparse M-FAC step.

    python examples/train_tokens.py [--steps 60] [--batch 16] [--dtype bf16]

A sequence counts up from a random token in steps of one, two or three; no data set is needed.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_06098_b200.dropout import Dropout  # noqa: E402
from paper_2306_06098_b200.loss import LinearCrossEntropy  # noqa: E402
from paper_2306_06098_b200.norm import RMSNorm  # noqa: E402
from paper_2306_06098_b200.optim import SparseMFAC  # noqa: E402

IGNORE = -100


class Attention(torch.nn.Module):
    def __init__(self, d: int, heads: int):
        super().__init__()
        self.heads = heads
        self.qkv = torch.nn.Linear(d, 3 * d, bias=False)
        self.out = torch.nn.Linear(d, d, bias=False)

    def forward(self, x):
        n, length, d = x.shape
        q, k, v = self.qkv(x).view(n, length, 3, self.heads, d // self.heads).permute(2, 0, 3, 1, 4)
        scores = q @ k.transpose(-2, -1) * (d // self.heads) ** -0.5
        mixed = torch.softmax(scores.float(), dim=-1).to(x.dtype) @ v
        return self.out(mixed.transpose(1, 2).reshape(n, length, d))


class Encoder(torch.nn.Module):
    def __init__(self, vocab: int, length: int, d: int = 128, heads: int = 4, layers: int = 2, p: float = 0.1,
                 seed: int = 0):
        super().__init__()
        self.tokens = torch.nn.Embedding(vocab + 1, d)  # the last one stands for a masked token
        self.places = torch.nn.Parameter(0.1 * torch.randn(length, d))
        torch.nn.init.normal_(self.tokens.weight, std=d ** -0.5)
        self.dropout = Dropout(p, seed=seed)
        self.first = RMSNorm(d)
        self.layers, self.norms = torch.nn.ModuleList(), torch.nn.ModuleList()
        for k in range(layers):
            self.layers += [Attention(d, heads),
                            torch.nn.Sequential(torch.nn.Linear(d, 4 * d), torch.nn.GELU(), torch.nn.Linear(4 * d, d))]
            self.norms += [RMSNorm(d, p=p, seed=seed + 2 * k + 1), RMSNorm(d, p=p, seed=seed + 2 * k + 2)]
        self.loss = LinearCrossEntropy(d, vocab + 1, self.tokens.weight, IGNORE)

    def forward(self, tokens, targets, dtype=torch.float32):
        h = self.dropout((self.tokens(tokens) + self.places).to(dtype))
        y = self.first(h)
        for layer, norm in zip(self.layers, self.norms):
            y, h = norm(layer(y), h)
        return self.loss(y, targets)


def batches(batch: int, length: int, vocab: int, seed: int, device):
    """Endless (tokens, targets): 15 % of the tokens are masked, and the others have no target."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def numbers(high, *shape):
        return torch.randint(0, high, shape, generator=gen, device=device)

    while True:
        tokens = (numbers(vocab, batch, 1) + (1 + numbers(3, batch, 1)) * torch.arange(length, device=device)) % vocab
        masked = torch.rand(batch, length, generator=gen, device=device) < 0.15
        yield torch.where(masked, vocab, tokens), torch.where(masked, tokens, IGNORE)


def train(steps: int = 60, batch: int = 16, length: int = 64, vocab: int = 1000, dtype=torch.float32, seed: int = 0,
          log=print):
    torch.manual_seed(seed)
    model = Encoder(vocab, length, seed=seed).cuda()
    opt = SparseMFAC(model.parameters(), lr=3e-3, m=16, density=0.02, damp=1e-4, max_grad_norm=1.0)
    losses = []
    for step, (tokens, targets) in zip(range(steps), batches(batch, length, vocab, seed, "cuda")):
        with torch.autocast("cuda", dtype, enabled=dtype != torch.float32):
            loss = model(tokens, targets, dtype)
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if step % 10 == 0 or step == steps - 1:
            log(f"step {step}: loss {loss.item():.4f}")
    return model, torch.stack(losses)


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--steps", type=int, default=60)
    parser.add_argument("--batch", type=int, default=16)
    parser.add_argument("--dtype", choices=("fp32", "bf16", "fp16"), default="fp32")
    args = parser.parse_args()
    train(args.steps, args.batch, dtype={"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[args.dtype])
