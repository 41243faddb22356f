"""Trains a CIFAR-sized ResNet-20 on synthetic images with the library's operators around the
optimizer step: group norm with its activation in every block (channels last, both directions), the
gradients of all layers gathered and clipped in one call, and the Sparse M-FAC step.

    python examples/train_resnet20.py [--steps 60] [--batch 128] [--dtype bf16]

The images are ten random prototypes plus noise, made from a seed; no data set is needed.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_06098_b200.norm import GroupNorm  # noqa: E402
from paper_2306_06098_b200.optim import SparseMFAC  # noqa: E402


class Block(torch.nn.Module):
    def __init__(self, c_in: int, c: int, stride: int, groups: int):
        super().__init__()
        self.conv1 = torch.nn.Conv2d(c_in, c, 3, stride, 1, bias=False)
        self.norm1 = GroupNorm(groups, c, act="relu")
        self.conv2 = torch.nn.Conv2d(c, c, 3, 1, 1, bias=False)
        self.norm2 = GroupNorm(groups, c)
        self.down = None
        if stride != 1 or c_in != c:
            self.down = torch.nn.Sequential(torch.nn.Conv2d(c_in, c, 1, stride, bias=False),
                                            GroupNorm(groups, c))

    def forward(self, x):
        y = self.norm2(self.conv2(self.norm1(self.conv1(x))))
        return torch.relu(y + (x if self.down is None else self.down(x)))


class ResNet20(torch.nn.Module):
    """272,474 parameters with group norm in place of batch norm."""

    def __init__(self, groups: int = 8, classes: int = 10):
        super().__init__()
        self.stem = torch.nn.Conv2d(3, 16, 3, 1, 1, bias=False)
        self.norm = GroupNorm(groups, 16, act="relu")
        blocks, c_in = [], 16
        for c, stride in ((16, 1), (32, 2), (64, 2)):
            for k in range(3):
                blocks.append(Block(c_in, c, stride if k == 0 else 1, groups))
                c_in = c
        self.blocks = torch.nn.Sequential(*blocks)
        self.head = torch.nn.Linear(64, classes)

    def forward(self, x):
        y = self.blocks(self.norm(self.stem(x)))
        return self.head(y.mean(dim=(2, 3)))


def batches(batch: int, seed: int, device):
    """Endless (images, labels): a prototype per class plus noise, channels last."""
    gen = torch.Generator(device=device).manual_seed(seed)
    protos = torch.randn(10, 3, 32, 32, generator=gen, device=device)
    while True:
        y = torch.randint(0, 10, (batch,), generator=gen, device=device)
        x = protos[y] + 1.0 * torch.randn(batch, 3, 32, 32, generator=gen, device=device)
        yield x.contiguous(memory_format=torch.channels_last), y


def train(steps: int, batch: int = 128, dtype: torch.dtype = torch.float32, seed: int = 0,
          max_grad_norm: float = 1.0, device="cuda", report=None):
    """Returns the losses of all steps and the optimizer."""
    torch.manual_seed(seed)
    model = ResNet20().to(device=device, memory_format=torch.channels_last)
    opt = SparseMFAC(model.parameters(), lr=0.3, m=32, density=0.01, damp=1e-4,
                     weight_decay=1e-4, clip_norm=1.0, max_grad_norm=max_grad_norm)
    losses = []
    data = batches(batch, seed + 1, device)
    for t in range(steps):
        x, y = next(data)
        opt.zero_grad()
        with torch.autocast("cuda", dtype=dtype, enabled=dtype != torch.float32):
            logits = model(x)
        loss = torch.nn.functional.cross_entropy(logits.float(), y)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
        if report and (t % report == 0 or t == steps - 1):
            print(f"step {t:4d}  loss {loss.item():.4f}  |g| {opt.last_grad_norm.item():.3f}")
    return [v.item() for v in losses], opt


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=128)
    ap.add_argument("--dtype", choices=("fp32", "bf16", "fp16"), default="fp32")
    a = ap.parse_args()
    dtype = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[a.dtype]
    losses, opt = train(a.steps, a.batch, dtype, report=10)
    assert opt.handle.status() == 0
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
