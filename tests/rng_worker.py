"""Worker for the world_size-2 gloo test of the modules' generators under DistributedDataParallel.
Launched by tests/test_module_generators.py through torch.distributed.run."""
import json
import os
import sys

import torch
import torch.distributed as dist

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
from paper_2306_06098_b200.dropout import Dropout, take  # noqa: E402
from paper_2306_06098_b200.norm import RMSNorm  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.linear = torch.nn.Linear(3, 3)
        self.drop, self.norm = Dropout(0.5), RMSNorm(3, affine=False, p=0.5)
        self.register_buffer("shared", torch.full((1,), float(dist.get_rank())))
        self.taken = []

    def forward(self, x):
        self.taken += [take(self.drop.rng).tolist(), take(self.norm.rng).tolist()]
        return self.linear(x)


def main():
    dist.init_process_group("gloo")
    rank = dist.get_rank()
    torch.manual_seed(100 + rank)
    model = Model()
    seeds = [model.drop.rng[0].item(), model.norm.rng[0].item()]
    wrapped = torch.nn.parallel.DistributedDataParallel(model)
    for _ in range(2):
        wrapped(torch.ones(2, 3)).sum().backward()
    print(json.dumps({"rank": rank, "seeds": seeds, "taken": model.taken, "shared": model.shared.item()}), flush=True)
    dist.barrier()
    dist.destroy_process_group()


if __name__ == "__main__":
    main()
