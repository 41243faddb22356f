"""The operators together, as a training step uses them: the torch.optim front end's gather and
clipping, and the example that trains a small channels-last ResNet with group norm."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24


def _example():
    spec = importlib.util.spec_from_file_location("train_resnet20", os.path.join(ROOT, "examples", "train_resnet20.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def params(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.nn.Parameter(torch.randn(s, generator=g, device="cuda"))
            for s in ((16, 8, 3, 3), (16,), (40, 30), (7,), (2, 3, 4, 5, 6))]


def gradients(ps, seed):
    """The layouts a backward pass leaves: channels-last, contiguous, transposed, none, permuted."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = [torch.randn(p.shape, generator=g, device="cuda") for p in ps]
    ps[0].grad = v[0].contiguous(memory_format=torch.channels_last)
    ps[1].grad = v[1]
    ps[2].grad = v[2].t().contiguous().t()
    ps[3].grad = None
    ps[4].grad = v[4].permute(4, 1, 3, 0, 2).contiguous().permute(3, 1, 4, 2, 0)
    for p, t in zip(ps, v):
        assert p.grad is None or torch.equal(p.grad, t)
    return torch.cat([torch.zeros_like(t).view(-1) if p.grad is None else t.reshape(-1) for p, t in zip(ps, v)])


def optimizer(ps, **more):
    from paper_2306_06098_b200.optim import SparseMFAC
    return SparseMFAC(ps, lr=0.1, m=4, density=0.1, damp=1e-3, **more)


def test_step_reads_every_layout_as_before():
    a, b = params(0), params(0)
    opt_a, opt_b = optimizer(a), optimizer(b)
    for t in range(6):
        flat = gradients(a, t)
        opt_a.step()
        assert torch.equal(opt_a._g, flat)  # bit for bit
        off = 0
        for p in b:
            n = p.numel()
            p.grad = flat[off:off + n].view(p.shape).clone()
            off += n
        opt_b.step()
        assert torch.equal(opt_a._theta, opt_b._theta)
    assert (opt_a.handle.error() == opt_b.handle.error()).all()


@pytest.mark.parametrize("scale", [1.0, 0.125])
def test_clipping_the_gradient(scale):
    ps = params(1)
    opt = optimizer(ps, max_grad_norm=3.0, grad_scale=scale)
    flat = gradients(ps, 9)
    norm = flat.double().norm().item() * scale
    assert norm > 3.0
    opt.step()
    assert abs(opt.last_grad_norm.item() - norm) <= 8 * U * norm
    want = flat.double() * scale * (3.0 / norm)
    assert ((opt._g.double() - want).abs() <= 8 * U * want.abs()).all()
    opt.max_grad_norm = 2 * norm
    for p in ps:
        p.grad = None
    flat = gradients(ps, 9)
    opt.step()
    assert torch.equal(opt._g, flat * scale)  # powers of two: exact
    with pytest.raises(ValueError):
        optimizer(params(2), max_grad_norm=-1.0)


def test_other_gradient_types():
    ps = params(3)
    opt = optimizer(ps)
    flat = gradients(ps, 5)
    opt.step()
    before = opt._g.clone()
    assert torch.equal(before, flat)
    assert opt._gradient(torch.nn.Parameter(torch.zeros(4, device="cuda"))) == 4
    p = torch.zeros(4, dtype=torch.float64, device="cuda", requires_grad=True)
    p.grad = torch.full((4,), 0.1, dtype=torch.float64, device="cuda")
    assert opt._gradient(p).dtype == torch.float32


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_example_learns(dtype):
    mod = _example()
    assert sum(p.numel() for p in mod.ResNet20().parameters()) == 272_474
    losses, opt = mod.train(40, 64, dtype)
    assert opt.handle.status() == 0
    first, last = sum(losses[:4]) / 4, sum(losses[-4:]) / 4
    assert last < 0.8 * first, losses


def test_example_model_agrees_with_torch_group_norm():
    """Loss and gradients of the example's model against the same model with torch's group norm in
    64 bits."""
    mod = _example()
    torch.manual_seed(1)
    model = mod.ResNet20().to(device="cuda", memory_format=torch.channels_last)

    class Plain(torch.nn.Module):
        def __init__(self, g):
            super().__init__()
            self.g = g

        def forward(self, x):
            y = torch.nn.functional.group_norm(x, self.g.groups, self.g.weight, self.g.bias, self.g.eps)
            return torch.relu(y) if self.g.act == "relu" else y

    import copy
    plain = copy.deepcopy(model).double()

    def swap(m):
        for name, child in m.named_children():
            if isinstance(child, mod.GroupNorm):
                setattr(m, name, Plain(child))
            else:
                swap(child)

    swap(plain)
    x, y = next(mod.batches(8, 3, "cuda"))
    with torch.backends.cudnn.flags(allow_tf32=False):
        loss = torch.nn.functional.cross_entropy(model(x), y)
        loss.backward()
    ref = torch.nn.functional.cross_entropy(plain(x.double()), y)
    ref.backward()
    assert abs(loss.item() - ref.item()) <= 1e-4 * abs(ref.item())
    got = torch.cat([p.grad.reshape(-1) for p in model.parameters()]).double()
    want = torch.cat([p.grad.reshape(-1) for p in plain.parameters()])
    # twenty layers of fp32 convolutions, and relus whose argument rounds across zero
    assert (got - want).norm() <= 1e-2 * want.norm()
