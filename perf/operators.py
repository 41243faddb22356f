"""Measured cases of the operators around an optimizer step.

Two families, as a training program calls them in one step:

* the gradients of a model, a list of many tensors: their global norm (`norm`), clipping
  them in place (`clip`), and gathering them, unscaled and clipped, into the flat fp32
  vector that the optimizer step reads (`gather`);
* group normalisation with an activation on channels-last tensors, forward (`gn_forward`)
  and backward (`gn_backward`).

`own` false computes the plain form with elementary torch operations in fp32; `own` true
calls the library.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
# in-place clipping is repeated on the same tensors, so the threshold follows a schedule that
# falls a little every pass: each pass has something to clip
DECAY = 0.9999


# ------------------------------------------------------------------ parameter shapes
def resnet20_shapes():
    """CIFAR ResNet-20, 272,474 parameters: convolutions, norms, one linear layer."""
    out = [(16, 3, 3, 3), (16,), (16,)]
    c_in = 16
    for c in (16, 32, 64):
        for _ in range(3):
            out += [(c, c_in, 3, 3), (c,), (c,), (c, c, 3, 3), (c,), (c,)]
            if c_in != c:
                out += [(c, c_in, 1, 1), (c,), (c,)]
            c_in = c
    return out + [(10, 64), (10,)]


def resnet18_shapes():
    """ImageNet ResNet-18, 11,689,512 parameters."""
    out = [(64, 3, 7, 7), (64,), (64,)]
    c_in = 64
    for c in (64, 128, 256, 512):
        for block in range(2):
            out += [(c, c_in, 3, 3), (c,), (c,), (c, c, 3, 3), (c,), (c,)]
            if block == 0 and c_in != c:
                out += [(c, c_in, 1, 1), (c,), (c,)]
            c_in = c
    return out + [(1000, 512), (1000,)]


def bert_base_shapes():
    """BERT-base without a head, 109,482,240 parameters; the two feed-forward matrices of a
    layer, four times as wide as the model, are held as four blocks each."""
    h = 768
    out = [(30522, h), (512, h), (2, h), (h,), (h,)]
    for _ in range(12):
        out += [(h, h), (h,)] * 4 + [(h,), (h,)]
        out += [(h, h), (h,)] * 4 + [(h, h)] * 4 + [(h,), (h,), (h,)]
    return out + [(h, h), (h,)]


def ragged_shapes(case):
    """`count` tensors of `total` elements whose sizes spread over orders of magnitude."""
    rng = random.Random(case["layout"])
    w = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(case["count"])]
    total = sum(w)
    out = []
    for x in w:
        n = max(1, int(case["total"] * x / total))
        rows = rng.choice((1, 1, 2, 3, 5, 8, 16, 64))
        out.append((rows, n // rows) if rows > 1 and n >= 2 * rows else (n,))
    return out


SHAPES = {"resnet20": lambda c: resnet20_shapes(), "resnet18": lambda c: resnet18_shapes(),
          "bert_base": lambda c: bert_base_shapes(), "ragged": ragged_shapes}


def layout(case):
    """[(shape, dtype name, absent, strided)] of the gradients, in the order of the parameters."""
    rng = random.Random(case.get("layout", 0) + 1)
    out = []
    for shape in SHAPES[case["set"]](case):
        absent = rng.random() < case["absent"]
        # mixed precision: matrices have half-precision gradients, vectors fp32 ones
        d = ("bf16" if len(shape) > 1 else "f32") if case["dtype"] == "mixed" else case["dtype"]
        out.append((shape, d, absent, bool(case["strided"]) and len(shape) > 1))
    return out


# ------------------------------------------------------------------ cases
def grads(name, op, set_, dtype, *, buckets=False, strided=False, absent=0.0, scale=1.0,
          clips=True, **more):
    return dict(name=name, op=op, set=set_, dtype=dtype, buckets=buckets, strided=strided,
                absent=absent, scale=scale, clips=clips, **more)


def gn(name, op, dtype, n, h, w, c, groups, act, pad=0):
    return dict(name=name, op=op, dtype=dtype, n=n, h=h, w=w, c=c, groups=groups, act=act, pad=pad)


def listed():
    return [
        # logging the gradient norm of a small model every step: launch latency
        grads("norm_resnet20_f32", "norm", "resnet20", "f32"),
        # the same for a transformer in mixed precision: one pass over 220 MB
        grads("norm_bert_base_mixed", "norm", "bert_base", "mixed"),
        # clipping between the backward pass and any optimizer, gradients in one bucket
        grads("clip_resnet18_f32", "clip", "resnet18", "f32", buckets=True),
        # what the optimizer does first: the gradients of channels-last convolutions into its
        # flat vector; small
        grads("gather_resnet20_channels_last", "gather", "resnet20", "f32", strided=True),
        # many odd sizes at odd addresses, fp16 with a loss scale, some parameters unused
        grads("gather_ragged_f16", "gather", "ragged", "f16", buckets=True, absent=0.1,
              scale=1.0 / 1024, count=301, total=23_456_789, layout=5),
        # the largest: BERT-base from bf16 gradients, clipped
        grads("gather_bert_base_bf16", "gather", "bert_base", "bf16"),
        # one image through the last stage of a ResNet-18: latency
        gn("gn_fwd_one_image_f16", "gn_forward", "f16", 1, 7, 7, 512, 32, "relu"),
        # first stage of a CIFAR ResNet-20 at batch 128
        gn("gn_fwd_resnet20_f32", "gn_forward", "f32", 128, 32, 32, 16, 8, "relu"),
        # the stem of an ImageNet ResNet-18 at batch 256, the largest activation it has
        gn("gn_fwd_resnet18_stem_bf16", "gn_forward", "bf16", 256, 112, 112, 64, 32, "relu"),
        # odd sizes, groups of five channels, a channel slice of a concatenation
        gn("gn_bwd_odd_f16", "gn_backward", "f16", 3, 37, 53, 120, 24, "silu", 15),
        # last stage of a CIFAR ResNet-20
        gn("gn_bwd_resnet20_f32", "gn_backward", "f32", 128, 8, 8, 64, 16, "silu"),
        # first stage of an ImageNet ResNet-18 at batch 256
        gn("gn_bwd_resnet18_bf16", "gn_backward", "bf16", 256, 56, 56, 64, 32, "silu"),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "clip", "gather", "gn_forward", "gn_backward"))
    if op.startswith("gn"):
        while True:
            groups, per = log_int(rng, 1, 64), log_int(rng, 1, 64)
            n, h, w = log_int(rng, 1, 256), log_int(rng, 1, 128), log_int(rng, 1, 128)
            size = n * h * w * groups * per
            # with a handful of values in a group the result is all rounding
            if h * w * per >= 16 and 1000 <= size <= 50_000_000:
                break
        acts = ("none", "silu", "relu") if op == "gn_forward" else ("none", "silu")
        # relu's derivative jumps at zero, where two roundings of the same value may differ in
        # sign: its backward is left to the tests, which keep away from the jump
        c = gn("", op, rng.choice(("f32", "bf16", "f16")), n, h, w, groups * per, groups,
               rng.choice(acts), rng.choice((0, 0, 0, 1, 8, 32)))
    else:
        dtype = rng.choice(("f32", "bf16", "f16", "mixed"))
        if op == "clip":  # half-precision values do not follow a threshold that falls slowly
            dtype = "f32"
        count = log_int(rng, 1, 500)
        c = grads("", op, "ragged", dtype,
                  buckets=op == "clip" or rng.random() < 0.5,
                  strided=op != "clip" and rng.random() < 0.25,
                  absent=rng.choice((0.0, 0.0, 0.2)) if count >= 20 else 0.0,
                  scale=1.0 / 1024 if dtype == "f16" else 1.0,
                  clips=op == "clip" or rng.random() < 0.7,
                  count=count, total=log_int(rng, 1000, 40_000_000),
                  layout=rng.randrange(1 << 30))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def prepare_grads(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    specs = layout(case)
    total = {}
    for shape, d, absent, _ in specs:
        if not absent:
            total[d] = total.get(d, 0) + math.prod(shape)
    loss_scale = 1.0 / case["scale"]
    store = {d: torch.randn(n, device="cuda", generator=gen).to(DTYPES[d])
             for d, n in sorted(total.items())}
    at = dict.fromkeys(store, 0)
    tensors = []
    for shape, d, absent, strided in specs:
        n = math.prod(shape)
        if absent:
            tensors.append(n)  # an unused parameter: only its number of coordinates is known
            continue
        t = store[d][at[d]:at[d] + n]
        at[d] += n
        # layers differ in the size of their gradients
        t.mul_(1e-3 * loss_scale * math.exp(rng.gauss(0.0, 1.0)))
        if not case["buckets"]:
            t = t.clone()
        if strided and len(shape) == 4:
            k, c, r, s = shape
            t = t.view(k, r, s, c).permute(0, 3, 1, 2)
        elif strided:
            t = t.view(shape[1], shape[0]).t()
        else:
            t = t.view(shape)
        tensors.append(t)
    here = [t for t in tensors if not isinstance(t, int)]
    norm = math.sqrt(sum(t.double().square().sum().item() for t in store.values())) * case["scale"]
    state = {"case": case, "tensors": tensors, "here": here, "passes": 0,
             "max_norm": 0.37 * norm if case["clips"] else 2.0 * norm,
             "norm": torch.zeros((), device="cuda")}
    if case["op"] == "gather":
        d = sum(math.prod(s[0]) for s in specs)
        state["flat"] = torch.empty(d, device="cuda")
    if case["op"] == "clip":
        state["store"] = [store[d] for d in sorted(store)]
    return state


def channels_last(case, dtype, gen, spread):
    """(n, c, h, w) with the channels last in memory, a slice of a wider tensor when pad > 0."""
    n, h, w, c, pad = (case[k] for k in ("n", "h", "w", "c", "pad"))
    t = torch.randn(n, h, w, c + pad, device="cuda", generator=gen)
    if spread:  # channels of a convolution's output differ in mean and size
        t.mul_(torch.exp(0.3 * torch.randn(c + pad, device="cuda", generator=gen)))
        t.add_(torch.randn(c + pad, device="cuda", generator=gen))
    return t.to(dtype)[..., :c].permute(0, 3, 1, 2)


def prepare_gn(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, c = DTYPES[case["dtype"]], case["c"]
    state = {"case": case, "x": channels_last(case, dtype, gen, True),
             "weight": 1.0 + 0.2 * torch.randn(c, device="cuda", generator=gen),
             "bias": 0.2 * torch.randn(c, device="cuda", generator=gen)}
    if case["op"] == "gn_backward":
        state["dy"] = channels_last(dict(case, pad=0), dtype, gen, False)
        state["mean"], state["rstd"] = statistics(grouped(state["x"], case["groups"]))
    return state


def prepare(case, seed):
    return prepare_gn(case, seed) if case["op"].startswith("gn") else prepare_grads(case, seed)


# ------------------------------------------------------------------ plain forms
def plain_flat(tensors):
    return torch.cat([torch.zeros(t, device="cuda") if isinstance(t, int)
                      else t.reshape(-1).float() for t in tensors])


def plain_factor(norm, max_norm):
    return torch.where(norm > max_norm, max_norm / norm, torch.ones_like(norm))


def plain_clip(state, max_norm):
    norm = plain_flat(state["here"]).square().sum().sqrt()
    f = plain_factor(norm, max_norm)
    [t.mul_(f) if t.dtype == torch.float32 else t.copy_(t.float() * f) for t in state["here"]]
    return norm


def plain_gather(state):
    g = plain_flat(state["tensors"]) * state["case"]["scale"]
    norm = g.square().sum().sqrt()
    torch.mul(g, plain_factor(norm, state["max_norm"]), out=state["flat"])
    return norm


def grouped(x, groups):
    """(n, c, h, w) -> fp32 (n, h w, groups, channels of a group)."""
    n, c, h, w = x.shape
    return x.permute(0, 2, 3, 1).float().reshape(n, h * w, groups, c // groups)


def statistics(v):
    mean = v.mean(dim=(1, 3))
    var = (v - mean[:, None, :, None]).square().mean(dim=(1, 3))
    return mean, 1.0 / torch.sqrt(var + EPS)


def ungrouped(v, x):
    n, c, h, w = x.shape
    return v.reshape(n, h, w, c).permute(0, 3, 1, 2).to(x.dtype)


def plain_gn_forward(s):
    x, groups, act = s["x"], s["case"]["groups"], s["case"]["act"]
    v = grouped(x, groups)
    mean, rstd = statistics(v)
    z = (v - mean[:, None, :, None]) * rstd[:, None, :, None]
    z = z * s["weight"].view(groups, -1) + s["bias"].view(groups, -1)
    if act == "relu":
        z = torch.where(z > 0, z, torch.zeros_like(z))
    elif act == "silu":
        z = z / (1.0 + torch.exp(-z))
    return ungrouped(z, x), mean, rstd


def plain_gn_backward(s):
    x, groups, act = s["x"], s["case"]["groups"], s["case"]["act"]
    weight, rstd = s["weight"].view(groups, -1), s["rstd"][:, None, :, None]
    xhat = (grouped(x, groups) - s["mean"][:, None, :, None]) * rstd
    dz = grouped(s["dy"], groups)
    if act != "none":
        z = xhat * weight + s["bias"].view(groups, -1)
        if act == "relu":
            dz = torch.where(z > 0, dz, torch.zeros_like(dz))
        else:
            sig = 1.0 / (1.0 + torch.exp(-z))
            dz = dz * (sig * (1.0 + z * (1.0 - sig)))
    dzx = dz * xhat
    dweight, dbias = dzx.sum(dim=(0, 1)).reshape(-1), dz.sum(dim=(0, 1)).reshape(-1)
    a = (dz * weight).mean(dim=(1, 3), keepdim=True)
    b = (dzx * weight).mean(dim=(1, 3), keepdim=True)
    dx = rstd * (dz * weight - a - xhat * b)
    return ungrouped(dx, x), dweight, dbias


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2306_06098_b200 import binding
    if op == "norm":
        if own:
            return binding.grad_norm(state["here"], scale=case["scale"], out=state["norm"])
        return plain_flat(state["here"]).square().sum().sqrt() * case["scale"]
    if op == "clip":
        max_norm = state["max_norm"] * DECAY ** state["passes"]
        state["passes"] += 1
        if own:
            norm = binding.clip_grads(state["here"], max_norm, out=state["norm"])
        else:
            norm = plain_clip(state, max_norm)
        return [norm, state["store"]]
    if op == "gather":
        if own:
            norm = binding.gather_grads(state["tensors"], state["flat"], state["max_norm"],
                                        scale=case["scale"], out=state["norm"])
        else:
            norm = plain_gather(state)
        return [norm, state["flat"]]
    if op == "gn_forward":
        if own:
            return list(binding.group_norm_forward(state["x"], case["groups"], state["weight"],
                                                   state["bias"], EPS, case["act"]))
        return list(plain_gn_forward(state))
    if own:
        return list(binding.group_norm_backward(state["dy"], state["x"], state["mean"],
                                                state["rstd"], case["groups"], state["weight"],
                                                state["bias"], case["act"]))
    return list(plain_gn_backward(state))


# ------------------------------------------------------------------ floors and 64 bits
def work(case):
    if case["op"].startswith("gn"):
        b, size = BYTES[case["dtype"]], case["n"] * case["h"] * case["w"] * case["c"]
        small = 8 * case["n"] * case["groups"] + 8 * case["c"]
        if case["op"] == "gn_forward":
            return {"bytes": 2 * b * size + small, "flops": 10 * size}
        return {"bytes": 3 * b * size + small + 8 * case["c"], "flops": 20 * size}
    present = [(math.prod(s), d) for s, d, absent, _ in layout(case) if not absent]
    read = sum(n * BYTES[d] for n, d in present)
    n = sum(n for n, _ in present)
    if case["op"] == "norm":
        return {"bytes": read + 4, "flops": 2 * n}
    if case["op"] == "clip":
        return {"bytes": 2 * read + 4, "flops": 3 * n}
    d = sum(math.prod(s) for s, _, _, _ in layout(case))
    return {"bytes": read + 4 * d + 4, "flops": 4 * n}


def exact(case, seed):
    s = prepare(case, seed)
    if not case["op"].startswith("gn"):
        sq = 0.0
        for t in s["here"]:
            sq = sq + (t.to(torch.float64) ** 2).sum()
        norm = torch.sqrt(sq) * case["scale"]
        if case["op"] == "norm":
            return norm
        f = min(1.0, s["max_norm"] / norm.item())
        if case["op"] == "clip":
            return [norm, [t.to(torch.float64) * f for t in s["store"]]]
        flat = torch.zeros(s["flat"].numel(), dtype=torch.float64, device="cuda")
        at = 0
        for t in s["tensors"]:
            n = t if isinstance(t, int) else t.numel()
            if not isinstance(t, int):
                flat[at:at + n].copy_(t.contiguous().view(-1))
            at += n
        return [norm, flat.mul_(f * case["scale"])]
    # the definition, differentiated by autograd
    x = s["x"].to(torch.float64).contiguous()
    weight, bias = s["weight"].double(), s["bias"].double()
    backward = case["op"] == "gn_backward"
    if backward:
        for t in (x, weight, bias):
            t.requires_grad_(True)
    n, c = x.shape[:2]
    v = x.reshape(n, case["groups"], -1)
    var, mean = torch.var_mean(v, dim=2, correction=0, keepdim=True)
    rstd = (var + EPS).rsqrt()
    z = ((v - mean) * rstd).reshape(x.shape) * weight[:, None, None] + bias[:, None, None]
    y = {"none": lambda q: q, "relu": torch.relu, "silu": lambda q: q * torch.sigmoid(q)}[case["act"]](z)
    if not backward:
        return [y, mean[:, :, 0], rstd[:, :, 0]]
    return list(torch.autograd.grad(y, (x, weight, bias), s["dy"].to(torch.float64)))
