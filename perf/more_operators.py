"""Measured cases of the operators that stand between and after the matrix products of a transformer.

Three families, as a training program (and an evaluation) calls them:

* root-mean-square norm of a residual stream: the residual's addition and the dropout before it, forward
  (`rms_forward`), backward (`rms_backward`), and forward with an output in 8 bits (`rms_quantize`);
* dropout with a counter-based generator, alone or with a residual, both directions (`dropout`);
* softmax cross entropy of a linear layer over a vocabulary: the losses of tokens (`loss_eval`) and the
  mean loss with the gradients of the hidden states and of the layer (`loss_train`).

`own` false computes the plain form with elementary torch operations in fp32; `own` true calls the library.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
E4M3_MOST = 448.0
IGNORE = -100
M32 = 0xFFFFFFFF


# ------------------------------------------------------------------ cases
def rms(name, op, dtype, rows, d, *, residual=True, p=0.0, pad=0, block=0):
    return dict(name=name, op=op, dtype=dtype, rows=rows, d=d, residual=residual, p=p, pad=pad,
                block=block)


def drop(name, dtype, rows, d, *, residual=False, p=0.1, pad=0):
    return dict(name=name, op="dropout", dtype=dtype, rows=rows, d=d, residual=residual, p=p, pad=pad)


def loss(name, op, dtype, n, d, v, *, labelled=1.0, scale=1.0):
    return dict(name=name, op=op, dtype=dtype, n=n, d=d, v=v, labelled=labelled, scale=scale)


def listed():
    return [
        # one token of a wide model: launch latency
        rms("rms_fwd_one_token_bf16", "rms_forward", "bf16", 1, 4096),
        # BERT-base, 32 sequences of 512: residual, dropout and norm behind each of its blocks
        rms("rms_fwd_bert_base_dropout_bf16", "rms_forward", "bf16", 16384, 768, p=0.1),
        # odd sizes, rows of a wider tensor, fp32
        rms("rms_bwd_odd_f32", "rms_backward", "f32", 1531, 1111, pad=5),
        # a wide model, 16384 tokens: the largest norm
        rms("rms_bwd_wide_bf16", "rms_backward", "bf16", 16384, 4096),
        # a handful of tokens in front of an 8-bit product, one scale a token
        rms("rms_quantize_few_tokens_f16", "rms_quantize", "f16", 7, 2048),
        # the same for a batch, one scale for each 128 columns
        rms("rms_quantize_blocks_bf16", "rms_quantize", "bf16", 8192, 4096, block=128),
        # odd sizes, rows of a wider tensor, fp32, behind the embedding
        drop("dropout_odd_f32", "f32", 517, 1001, pad=3, p=0.25),
        # a wide model's residual stream, forward and backward
        drop("dropout_wide_bf16", "bf16", 16384, 4096, residual=True),
        # scoring four tokens with BERT-base's vocabulary: one pass over the layer
        loss("loss_few_tokens_bf16", "loss_eval", "bf16", 4, 768, 30522),
        # BERT-base's masked tokens: 15 % of 32 sequences of 512 have a label
        loss("loss_bert_base_masked_bf16", "loss_train", "bf16", 16384, 768, 30522, labelled=0.15),
        # odd sizes, fp32, every token labelled
        loss("loss_odd_f32", "loss_train", "f32", 1003, 509, 10007),
        # a wide model with a large vocabulary: the largest loss
        loss("loss_wide_bf16", "loss_train", "bf16", 8192, 4096, 64000, labelled=0.98),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rms_forward", "rms_backward", "rms_quantize", "dropout", "loss_eval",
                     "loss_train"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    if op.startswith("loss"):
        while True:
            n, d, v = log_int(rng, 1, 16384), log_int(rng, 32, 4096), log_int(rng, 500, 100_000)
            if rng.random() < 0.6:
                d = max(32, d // 32 * 32)
            if n * d * v <= (2e11 if dtype == "f32" else 1.2e12):
                break
        c = loss("", op, dtype, n, d, v, labelled=rng.choice((1.0, 1.0, 0.9, 0.5, 0.15)),
                 scale=1024.0 if dtype == "f16" and op == "loss_train" else 1.0)
    else:
        while True:
            rows, d = log_int(rng, 1, 32768), log_int(rng, 32, 16384)
            if rng.random() < 0.6:
                d = max(32, d // 32 * 32)
            if rows * d <= 50_000_000:
                break
        residual, pad = rng.random() < 0.6, rng.choice((0, 0, 0, 1, 8, 64))
        p = rng.choice((0.0, 0.1, 0.3))
        if op == "dropout":
            c = drop("", dtype, rows, d, residual=residual, p=p or 0.5, pad=pad)
        else:
            c = rms("", op, dtype, rows, d, residual=residual, pad=pad,
                    p=0.0 if op == "rms_quantize" else p,
                    block=rng.choice((0, 32, 64, 128)) if op == "rms_quantize" else 0)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    if case["op"].startswith("loss"):
        n, d, v = case["n"], case["d"], case["v"]
        weight = randn(v, d).mul_(2.0 / math.sqrt(d))
        targets = torch.randint(0, v, (n,), device="cuda", generator=gen)
        # a model that has learned something: its hidden states lean towards the target's row
        hidden = randn(n, d).add_(weight[targets], alpha=2.5)
        ignored = n - max(1, round(n * case["labelled"]))
        targets[torch.randperm(n, device="cuda", generator=gen)[:ignored]] = IGNORE
        train = case["op"] == "loss_train"
        return {"case": case, "targets": targets,
                "hidden": hidden.to(dtype).requires_grad_(train),
                "weight": weight.to(dtype).requires_grad_(train),
                # a loss scale, as fp16 gradients need one
                "scale": torch.tensor(case["scale"], device="cuda")}

    rows, d, pad = case["rows"], case["d"], case["pad"]

    def stream():  # activations: columns of different size
        t = randn(rows, d + pad)
        return t.mul_(torch.exp(0.5 * randn(d + pad))).to(dtype)[:, :d]

    state = {"case": case, "x": stream(), "residual": stream() if case["residual"] else None,
             # seed and offset of the generator
             "rng": torch.randint(0, 1 << 62, (2,), device="cuda", generator=gen)}
    if case["op"] == "dropout":
        state["dy"] = randn(rows, d).to(dtype)
        return state
    state["weight"] = 1.0 + 0.2 * randn(d)
    if case["op"] == "rms_backward":
        state["dy"] = randn(rows, d).to(dtype)
        state["dh"] = randn(rows, d).to(dtype) if case["residual"] else None
        h = state["x"].float()
        state["rstd"] = 1.0 / torch.sqrt(h.square().mean(dim=1) + EPS)
    return state


# ------------------------------------------------------------------ plain forms
def philox(counters, rng):
    """Philox4x32-10 on 64-bit counters: four words each, as int64 (n, 4)."""
    seed, offset = rng[0], rng[1]
    a, b = counters & M32, (counters >> 32) & M32
    c, d = (offset & M32).expand_as(a), ((offset >> 32) & M32).expand_as(a)
    k0, k1 = seed & M32, (seed >> 32) & M32
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57  # modulo 2^64
        a, b, c, d = (((q >> 32) & M32) ^ b ^ k0, q & M32, ((p >> 32) & M32) ^ d ^ k1, p & M32)
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return torch.stack((a, b, c, d), dim=1)


def plain_dropout(x, p, rng):
    """fp32 values of x, a share p of them dropped and the others scaled."""
    x = x.float()
    if p == 0.0:
        return x
    threshold, n = round(p * 65536), x.numel()
    words = philox(torch.arange((n + 7) // 8, device=x.device), rng)
    numbers = torch.stack((words & 0xFFFF, words >> 16), dim=2).reshape(-1)[:n].view(x.shape)
    return torch.where(numbers < threshold, torch.zeros_like(x), x * (65536 / (65536 - threshold)))


def plain_sum(s):
    """(h in the stream's type, h in fp32)"""
    case, x = s["case"], s["x"]
    h = plain_dropout(x, case["p"], s["rng"])
    if case["residual"]:
        h = h + s["residual"].float()
    h = h.to(x.dtype)
    return h, h.float()


def plain_rms_forward(s):
    h, v = plain_sum(s)
    rstd = 1.0 / torch.sqrt(v.square().mean(dim=1) + EPS)
    return [(v * rstd[:, None] * s["weight"]).to(h.dtype), h, rstd]


def plain_rms_backward(s):
    case, h, r = s["case"], s["x"].float(), s["rstd"][:, None]
    dy = s["dy"].float()
    g = dy * s["weight"]
    dz = r * (g - h * r * r * (g * h).mean(dim=1, keepdim=True))
    if case["residual"]:
        dz = dz + s["dh"].float()
    dresidual = dz.to(s["x"].dtype)
    dx = plain_dropout(dz, case["p"], s["rng"]).to(s["x"].dtype)
    return [dx, dresidual, (dy * h * r).sum(dim=0)]


def plain_rms_quantize(s):
    h, v = plain_sum(s)
    rows, d = v.shape
    z = v * (1.0 / torch.sqrt(v.square().mean(dim=1, keepdim=True) + EPS)) * s["weight"]
    block = s["case"]["block"] or d
    blocks = -(-d // block)
    padded = torch.zeros(rows, blocks * block, device=z.device)
    padded[:, :d] = z
    padded = padded.view(rows, blocks, block)
    scale = padded.abs().amax(dim=2) / E4M3_MOST
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    q = (padded / scale[:, :, None]).reshape(rows, -1)[:, :d]
    return [q.to(torch.float8_e4m3fn), scale, h]


def plain_drop_train(s):
    case, x = s["case"], s["x"]
    y = plain_dropout(x, case["p"], s["rng"])
    if case["residual"]:
        y = y + s["residual"].float()
    return [y.to(x.dtype), plain_dropout(s["dy"], case["p"], s["rng"]).to(x.dtype)]


def plain_logits(s):
    """fp32 logits of the tokens that have a target; those tokens, and their targets"""
    at = torch.nonzero(s["targets"] != IGNORE)[:, 0]
    hidden, weight = s["hidden"].detach()[at].float(), s["weight"].detach().float()
    return hidden @ weight.t(), hidden, weight, at, s["targets"][at]


def plain_loss_eval(s):
    logits, _, _, at, targets = plain_logits(s)
    top = logits.amax(dim=1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(logits - top).sum(dim=1))
    out = torch.zeros(s["targets"].numel(), device=logits.device)
    out[at] = lse - logits[torch.arange(at.numel(), device=at.device), targets]
    return out


def plain_loss_train(s):
    logits, hidden, weight, at, targets = plain_logits(s)
    each = torch.arange(at.numel(), device=at.device)
    top = logits.amax(dim=1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(dim=1, keepdim=True)
    mean = (top[:, 0] + torch.log(total[:, 0]) - logits[each, targets]).mean()
    grad = e / total
    grad[each, targets] -= 1.0
    grad *= s["scale"] / at.numel()
    dhidden = torch.zeros_like(s["hidden"])
    dhidden[at] = (grad @ weight).to(dhidden.dtype)
    return [mean, dhidden, (grad.t() @ hidden).to(s["weight"].dtype)]


# ------------------------------------------------------------------ one pass
def run_own(s):
    from paper_2306_06098_b200 import binding, loss as losses
    case = s["case"]
    op = case["op"]
    if op == "rms_forward":
        return list(binding.rms_norm_forward(s["x"], s["weight"], EPS, s["residual"], case["p"],
                                             s["rng"]))
    if op == "rms_backward":
        return list(binding.rms_norm_backward(s["dy"], s["x"], s["rstd"], s["weight"], s["dh"],
                                              case["p"], s["rng"]))
    if op == "rms_quantize":
        return list(binding.rms_norm_quantize(s["x"], s["weight"], EPS, s["residual"],
                                              case["block"], "e4m3"))
    if op == "dropout":
        return [binding.dropout(s["x"], case["p"], s["rng"], s["residual"]),
                binding.dropout(s["dy"], case["p"], s["rng"])]
    if op == "loss_eval":
        return losses.linear_cross_entropy(s["hidden"], s["weight"], s["targets"], IGNORE, "none")
    value = losses.linear_cross_entropy(s["hidden"], s["weight"], s["targets"], IGNORE, "mean")
    grads = torch.autograd.grad(value, (s["hidden"], s["weight"]), s["scale"])
    return [value.detach(), *grads]


PLAIN = {"rms_forward": plain_rms_forward, "rms_backward": plain_rms_backward,
         "rms_quantize": plain_rms_quantize, "dropout": plain_drop_train,
         "loss_eval": plain_loss_eval, "loss_train": plain_loss_train}


def run(state):
    return run_own(state) if own else PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ floors and 64 bits
def work(case):
    b = BYTES[case["dtype"]]
    if case["op"].startswith("loss"):
        n, d, v = case["n"], case["d"], case["v"]
        used = max(1, round(n * case["labelled"]))  # tokens that have a target
        if case["op"] == "loss_eval":
            return {"bytes": b * d * (used + v) + 12 * n, "flops": 2 * used * v * d}
        return {"bytes": b * d * (used + n + 2 * v) + 8 * n + 4, "flops": 6 * used * v * d}
    rows, d = case["rows"], case["d"]
    size = rows * d
    if case["op"] == "dropout":
        return {"bytes": b * size * (5 if case["residual"] else 4), "flops": 2 * size}
    streams = 2 if case["residual"] else 1
    if case["op"] == "rms_forward":
        summed = case["residual"] or case["p"] > 0
        return {"bytes": b * size * (streams + 1 + summed) + 4 * (rows + d), "flops": 5 * size}
    if case["op"] == "rms_quantize":
        blocks = -(-d // (case["block"] or d))
        return {"bytes": b * size * (2 * streams - 1) + size + 4 * (rows * blocks + d),
                "flops": 7 * size}
    return {"bytes": b * size * (streams + 2 + (case["p"] > 0)) + 4 * rows + 8 * d,
            "flops": 10 * size}


def exact_kept(shape, p, rng):
    """Which elements stay: Philox4x32-10 again, its products put together from 16-bit halves."""
    def product(x, m):  # (high, low) words of x m
        lo, hi = x * (m & 0xFFFF), x * (m >> 16)
        mid = (lo >> 16) + (hi & 0xFFFF)
        return (hi >> 16) + (mid >> 16), ((mid & 0xFFFF) << 16) | (lo & 0xFFFF)

    seed, offset = (int(t) & 0xFFFFFFFFFFFFFFFF for t in rng.tolist())
    count = math.prod(shape)
    at = torch.arange(-(-count // 8), device="cuda")
    word = [at % (1 << 32), at // (1 << 32), torch.full_like(at, offset % (1 << 32)),
            torch.full_like(at, offset // (1 << 32))]
    for turn in range(10):
        key = [(seed % (1 << 32) + turn * 0x9E3779B9) % (1 << 32),
               (seed // (1 << 32) + turn * 0xBB67AE85) % (1 << 32)]
        h0, l0 = product(word[0], 0xD2511F53)
        h1, l1 = product(word[2], 0xCD9E8D57)
        word = [h1 ^ word[1] ^ key[0], l1, h0 ^ word[3] ^ key[1], l0]
    numbers = torch.empty(at.numel(), 8, dtype=torch.int64, device="cuda")
    for j in range(8):
        numbers[:, j] = word[j // 2] // (1 << 16 * (j % 2)) % (1 << 16)
    return (numbers.view(-1)[:count] >= round(p * 65536)).view(shape)


def exact_dropout(x, case, rng):
    if case["p"] == 0.0:
        return x
    return x * exact_kept(x.shape, case["p"], rng) / (1.0 - round(case["p"] * 65536) / 65536.0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("loss"):
        used = s["targets"] >= 0
        hidden = s["hidden"].detach()[used].double()
        weight = s["weight"].detach().double()
        train = case["op"] == "loss_train"
        hidden.requires_grad_(train)
        weight.requires_grad_(train)
        logits = torch.nn.functional.linear(hidden, weight)
        each = torch.logsumexp(logits, 1) - logits.gather(1, s["targets"][used][:, None])[:, 0]
        if not train:
            out = torch.zeros(case["n"], dtype=torch.float64, device="cuda")
            out[used] = each
            return out
        value = each.sum() / each.numel()
        grads = torch.autograd.grad(value, (hidden, weight), s["scale"].double())
        full = torch.zeros(case["n"], case["d"], dtype=torch.float64, device="cuda")
        full[used] = grads[0]
        return [value.detach(), full, grads[1]]
    x, rng = s["x"].double(), s["rng"]
    if case["op"] == "dropout":
        y = exact_dropout(x, case, rng)
        if case["residual"]:
            y = y + s["residual"]
        return [y, exact_dropout(s["dy"].double(), case, rng)]
    weight = s["weight"].double()
    if case["op"] == "rms_backward":
        # the definition, differentiated by autograd
        x.requires_grad_(True)
        weight.requires_grad_(True)
        y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * weight
        dz, dweight = torch.autograd.grad(y, (x, weight), s["dy"].double())
        if case["residual"]:
            dz = dz + s["dh"]
        return [exact_dropout(dz, case, rng), dz, dweight]
    h = exact_dropout(x, case, rng)
    if case["residual"]:
        h = h + s["residual"]
    h = h.to(s["x"].dtype).double()  # the sum is kept in the stream's type
    rstd = torch.rsqrt((h * h).mean(1) + EPS)
    y = h * rstd[:, None] * weight
    if case["op"] == "rms_forward":
        return [y, h, rstd]
    # an element's 8-bit value hangs on which side of a border it falls
    tops = [part.abs().amax(1) for part in y.split(case["block"] or case["d"], dim=1)]
    return [None, torch.stack(tops, 1) / E4M3_MOST, h]
