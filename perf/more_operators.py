"""What a data-parallel training step of a token model runs beside the collective, its 4-bit layers and AdamW, as measurable cases: one pass of each through the public calls.

`op` names what a case runs:

  norm        zc_layer_norm, and with `train` zc_layer_norm_backward behind it: the gradients of input, weight and bias
  embed       zc_embedding: rows of a table, times a factor
  embed_grad  zc_embedding_backward: the table's gradient, rows summed by token
  muon        zc_muon: one step over matrices of one shape, their momentum orthogonalised by Newton-Schulz products

Sizes are generic ones of layers and vocabularies (powers of two between 2^8 and 2^14, and odd ones beside them).
"""
import math

import torch

own = False
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "": 0}


def listed():
    return [
        # serving, one token's activations
        dict(name="norm_token", op="norm", rows=1, cols=4096, x="bf16", y="bf16", w="bf16", train=False, add=False),
        # a small odd layer in 32 bits, forward and backward
        dict(name="norm_odd", op="norm", rows=333, cols=1001, x="f32", y="f32", w="f32", train=True, add=False),
        # wide rows, ordinary batch
        dict(name="norm_wide", op="norm", rows=512, cols=16384, x="f16", y="f16", w="f32", train=True, add=False),
        # a training step: a residual stream in 32 bits, layers in 16; the gradient joins the stream's
        dict(name="norm_train", op="norm", rows=16384, cols=4096, x="f32", y="bf16", w="f32", train=True, add=True),
        # serving, a batch of 24 sequences, a token each
        dict(name="embed_tokens", op="embed", n=24, vocab=50021, cols=4096, table="bf16", y="bf16", pad=0.0, bits=64),
        # long prompts; weights in 32 bits
        dict(name="embed_prompt", op="embed", n=16384, vocab=50021, cols=2048, table="f32", y="bf16", pad=0.1, bits=32),
        # a small odd table whose gradient is gathered over micro-batches
        dict(name="embed_grad_odd", op="embed_grad", n=5117, vocab=1009, cols=777, y="f32", grad="f32", pad=0.0, bits=64, add=True),
        # a training batch with padding behind its sequences; the whole gradient for the collective
        dict(name="embed_grad_batch", op="embed_grad", n=32768, vocab=50021, cols=2048, y="bf16", grad="f32", pad=0.1, bits=64, add=False),
        # a small model's matrices
        dict(name="muon_small", op="muon", count=24, rows=256, cols=512, params="bf16", grads="bf16", copies="", wide=False, nesterov=True, clip=False),
        # tall odd matrices in 32 bits
        dict(name="muon_odd", op="muon", count=3, rows=1531, cols=333, params="f32", grads="f32", copies="", wide=True, nesterov=False, clip=False),
        # mixed precision: weights in 32 bits with copies in 16, a clip's factor
        dict(name="muon_mixed", op="muon", count=6, rows=1024, cols=4096, params="f32", grads="bf16", copies="bf16", wide=True, nesterov=True, clip=True),
        # a large matrix in 16 bits
        dict(name="muon_large", op="muon", count=1, rows=4096, cols=8192, params="bf16", grads="bf16", copies="", wide=False, nesterov=True, clip=False),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "embed", "embed_grad", "embed_grad", "muon", "muon"])
    if op == "norm":
        cols = _log(rng, 3, 20000)
        train = rng.random() < 0.7
        return dict(op=op, rows=_log(rng, 1, min(40000, (1 << 26) // cols)), cols=cols, x=rng.choice(["f32", "bf16", "f16"]), y=rng.choice(["bf16", "f32"]),
                    w=rng.choice(["f32", "bf16"]), train=train, add=train and rng.random() < 0.5)
    if op == "embed":
        cols = _log(rng, 8, 8192)
        return dict(op=op, n=_log(rng, 1, min(65536, (1 << 25) // cols)), vocab=_log(rng, 50, min(200000, (1 << 27) // cols)), cols=cols, table=rng.choice(["f32", "bf16"]),
                    y=rng.choice(["bf16", "f32", "f16"]), pad=rng.choice([0.0, 0.2]), bits=rng.choice([32, 64]))
    if op == "embed_grad":
        cols = _log(rng, 8, 8192)
        return dict(op=op, n=_log(rng, 1, min(65536, (1 << 26) // cols)), vocab=_log(rng, 50, min(200000, (1 << 26) // cols)), cols=cols, y=rng.choice(["f32", "bf16"]),
                    grad=rng.choice(["f32", "f32", "bf16"]), pad=rng.choice([0.0, 0.5]), bits=rng.choice([32, 64]), add=rng.random() < 0.5)
    rows, cols = _log(rng, 17, 4096), _log(rng, 17, 4096)
    wide = rng.random() < 0.5
    return dict(op=op, count=_log(rng, 1, max(1, min(30, (1 << 24) // (rows * cols)))), rows=rows, cols=cols, params="f32" if wide else "bf16", grads=rng.choice(["f32", "bf16"]),
                copies=rng.choice(["", "bf16"]), wide=wide, nesterov=rng.random() < 0.5, clip=rng.random() < 0.5)


# ---- the inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(shape, g, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _activations(rows, cols, g, dtype):
    """Rows of different magnitude and mean, and a few columns that stand out."""
    x = _normal((rows, cols), g)
    x *= 1 + 15 * (torch.rand((1, cols), generator=g, device=DEV) < 0.01)
    x += 0.5 * _normal((rows, 1), g)
    x *= torch.exp(0.5 * _normal((rows, 1), g))
    return x.to(dtype)


def _tokens(case, g):
    """Token k about as often as 1 / (k + 1) says, as in text; padding (-1) behind the sequences."""
    n, vocab = case["n"], case["vocab"]
    t = torch.exp(torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * math.log(vocab + 1)).long() - 1
    t.clamp_(0, vocab - 1)
    if case["pad"]:
        length = 256                                       # of a sequence, the last share of which is padding, more or less
        ends = length * (1 - 2 * case["pad"] * torch.rand(-(-n // length), generator=g, device=DEV))
        t[torch.arange(n, device=DEV) % length >= ends.repeat_interleave(length)[:n]] = -1
    return t.to(torch.int32 if case["bits"] == 32 else torch.int64)


def _gradient_like(shape, g):
    """A few strong directions over weaker ones, as gradients of matrices have them."""
    count, rows, cols = shape
    strong = _normal((count, rows, 8), g) @ _normal((count, 8, cols), g)
    return (strong + _normal(shape, g)).mul_(1e-3)


def _padded(n):
    return -(-n // 32) * 32


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        y = TYPES[case["y"]]
        s = dict(case=case, x=_activations(rows, cols, g, TYPES[case["x"]]), w=(1 + 0.2 * _normal((cols,), g)).to(TYPES[case["w"]]), b=(0.1 * _normal((cols,), g)).to(TYPES[case["w"]]),
                 out=torch.empty((rows, cols), dtype=y, device=DEV), stats=torch.empty((2, rows), device=DEV))
        if case["train"]:
            s.update(dy=_normal((rows, cols), g, y), dx=_normal((rows, cols), g, TYPES[case["x"]]), dw=torch.empty(cols, device=DEV), db=torch.empty(cols, device=DEV),
                     ws=torch.empty(65536 + 16384 * (cols + 64), dtype=torch.uint8, device=DEV))
        return s
    if case["op"] == "embed":
        return dict(case=case, tokens=_tokens(case, g), table=_normal((case["vocab"], case["cols"]), g, TYPES[case["table"]]),
                    out=torch.empty((case["n"], case["cols"]), dtype=TYPES[case["y"]], device=DEV))
    if case["op"] == "embed_grad":
        n, vocab, cols = case["n"], case["vocab"], case["cols"]
        return dict(case=case, tokens=_tokens(case, g), dy=_normal((n, cols), g, TYPES[case["y"]]), grad=_normal((vocab, cols), g, TYPES[case["grad"]]),
                    ws=torch.empty((1 << 20) + 64 * n + 16 * vocab + (n // 8 + 2) * 8 * (cols + 64), dtype=torch.uint8, device=DEV))
    count, rows, cols = case["count"], case["rows"], case["cols"]
    params = _normal((count, rows, cols), g).mul_(0.02).to(TYPES[case["params"]])
    grads = _gradient_like((count, rows, cols), g).to(TYPES[case["grads"]])
    copies = params.to(TYPES[case["copies"]]) if case["copies"] else None
    state = torch.zeros((count, _padded(rows * cols)), device=DEV)
    state[:, :rows * cols] = _gradient_like((count, rows, cols), g).view(count, -1)
    return dict(case=case, all_params=params, all_copies=copies, all_grads=grads, params=list(params), grads=list(grads), copies=list(copies) if copies is not None else None,
                state=state, ws=torch.empty((1 << 20) + 24 * count * (rows + 256) * (cols + 256), dtype=torch.uint8, device=DEV),
                grad_scale=torch.full((1,), 0.37 + 0.01 * (seed % 7), device=DEV) if case["clip"] else None)


# ---- one pass

EPS = 1e-5
FACTOR = 1.7
LR, MOMENTUM, DECAY, ITERATIONS = 0.1, 0.95, 0.1, 5
A, B, C, LEAST = 3.4445, -4.7750, 2.0315, 1e-7


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "embed": _own_embed, "embed_grad": _own_embed_grad, "muon": _own_muon}[op](state)
    return {"norm": _plain_norm, "embed": _plain_embed, "embed_grad": _plain_embed_grad, "muon": _plain_muon}[op](state)


def _norm_outputs(s):
    return {k: s[k] for k in (("out", "stats", "dx", "dw", "db") if s["case"]["train"] else ("out", "stats"))}


def _muon_outputs(s):
    return dict(params=s["all_params"], copies=s["all_copies"], momentum=s["state"])


# ---- by the framework's calls

def _check(status):
    if status:
        import paper_2502_18554_amd as zc
        raise zc.ZcError(status, "more_operators")


def _own_norm(s):
    import paper_2502_18554_amd as zc
    _check(zc.zc_layer_norm(s["x"], s["w"], s["b"], s["out"], s["stats"], eps=EPS))
    if s["case"]["train"]:
        _check(zc.zc_layer_norm_backward(s["dy"], s["x"], s["stats"], s["w"], s["dx"], s["dw"], s["db"], s["ws"], add=s["case"]["add"]))
    return _norm_outputs(s)


def _own_embed(s):
    import paper_2502_18554_amd as zc
    _check(zc.zc_embedding(s["table"], s["tokens"], s["out"], scale=FACTOR))
    return s["out"]


def _own_embed_grad(s):
    import paper_2502_18554_amd as zc
    _check(zc.zc_embedding_backward(s["dy"], s["tokens"], s["grad"], s["ws"], scale=FACTOR, add=s["case"]["add"]))
    return s["grad"]


def _own_muon(s):
    import paper_2502_18554_amd as zc
    _check(zc.zc_muon(s["params"], s["grads"], s["state"], s["ws"], LR, momentum=MOMENTUM, weight_decay=DECAY, iterations=ITERATIONS, nesterov=s["case"]["nesterov"],
                      wide=s["case"]["wide"], d_copies=s["copies"], d_grad_scale=s["grad_scale"]))
    return _muon_outputs(s)


# ---- in plain form

def _plain_norm(s):
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    mean = x.mean(dim=1, keepdim=True)
    centred = x - mean
    rstd = 1 / torch.sqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
    normed = centred * rstd
    s["out"].copy_(normed * w + b)
    s["stats"].copy_(torch.cat([mean, rstd], dim=1).t())
    if s["case"]["train"]:
        dy = s["dy"].float()
        h = dy * w
        dx = rstd * (h - h.mean(dim=1, keepdim=True) - normed * (h * normed).mean(dim=1, keepdim=True))
        s["dx"].copy_(dx + s["dx"] if s["case"]["add"] else dx)
        s["dw"].copy_((dy * normed).sum(dim=0))
        s["db"].copy_(dy.sum(dim=0))
    return _norm_outputs(s)


def _plain_embed(s):
    t = s["tokens"].long()
    there = (t >= 0) & (t < s["case"]["vocab"])
    rows = s["table"][torch.where(there, t, 0)].float() * FACTOR
    s["out"].copy_(torch.where(there.unsqueeze(1), rows, 0))
    return s["out"]


def _plain_embed_grad(s):
    t, vocab = s["tokens"].long(), s["case"]["vocab"]
    there = (t >= 0) & (t < vocab)
    sums = torch.zeros((vocab + 1, s["case"]["cols"]), device=DEV)            # (the last row: what belongs to no token)
    sums.index_add_(0, torch.where(there, t, vocab), s["dy"].float())
    sums = sums[:vocab] * FACTOR
    s["grad"].copy_(sums + s["grad"] if s["case"]["add"] else sums)
    return s["grad"]


def _plain_muon(s):
    case = s["case"]
    count, rows, cols = case["count"], case["rows"], case["cols"]
    g = torch.stack(s["grads"]).float()
    if s["grad_scale"] is not None:
        g = g * s["grad_scale"]
    m = s["state"][:, :rows * cols].view(count, rows, cols) * MOMENTUM + g * (1 - MOMENTUM)
    x = m * MOMENTUM + g * (1 - MOMENTUM) if case["nesterov"] else m
    x = x / x.double().square().sum(dim=(1, 2), keepdim=True).sqrt().clamp(min=LEAST).float()
    if rows > cols:
        x = x.transpose(1, 2).contiguous()
    for _ in range(ITERATIONS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = x * A + torch.bmm(gram * B + torch.bmm(gram, gram) * C, x)
    if rows > cols:
        x = x.transpose(1, 2)
    p = torch.stack(s["params"]).float() * (1 - LR * DECAY) - x * (LR * math.sqrt(max(1, rows / cols)))
    if s["grad_scale"] is not None:                        # (a factor that is not finite: nothing happens)
        fine = torch.isfinite(s["grad_scale"])
        p = torch.where(fine, p, s["all_params"])
        m = torch.where(fine, m, s["state"][:, :rows * cols].view(count, rows, cols))
    s["state"][:, :rows * cols] = m.view(count, -1)
    s["all_params"].copy_(p)
    if s["all_copies"] is not None:
        s["all_copies"].copy_(p)
    return _muon_outputs(s)


# ---- what one pass cannot do without

def _distinct(n, vocab):
    """How many different tokens a call meets, on average."""
    k = torch.arange(vocab, dtype=torch.float64)
    share = torch.log((k + 2) / (k + 1)) / math.log(vocab + 1)
    return float((1 - torch.exp(n * torch.log1p(-share.clamp(max=1 - 1e-12)))).sum())


def work(case):
    if case["op"] == "norm":
        values, x, y = case["rows"] * case["cols"], BYTES[case["x"]], BYTES[case["y"]]
        bytes_, flops = values * (x + y) + 8 * case["rows"] + 2 * case["cols"] * BYTES[case["w"]], 8 * values
        if case["train"]:
            bytes_ += values * (x + y + x * (2 if case["add"] else 1)) + 8 * case["rows"] + case["cols"] * (8 + BYTES[case["w"]])
            flops += 16 * values
        return dict(bytes=bytes_, flops=flops)
    if case["op"] == "muon":
        values, least, most = case["count"] * case["rows"] * case["cols"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # A and A A are symmetric: half of each is a product's worth of the other half
        return dict(bytes=values * (2 * BYTES[case["params"]] + BYTES[case["grads"]] + BYTES[case["copies"]] + 8), flops=case["count"] * ITERATIONS * (3 * least * least * most + least ** 3))
    there = case["n"] * (1 - case["pad"])
    rows = _distinct(int(there), case["vocab"])
    if case["op"] == "embed":
        return dict(bytes=case["cols"] * (rows * BYTES[case["table"]] + case["n"] * BYTES[case["y"]]) + case["n"] * case["bits"] // 8, flops=case["n"] * case["cols"])
    grad = BYTES[case["grad"]]
    return dict(bytes=case["cols"] * (there * BYTES[case["y"]] + (2 * rows if case["add"] else case["vocab"]) * grad) + case["n"] * case["bits"] // 8, flops=there * case["cols"])


# ---- from the definitions, in 64 bits

def _exact_norm(s):
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    dev = torch.sqrt(var + EPS)
    hat = (x - mean) / dev
    out = dict(out=torch.addcmul(b, hat, w), stats=torch.stack([mean[:, 0], 1 / dev[:, 0]]))
    if s["case"]["train"]:
        # y = hat w + b, hat = P x / dev with P the projection off the constants: the gradient goes back through both
        dy = s["dy"].double()
        dhat = dy * w
        along = (dhat * hat).sum(dim=1, keepdim=True) / x.shape[1]
        dx = (dhat - along * hat) / dev
        dx -= dhat.sum(dim=1, keepdim=True) / x.shape[1] / dev
        out.update(dx=dx + s["dx"].double() if s["case"]["add"] else dx, dw=torch.einsum("rc,rc->c", dy, hat), db=dy.sum(dim=0))
    return out


def _exact_embed(s):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    at = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < s["case"]["vocab"]))[:, 0]
    out[at] = s["table"].index_select(0, s["tokens"].index_select(0, at).long()).double().mul(FACTOR)
    return out


def _exact_embed_grad(s):
    at = torch.nonzero((s["tokens"] >= 0) & (s["tokens"] < s["case"]["vocab"]))[:, 0]
    t = s["tokens"][at].long()
    order = torch.argsort(t, stable=True)
    found, counts = torch.unique_consecutive(t[order], return_counts=True)
    total = s["grad"].double() if s["case"]["add"] else torch.zeros(s["grad"].shape, dtype=torch.float64, device=DEV)
    if at.numel():
        sums = torch.segment_reduce(s["dy"][at[order]].double(), "sum", lengths=counts, axis=0)
        total[found] += FACTOR * sums
    return total


def _exact_muon(s):
    case = s["case"]
    size = case["rows"] * case["cols"]
    scale = float(s["grad_scale"].double()) if s["grad_scale"] is not None else 1.0
    params, momentum = s["all_params"].double(), s["state"].double()
    for i, g in enumerate(s["grads"]):
        g = g.double() * scale
        m = momentum[i, :size].view(g.shape)
        m += (g - m) * (1 - MOMENTUM)
        u = torch.lerp(g, m, MOMENTUM) if case["nesterov"] else m.clone()
        u /= max(float(torch.linalg.vector_norm(u)), LEAST)
        turned = u.shape[0] > u.shape[1]
        u = u.t().contiguous() if turned else u
        for _ in range(ITERATIONS):
            square = u @ u.t().contiguous()
            once = square @ u
            u = A * u + B * once + C * (square @ once)
        step = u.t() if turned else u
        params[i] = params[i] * (1 - LR * DECAY) - LR * max(1.0, case["rows"] / case["cols"]) ** 0.5 * step
    return dict(params=params, copies=params if case["copies"] else None, momentum=momentum)


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "embed": _exact_embed, "embed_grad": _exact_embed_grad, "muon": _exact_muon}[case["op"]](s)
