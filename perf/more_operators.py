"""The two ends of a training step of a network such as a prior head, as cases that can be timed: the loss over what it predicts and the update of its weights.

  loss      softmax cross entropy of rows of a network's last stream `u` [rows, cols] against a table of classes `weight` [classes, cols]
            (values of a latent, tokens): loss = lse - logit of the target, lse the logarithm of the sum of the exponentials
  loss_bwd  its gradients for `u` and `weight`, out of lse; the gradient of lse itself (a penalty on it) may come in too
  orth      a gradient [rows, cols], or several, made nearly orthogonal by five steps of an odd polynomial (Newton-Schulz products)
  muon      the step of an optimiser around that: momentum, orthogonalising, decay, and the weights changed in place

`own` false computes the plain form in elementary 32-bit operations, `own` true calls the package.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
STEPS, QUINTIC, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
RATE, BETA, DECAY = 0.02, 0.95, 0.1
LARGEST_FLOPS = 6.6e12    # of one pass
LARGEST_LOGITS = 1 << 29  # rows x classes
LARGEST_TABLE = 1 << 28   # elements of one matrix


def listed():
    def loss(name, op, rows, classes, cols, type, dead=0.0, **more):
        return dict(name=name, op=op, rows=rows, classes=classes, cols=cols, type=type, dead=dead, **more)

    def update(name, op, count, rows, cols, **more):
        return dict(name=name, op=op, count=count, rows=rows, cols=cols, **more)
    return [
        # one position scored through a trained network: the whole table is read for it, latency and bandwidth count
        loss("loss_one_row", "loss", 1, 32768, 1024, "bf16"),
        # ragged sequences with padding, a width and a number of classes that are multiples of nothing, 32 bits
        loss("loss_ragged", "loss", 1023, 10007, 1111, "f32", dead=0.1),
        # validation of a large batch over a large table
        loss("loss_wide", "loss", 8192, 65536, 4096, "bf16"),
        # a prior head of the 64x64 flow, level 1: 128 images x 32 x 32 positions, width 512, a latent's values as classes
        loss("loss_bwd_head", "loss_bwd", 131072, 256, 512, "bf16", penalty=False),
        # padding, half precision, odd sizes, with a penalty on lse
        loss("loss_bwd_ragged", "loss_bwd", 1000, 5003, 520, "f16", dead=0.2, penalty=True),
        # the largest ordinary training step
        loss("loss_bwd_wide", "loss_bwd", 8192, 32768, 4096, "bf16", penalty=True),
        # the weight of one layer of the paper's 128 wide networks
        update("orth_small", "orth", 1, 128, 128, type="bf16", out="bf16"),
        # an odd, tall 32-bit gradient, result in 32 bits
        update("orth_ragged", "orth", 1, 1111, 520, type="f32", out="f32"),
        # a large square projection
        update("orth_wide", "orth", 1, 4096, 4096, type="f32", out="bf16"),
        # the projections into the hidden layers of a prior of width 512, eight blocks, together
        update("muon_blocks", "muon", 8, 2048, 512, type="f32", grad="f32"),
        # three odd, tall layers in half precision
        update("muon_ragged", "muon", 3, 777, 333, type="f16", grad="f16"),
        # a large projection of a network kept in 16 bits
        update("muon_wide", "muon", 1, 4096, 8192, type="bf16", grad="bf16"),
    ]


def _log(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _cols(rng, low, high):
    c = _log(rng, low, high)
    return c if rng.random() < 0.5 or c < 128 else c // 64 * 64


def draw(rng):
    op = rng.choice(("loss", "loss_bwd", "loss_bwd", "orth", "muon"))
    kind = rng.choice(("bf16", "bf16", "bf16", "f16", "f32"))
    top = LARGEST_FLOPS / (4 if kind == "f32" else 1)
    if op in ("loss", "loss_bwd"):
        cols, classes = _cols(rng, 8, 8192), _log(rng, 2, 131072)
        classes = min(classes, LARGEST_TABLE // cols)
        most = min(131072, LARGEST_LOGITS // classes, LARGEST_TABLE // cols, int(top / 6 / (cols * classes)))
        rows = _log(rng, 1, max(1, most))
        case = dict(op=op, rows=rows, classes=classes, cols=cols, type=kind, dead=rng.choice((0.0, 0.0, 0.15)))
        return dict(case, penalty=rng.random() < 0.5) if op == "loss_bwd" else case
    rows, cols, count = _cols(rng, 8, 8192), _cols(rng, 8, 8192), rng.choice((1, 1, 2, 3, 8))
    while count > 1 and (count * rows * cols > LARGEST_TABLE // 4 or _products(count, rows, cols) > top / 2):
        count -= 1
    while _products(count, rows, cols) > top / 2:
        rows, cols = rows // 2, cols // 2
    if op == "muon":
        return dict(op=op, count=count, rows=rows, cols=cols, type=kind, grad=rng.choice((kind, "f32")))
    return dict(op=op, count=count, rows=rows, cols=cols, type=rng.choice((kind, "f32")), out=kind)


# ---- inputs ----

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def spread(n, by):  # per-channel magnitudes: a few channels carry far more than the others
        return torch.exp(by * normal(n))

    s = dict(case)
    if case["op"] in ("loss", "loss_bwd"):
        rows, classes, cols, kind = case["rows"], case["classes"], case["cols"], TYPES[case["type"]]
        weight = normal(classes, cols) * spread(cols, 0.4) / math.sqrt(cols)
        # a few classes are most of the targets, and a trained network leans towards the right one
        s["target"] = (classes * torch.rand(rows, generator=gen, device="cuda") ** 3).long().clamp_(0, classes - 1)
        u = normal(rows, cols)
        for at in range(0, rows, 16384):
            u[at:at + 16384] += 3.0 * weight[s["target"][at:at + 16384]]
        s["live"] = None
        if case["dead"]:  # what stands in padded rows is anything
            s["live"] = torch.rand(rows, generator=gen, device="cuda") >= case["dead"]
            s["live"][0] = True
            u[~s["live"]] = float("nan")
            s["target"][~s["live"]] = -1
        s["u"], s["weight"] = u.to(kind), weight.to(kind)
        if case["op"] == "loss_bwd":
            s["lse"] = _plain_loss(s)["lse"]  # what the forward pass left
            n = rows if s["live"] is None else int(s["live"].sum())
            s["dloss"] = torch.full((rows,), 1.0 / n, device="cuda")
            s["dlse"] = 2e-3 * s["lse"] / n if case["penalty"] else None
        return s
    count, rows, cols = case["count"], case["rows"], case["cols"]
    low = min(rows, cols) // 8 + 1  # a few directions carry most of a gradient, the rest is noise
    g = [torch.matmul(normal(rows, low) * torch.arange(1, low + 1, device="cuda") ** -0.5, normal(low, cols)) / math.sqrt(low) + 0.5 * normal(rows, cols)
         for _ in range(count)]
    g = [1e-3 * x * spread(cols, 0.4) for x in g]
    if case["op"] == "orth":
        s["g"] = torch.stack(g).to(TYPES[case["type"]]) if count > 1 else g[0].to(TYPES[case["type"]])
    else:
        s["grads"] = [x.to(TYPES[case["grad"]]) for x in g]
        s["momenta"] = [3e-3 * normal(rows, cols) for _ in range(count)]
        s["weights"] = [(normal(rows, cols) / math.sqrt(cols)).to(TYPES[case["type"]]) for _ in range(count)]
    return s


# ---- the plain form ----

def _plain_logits(s):
    u = s["u"].float()
    if s["live"] is not None:
        u = torch.where(s["live"][:, None], u, torch.zeros_like(u))
    return u, torch.matmul(u, s["weight"].float().t())


def _picked(s):
    """The target of each row, 0 in padded ones."""
    return s["target"].clamp_min(0)[:, None]


def _only(live, x):
    return x if live is None else torch.where(live, x, torch.zeros_like(x))


def _plain_loss(s):
    logits = _plain_logits(s)[1]
    top = logits.amax(1)
    picked = logits.gather(1, _picked(s))[:, 0]
    lse = top + torch.log(logits.sub_(top[:, None]).exp_().sum(1))
    return {"loss": _only(s["live"], lse - picked), "lse": _only(s["live"], lse)}


def _plain_loss_bwd(s):
    u, g = _plain_logits(s)
    dloss = _only(s["live"], s["dloss"])
    both = dloss if s["dlse"] is None else dloss + _only(s["live"], s["dlse"])
    g = g.sub_(s["lse"][:, None]).exp_().mul_(both[:, None])
    g.scatter_add_(1, _picked(s), -dloss[:, None])
    return {"du": torch.matmul(g, s["weight"].float()).to(s["u"].dtype), "dweight": torch.matmul(g.t(), u).to(s["weight"].dtype)}


def _plain_orth(g):
    """[count, rows, cols], 32 bits."""
    a, b, c = QUINTIC
    x = (g / (g.double().square().sum((1, 2), keepdim=True).sqrt() + EPS)).float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    for _ in range(STEPS):
        p = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * p + c * torch.matmul(p, p), x)
    return x.transpose(1, 2).contiguous() if tall else x


def _scale(s):
    return math.sqrt(max(1.0, s["rows"] / s["cols"]))


def _plain_muon(s):
    g, m = torch.stack(s["grads"]).float(), torch.stack(s["momenta"])
    m = BETA * m + g
    step = _plain_orth(g + BETA * m)
    w = (1 - RATE * DECAY) * torch.stack(s["weights"]).float() - RATE * _scale(s) * step
    for i in range(s["count"]):
        s["momenta"][i].copy_(m[i])
        s["weights"][i].copy_(w[i])
    return {"weights": s["weights"], "momenta": s["momenta"]}


# ---- the package's calls ----

def _own_loss(s):
    import paper_2206_08869_amd as iodf
    loss, lse = iodf.class_loss(s["u"], s["weight"], s["target"], live=s["live"])
    return {"loss": loss, "lse": lse}


def _own_loss_bwd(s):
    import paper_2206_08869_amd as iodf
    du, dweight = iodf.class_loss_backward(s["u"], s["weight"], s["target"], s["lse"], s["dloss"], dlse=s["dlse"], live=s["live"])
    return {"du": du, "dweight": dweight}


def _own_orth(s):
    import paper_2206_08869_amd as iodf
    return iodf.orthogonalise(s["g"], steps=STEPS, coefficients=QUINTIC, eps=EPS, dtype=TYPES[s["out"]])


def _own_muon(s):
    import paper_2206_08869_amd as iodf
    iodf.muon_step(s["weights"], s["grads"], s["momenta"], RATE, beta=BETA, nesterov=True, decay=DECAY, scale=_scale(s), steps=STEPS,
                   coefficients=QUINTIC, eps=EPS)
    return {"weights": s["weights"], "momenta": s["momenta"]}


def run(state):
    op = state["op"]
    if own:
        return {"loss": _own_loss, "loss_bwd": _own_loss_bwd, "orth": _own_orth, "muon": _own_muon}[op](state)
    if op == "orth":
        g = state["g"]
        return _plain_orth(g.float().view(-1, state["rows"], state["cols"])).to(TYPES[state["out"]]).view(g.shape)
    return {"loss": _plain_loss, "loss_bwd": _plain_loss_bwd, "muon": _plain_muon}[op](state)


def _products(count, rows, cols):
    """Operations of the orthogonalising: of the two symmetric products a half."""
    m, n = min(rows, cols), max(rows, cols)
    return count * STEPS * (3.0 * m * m * n + float(m) ** 3)


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    rows, cols = case["rows"], case["cols"]
    if case["op"] in ("loss", "loss_bwd"):
        tensors = size[case["type"]] * cols * (rows + case["classes"])
        flops = 2.0 * rows * cols * case["classes"]
        mask = rows if case["dead"] else 0
        if case["op"] == "loss":
            return {"bytes": tensors + 16 * rows + mask, "flops": flops}
        return {"bytes": 2 * tensors + (20 if case["penalty"] else 16) * rows + mask, "flops": 3 * flops}
    n = case["count"] * rows * cols
    if case["op"] == "orth":
        return {"bytes": n * (size[case["type"]] + size[case["out"]]), "flops": _products(case["count"], rows, cols)}
    return {"bytes": n * (2 * size[case["type"]] + size[case["grad"]] + 8), "flops": _products(case["count"], rows, cols)}


# ---- the definition in 64 bits ----

def _exact_orth(g):
    """One matrix, by the definition: p(X) = aX + b (XX')X + c (XX')(XX')X, on the side that is shorter."""
    g = g.double()
    x = g / (torch.linalg.vector_norm(g) + EPS)
    for _ in range(STEPS):
        if x.shape[0] <= x.shape[1]:
            left = x @ x.t().contiguous()
            once = left @ x
            twice = left @ once
        else:
            right = x.t().contiguous() @ x
            once = x @ right
            twice = once @ right
        x = QUINTIC[0] * x + QUINTIC[1] * once + QUINTIC[2] * twice
    return x


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "orth":
        g = s["g"]
        return _exact_orth(g) if g.dim() == 2 else torch.stack([_exact_orth(x) for x in g])
    if op == "muon":
        momenta, weights = [], []
        for w, g, m in zip(s["weights"], s["grads"], s["momenta"]):
            momenta.append(m.double() * BETA + g.double())
            weights.append(w.double() * (1 - RATE * DECAY) - RATE * _scale(case) * _exact_orth(g.double() + BETA * momenta[-1]))
        return {"weights": weights, "momenta": momenta}
    rows = case["rows"]
    live = torch.ones(rows, dtype=torch.bool, device="cuda") if s["live"] is None else s["live"]
    table, u = s["weight"].double(), s["u"].double().masked_fill(~live[:, None], 0.0)
    per = max(1, (1 << 28) // case["classes"])  # rows at a time
    first, second, dtable = [], [], torch.zeros_like(table)
    for at in range(0, rows, per):
        part, here = slice(at, at + per), live[at:at + per].double()
        target = s["target"][part].clamp(min=0)
        logits = u[part] @ table.t().contiguous()
        if op == "loss":
            lse = torch.logsumexp(logits, 1)
            first.append((lse - logits[torch.arange(len(target), device="cuda"), target]) * here)
            second.append(lse * here)
            continue
        up = s["dloss"][part].double() * here
        penalty = torch.zeros_like(up) if s["dlse"] is None else s["dlse"][part].double().masked_fill(here == 0, 0.0)
        probability = torch.exp(logits - s["lse"][part].double()[:, None])
        probability[here == 0] = 0.0
        g = probability * (up + penalty)[:, None]
        g[torch.arange(len(target), device="cuda"), target] -= up
        first.append(g @ table)
        dtable += g.t().contiguous() @ u[part]
    return {"loss": torch.cat(first), "lse": torch.cat(second)} if op == "loss" else {"du": torch.cat(first), "dweight": dtable}
