"""The operators of training a network of residual blocks out of 8-bit activation checkpoints, as cases that can be timed.

A residual network (such as a prior head that is fitted to the latents of a flow) is a stream `h` [rows, cols] to which each
block adds `alpha * gate * norm(f)`, `f` the block's output, and from whose norm the next block reads. Rows are positions
of images or tokens. What the backward pass needs is kept in 8 bits:

  join   the end of one block and the start of the next in one pass, and its gradients out of the checkpoint
  glu    the gated activation act(a) * b inside a block, and its gradients out of the checkpoint
  wgrad  the gradient of a linear layer's weight, its input read from the checkpoint
  pack   a tensor into a checkpoint and back

A checkpoint holds groups of 32 columns as whole numbers q in -127..127 and one exponent byte e: the values q * 2^(e - 133).
`own` false computes the plain form in elementary 32-bit operations, `own` true calls the package.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-6
LARGEST = 1 << 27         # elements of one activation
LARGEST_FLOPS = 5.4e11    # of a weight gradient


def listed():
    def case(name, op, rows, cols, **more):
        return dict(name=name, op=op, rows=rows, cols=cols, **more)
    return [
        # one position at a time through a trained network of the dense flow's width: nothing is kept, latency counts
        case("join_fwd_one_row", "join", 1, 512, stream="bf16", block="bf16", groups=1, dead=0.0, save=False),
        # a prior head of the 64x64 flow, level 1: 128 images x 32 x 32 positions, width 512, the stream kept in 32 bits
        case("join_fwd_head", "join", 131072, 512, stream="f32", block="bf16", groups=1, dead=0.0, save=True),
        # seven ragged sequences with padding, a gate for each, a width that is a multiple of nothing
        case("join_bwd_ragged", "join_bwd", 4095, 1111, stream="f32", block="f32", groups=7, dead=0.2),
        # the largest ordinary training step: 32768 positions, width 4096
        case("join_bwd_wide", "join_bwd", 32768, 4096, stream="bf16", block="bf16", groups=1, dead=0.0),
        # inside a block, the hidden width four times a stream of 1024
        case("glu_fwd_wide", "glu", 32768, 4096, type="bf16", act="silu", dead=0.0, save=True),
        # an odd width, padding, 32 bits
        case("glu_bwd_ragged", "glu_bwd", 8195, 1365, type="f32", act="gelu", dead=0.1),
        case("glu_bwd_wide", "glu_bwd", 32768, 4096, type="bf16", act="silu", dead=0.0),
        # a small odd layer (the paper's 128 wide networks have such first and last layers)
        case("wgrad_ragged", "wgrad", 1000, 72, out=130, type="bf16", scale=True, dead=0.1),
        # a square projection of a prior head over all positions of a batch: few weights, a long sum
        case("wgrad_head", "wgrad", 131072, 512, out=512, type="bf16", scale=True, dead=0.0),
        # a large square projection
        case("wgrad_wide", "wgrad", 16384, 4096, out=4096, type="bf16", scale=False, dead=0.0),
        # the input of a projection that no norm precedes: a handful of rows, and a whole batch
        case("pack_rows", "pack", 37, 520, type="f32", dead=0.0),
        case("pack_head", "pack", 131072, 512, type="bf16", dead=0.0),
    ]


def _log(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _cols(rng, high):
    c = _log(rng, 8, high)
    return c if rng.random() < 0.5 or c < 64 else c // 32 * 32


def draw(rng):
    op = rng.choice(("join", "join_bwd", "glu", "glu_bwd", "wgrad", "wgrad", "pack"))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    stream = rng.choice((kind, "f32"))
    dead = rng.choice((0.0, 0.0, 0.15))
    cols = _cols(rng, 8192 if op != "wgrad" else 4096)
    rows = _log(rng, 1, min(131072, LARGEST // (2 if "f32" in (kind, stream) else 1) // cols))
    case = dict(op=op, rows=rows, cols=cols, dead=dead)
    if op in ("join", "join_bwd"):
        groups = rng.choice([g for g in (1, 1, 1, 2, 3, 4, 8, rows) if rows % g == 0])
        case.update(stream=stream, block=kind, groups=groups)
    elif op == "wgrad":
        kind = rng.choice(("bf16", "bf16", "bf16", kind))
        out = min(_cols(rng, 4096), LARGEST // rows)
        top = LARGEST_FLOPS / 2 / (1 if kind == "bf16" else 4)
        case.update(out=max(1, min(out, int(top / (rows * cols)))), type=kind, scale=rng.random() < 0.5)
    else:
        case.update(type=kind)
    if op in ("glu", "glu_bwd"):
        case.update(act=rng.choice(("silu", "gelu", "relu")))
    if op in ("join", "glu"):
        case.update(save=rng.random() < 0.7)
    return case


# ---- inputs ----

def _codes(x):
    """A checkpoint of x, as the package lays it out: q int8 [rows, pitch], e uint8 [rows, pitch / 32], pitch the columns rounded up to 32."""
    rows, cols = x.shape
    pitch = -(-cols // 32) * 32
    v = torch.nn.functional.pad(x.float(), (0, pitch - cols)).view(rows, pitch // 32, 32)
    e = ((v.abs().amax(2).view(torch.int32) + 0x10000) >> 23).clamp_(16, 254)
    q = torch.round(v * ((260 - e) << 23).view(torch.float32).unsqueeze(2)).clamp_(-127, 127)
    return q.to(torch.int8).view(rows, pitch), e.to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, rows, cols = case["op"], case["rows"], case["cols"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def spread(n, by):  # per-channel magnitudes: a few channels carry far more than the others
        return torch.exp(by * normal(n))

    s = dict(case)
    live = None
    if case["dead"]:
        live = torch.rand(rows, generator=gen, device="cuda") >= case["dead"]
        live[0] = True

    def masked(t):  # what stands in padded rows is anything
        if live is not None:
            t[~live] = float("nan")
        return t

    s["live"] = live
    if op in ("join", "join_bwd"):
        th, tf = TYPES[case["stream"]], TYPES[case["block"]]
        s["alpha"] = torch.full((1,), 0.7, device="cuda")
        s["gate"] = torch.sigmoid(normal(case["groups"], cols) + 1.0)
        s["w_post"] = 1.0 + 0.2 * normal(cols)
        s["w_pre"] = 1.0 + 0.2 * normal(cols)
        if op == "join":
            s["h"] = (normal(rows, cols) * spread(cols, 0.7)).to(th)
            s["f"] = masked((0.3 * normal(rows, cols) * spread(cols, 0.4)).to(tf))
        else:
            x, n = normal(rows, cols) * spread(cols, 0.4), normal(rows, cols) * spread(cols, 0.4)
            s["inv_pre"] = 0.2 + torch.rand(rows, generator=gen, device="cuda")
            s["inv_post"] = 1.0 + 2.0 * torch.rand(rows, generator=gen, device="cuda")
            if live is not None:
                for t in (x, n, s["inv_pre"], s["inv_post"]):
                    t[~live] = 0
            s["dh"] = (1e-2 * (normal(rows, cols) + 0.1 * n)).to(th)
            s["du"] = masked((1e-2 * (normal(rows, cols) - 0.1 * x)).to(tf))
            s["x"], s["n"] = _codes(x), _codes(n)
    elif op == "glu":
        ab = masked((normal(rows, 2 * cols) * spread(2 * cols, 0.4)).to(TYPES[case["type"]]))
        s["a"], s["b"] = ab[:, :cols], ab[:, cols:]  # the two halves of one projection
    elif op == "glu_bwd":
        a, b = normal(rows, cols) * spread(cols, 0.4), normal(rows, cols) * spread(cols, 0.4)
        if live is not None:
            a[~live] = 0
            b[~live] = 0
        s["a"], s["b"] = _codes(a), _codes(b)
        s["dy"] = masked((1e-2 * normal(rows, cols)).to(TYPES[case["type"]]))
    elif op == "wgrad":
        x = normal(rows, cols) * spread(cols, 0.4)
        s["w"] = 1.0 + 0.2 * normal(cols) if case["scale"] else None
        dy = 1e-2 * (normal(rows, case["out"]) + 0.1 * x[:, :1])
        if live is not None:
            x[~live] = 0
        s["x"] = _codes(x)
        s["dy"] = masked(dy.to(TYPES[case["type"]]))
    else:
        s["v"] = masked((normal(rows, cols) * spread(cols, 1.0)).to(TYPES[case["type"]]))
    return s


# ---- the plain form ----

def _values(code, cols):
    """What a checkpoint stands for, in 32 bits."""
    q, e = code
    step = ((e.to(torch.int32) - 6) << 23).view(torch.float32)
    return (q.float().view(q.shape[0], -1, 32) * step.unsqueeze(2)).view(q.shape[0], -1)[:, :cols]


def _kept(x):
    """What remains of x in a checkpoint. Exact in bfloat16: seven bits and a sign times a power of two."""
    return _values(_codes(x), x.shape[1]).to(torch.bfloat16)


def _act(a, kind):
    """act(a) and its derivative."""
    if kind == "relu":
        return a.clamp_min(0), (a > 0).float()
    if kind == "silu":
        s = 1 / (1 + torch.exp(-a))
        return a * s, s * (1 + a * (1 - s))
    k = 2 * math.sqrt(2 / math.pi)
    s = 1 / (1 + torch.exp(-k * (a + 0.044715 * a * a * a)))
    return a * s, s + a * s * (1 - s) * k * (1 + 3 * 0.044715 * a * a)


def _only(live, x):
    return x if live is None else torch.where(live.view(-1, *[1] * (x.dim() - 1)), x, torch.zeros_like(x))


def _rows_of(gate, rows):
    """The gate of each row: [1, cols] or [rows, cols]."""
    return gate if gate.shape[0] == 1 else gate.repeat_interleave(rows // gate.shape[0], 0)


def _plain_join(s):
    live, h, f = s["live"], s["h"].float(), _only(s["live"], s["f"].float())
    inv_post = torch.rsqrt((f * f).mean(1) + EPS)
    n = f * inv_post[:, None]
    z = h + s["alpha"] * _rows_of(s["gate"], s["rows"]) * s["w_post"] * n
    inv_pre = torch.rsqrt((z * z).mean(1) + EPS)
    x = _only(live, z * inv_pre[:, None])
    out = {"h": z.to(s["h"].dtype), "u": (x * s["w_pre"]).to(s["f"].dtype)}
    if s["save"]:
        out.update(x=_kept(x), n=_kept(n), inv_pre=_only(live, inv_pre), inv_post=_only(live, inv_post))
    return out


def _plain_join_bwd(s):
    live, rows, cols = s["live"], s["rows"], s["cols"]
    x, n = _values(s["x"], cols), _values(s["n"], cols)
    dh, du = s["dh"].float(), _only(live, s["du"].float())
    gate = _rows_of(s["gate"], rows)
    dx = du * s["w_pre"]
    dz = dh + s["inv_pre"][:, None] * (dx - x * (dx * x).mean(1, keepdim=True))
    dn = s["alpha"] * gate * s["w_post"] * dz
    df = _only(live, s["inv_post"][:, None] * (dn - n * (dn * n).mean(1, keepdim=True)))
    share = (dz * n).view(s["groups"], -1, cols).sum(1)  # of a gate, before alpha and the norm's weight
    return {"dh": dz.to(s["dh"].dtype), "df": df.to(s["du"].dtype), "dgate": s["alpha"] * s["w_post"] * share,
            "dw_post": s["alpha"] * (s["gate"] * share).sum(0), "dw_pre": (du * x).sum(0),
            "dalpha": (s["gate"] * s["w_post"] * share).sum().view(1)}


def _plain_glu(s):
    a, b = _only(s["live"], s["a"].float()), _only(s["live"], s["b"].float())
    out = {"y": (_act(a, s["act"])[0] * b).to(s["a"].dtype)}
    if s["save"]:
        out.update(a=_kept(a), b=_kept(b))
    return out


def _plain_glu_bwd(s):
    a, b, dy = _values(s["a"], s["cols"]), _values(s["b"], s["cols"]), _only(s["live"], s["dy"].float())
    y, slope = _act(a, s["act"])
    return {"da": (dy * b * slope).to(s["dy"].dtype), "db": (dy * y).to(s["dy"].dtype), "y": _kept(y * b)}


def _plain_wgrad(s):
    dw = torch.matmul(_only(s["live"], s["dy"].float()).t(), _values(s["x"], s["cols"]))
    return dw if s["w"] is None else dw * s["w"]


def _plain_pack(s):
    return _kept(_only(s["live"], s["v"].float()))


# ---- the package's calls ----

def _own_join(s):
    import paper_2206_08869_amd as iodf
    h, u, saved = iodf.join(s["h"], s["f"], s["alpha"], s["gate"], s["w_post"], s["w_pre"], live=s["live"], eps=EPS, save=s["save"])
    out = {"h": h, "u": u}
    if saved is not None:
        out.update(x=iodf.unpack(saved.x), n=iodf.unpack(saved.n), inv_pre=saved.inv_pre, inv_post=saved.inv_post)
    return out


def _own_join_bwd(s):
    import paper_2206_08869_amd as iodf
    saved = iodf.JoinSaved(iodf.Codes(*s["x"], s["cols"]), iodf.Codes(*s["n"], s["cols"]), s["inv_pre"], s["inv_post"])
    g = iodf.join_backward(saved, s["dh"], s["du"], s["alpha"], s["gate"], s["w_post"], s["w_pre"], live=s["live"])
    return {"dh": g.dh, "df": g.df, "dgate": g.dgate, "dw_post": g.dw_post, "dw_pre": g.dw_pre, "dalpha": g.dalpha}


def _own_glu(s):
    import paper_2206_08869_amd as iodf
    y, saved = iodf.glu(s["a"], s["b"], s["act"], live=s["live"], save=s["save"])
    return {"y": y} if saved is None else {"y": y, "a": iodf.unpack(saved.a), "b": iodf.unpack(saved.b)}


def _own_glu_bwd(s):
    import paper_2206_08869_amd as iodf
    saved = iodf.GluSaved(iodf.Codes(*s["a"], s["cols"]), iodf.Codes(*s["b"], s["cols"]))
    da, db, y = iodf.glu_backward(saved, s["dy"], s["act"], live=s["live"])
    return {"da": da, "db": db, "y": iodf.unpack(y)}


def _own_wgrad(s):
    import paper_2206_08869_amd as iodf
    return iodf.weight_grad(iodf.Codes(*s["x"], s["cols"]), s["dy"], col_scale=s["w"], live=s["live"])


def _own_pack(s):
    import paper_2206_08869_amd as iodf
    return iodf.unpack(iodf.pack(s["v"], live=s["live"]))


PLAIN = {"join": _plain_join, "join_bwd": _plain_join_bwd, "glu": _plain_glu, "glu_bwd": _plain_glu_bwd, "wgrad": _plain_wgrad,
         "pack": _plain_pack}
OWN = {"join": _own_join, "join_bwd": _own_join_bwd, "glu": _own_glu, "glu_bwd": _own_glu_bwd, "wgrad": _own_wgrad, "pack": _own_pack}


def run(state):
    return (OWN if own else PLAIN)[state["op"]](state)


def work(case):
    """Bytes of the inputs and outputs, a checkpoint that is an input at 33/32 bytes an element, one that is an output as the bfloat16 values that come back."""
    op, rows, cols = case["op"], case["rows"], case["cols"]
    size = {"bf16": 2, "f16": 2, "f32": 4}
    n = rows * cols
    code = 33 / 32
    mask = rows if case["dead"] else 0
    if op in ("join", "join_bwd"):
        sh, sf = size[case["stream"]], size[case["block"]]
        params = 4 * (case["groups"] * cols + 2 * cols + 1)
        if op == "join":
            return {"bytes": n * (2 * sh + 2 * sf + (4 if case["save"] else 0)) + params + mask + (8 * rows if case["save"] else 0), "flops": 14 * n}
        return {"bytes": n * (2 * sh + 2 * sf + 2 * code) + 2 * params + mask + 8 * rows, "flops": 24 * n}
    t = size[case["type"]]
    if op == "glu":
        return {"bytes": n * (3 * t + (4 if case["save"] else 0)) + mask, "flops": 10 * n}
    if op == "glu_bwd":
        return {"bytes": n * (3 * t + 2 * code + 2) + mask, "flops": 20 * n}
    if op == "wgrad":
        return {"bytes": rows * case["out"] * t + n * code + 4 * case["out"] * cols + mask, "flops": 2.0 * n * case["out"]}
    return {"bytes": n * (t + 2) + mask, "flops": 4 * n}


# ---- the definition in 64 bits ----

def exact(case, seed):
    """From the formulas, row by row in 64 bits. Codes of computed numbers have no such value: which of two neighbouring codes a
    number on their border gets is a matter of its last bit."""
    s = prepare(case, seed)
    op, rows, cols = case["op"], case["rows"], case["cols"]
    alive = torch.ones(rows, dtype=torch.bool, device="cuda") if s["live"] is None else s["live"]

    def wide(t):  # 64 bits; rows that are padding count as zeros
        return t.double().masked_fill_(~alive[:, None], 0.0)

    def decoded(code):
        q, e = code
        return (q.double() * torch.exp2(e.double() - 133.0).repeat_interleave(32, dim=1))[:, :cols]

    def rounded(v):
        """v's checkpoint by its definition: the least power of two with which no code passes 127."""
        pad = torch.zeros(rows, -cols % 32, dtype=torch.float64, device="cuda")
        g = torch.cat((v, pad), 1).reshape(rows, -1, 32)
        top = g.abs().amax(2, keepdim=True)
        power = torch.floor(torch.log2(top.clamp_min(2.0 ** -111))) - 6
        power = power + (torch.round(top * torch.exp2(-power)) > 127)
        return (torch.round(g * torch.exp2(-power)) * torch.exp2(power)).reshape(rows, -1)[:, :cols]

    def gated(a):
        if case["act"] == "relu":
            return torch.relu(a), torch.heaviside(a, torch.zeros((), dtype=torch.float64, device="cuda"))
        if case["act"] == "silu":
            sig = torch.sigmoid(a)
            return a * sig, sig + a * sig * torch.sigmoid(-a)
        r = math.sqrt(2 / math.pi)
        th = torch.tanh(r * (a + 0.044715 * a ** 3))
        return 0.5 * a * (1 + th), 0.5 * (1 + th) + 0.5 * a * (1 - th ** 2) * r * (1 + 0.134145 * a ** 2)

    if op == "pack":
        return rounded(wide(s["v"]))
    if op == "wgrad":
        dw = wide(s["dy"]).t().contiguous() @ decoded(s["x"])
        return dw if s["w"] is None else dw * s["w"].double()
    if op == "glu":
        a, b = wide(s["a"]), wide(s["b"])
        out = {"y": gated(a)[0] * b}
        return dict(out, a=rounded(a), b=rounded(b)) if case["save"] else out
    if op == "glu_bwd":
        a, b, dy = decoded(s["a"]), decoded(s["b"]), wide(s["dy"])
        y, slope = gated(a)
        return {"da": dy * b * slope, "db": dy * y, "y": None}
    alpha, wp, wq = s["alpha"].double(), s["w_post"].double(), s["w_pre"].double()
    per_row = rows // case["groups"]
    gate = s["gate"].double()
    full = gate if case["groups"] == 1 else gate[torch.arange(rows, device="cuda") // per_row]
    if op == "join":
        f = wide(s["f"])
        ip = (f.square().sum(1) / cols + EPS) ** -0.5
        z = s["h"].double() + alpha * full * wp * (f * ip[:, None])
        iq = (z.square().sum(1) / cols + EPS) ** -0.5
        out = {"h": z, "u": wide(z * iq[:, None] * wq)}
        return dict(out, x=None, n=None, inv_pre=iq * alive, inv_post=ip * alive) if case["save"] else out
    x, n, du = decoded(s["x"]), decoded(s["n"]), wide(s["du"])
    ip, iq = s["inv_post"].double()[:, None], s["inv_pre"].double()[:, None]
    g = du * wq
    dz = s["dh"].double() + iq * (g - x * ((g * x).sum(1, keepdim=True) / cols))
    dn = alpha * full * wp * dz
    df = ip * (dn - n * ((dn * n).sum(1, keepdim=True) / cols))
    each = (dz * n).reshape(case["groups"], per_row, cols).sum(1)
    return {"dh": dz, "df": wide(df), "dgate": alpha * wp * each, "dw_post": (alpha * gate * each).sum(0), "dw_pre": (du * x).sum(0),
            "dalpha": (gate * wp * each).sum().reshape(1)}
