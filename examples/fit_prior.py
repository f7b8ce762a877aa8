"""Fits a prior to a flow's own latents, out of 8-bit activation checkpoints.

A flow's prior gives every latent a discretised logistic distribution; the closer its mean and scale, the fewer bits the coder needs. This program
takes images through `Flow.forward` and trains a residual network that predicts the level-1 latents of a position from the deeper levels' latents
there, which a decoder has before it (levels are decoded from the deepest one up). The network is a stream of residual blocks with norms around each
block, a gate and a residual scale; all that its backward pass keeps of them is in 8 bits. The bits that it prints are what such a prior would need;
the coder itself keeps to the blob's integer prior, which is the same to the bit everywhere, as a network in bfloat16 is not.

With `--loss classes` the network gives each value of a latent a probability of its own instead of a logistic distribution's: softmax cross entropy against a
table of values for each channel, whose logits are never kept. With `--optimiser muon` the blocks' weights take orthogonalised updates.

    python examples/fit_prior.py --model paper_res32 --images 64 --steps 60
    python examples/fit_prior.py --model paper_res32 --images 64 --steps 60 --loss classes --optimiser muon
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2206_08869_amd as iodf  # noqa: E402
from synth import CONFIGS, make_blob, make_images  # noqa: E402


def latents(model, images):
    """(target [rows, C_z] of level 1, context [rows, channels] of the deeper levels at the same place), float32, a row for each position."""
    cfg = CONFIGS[model]
    flow = iodf.Flow(make_blob(cfg), max_batch=images, device=0)
    x = torch.from_numpy(make_images(cfg, batch=images)).cuda()
    z, _ = flow.forward(x, want_codes=False)
    torch.cuda.synchronize()
    h1, w1 = cfg.level_hw(1)
    chunks, at = [], 0
    for level in range(1, cfg.levels + 1):
        (h, w), c = cfg.level_hw(level), cfg.z_chunk_channels(level)
        chunk = z[:, at:at + c * h * w].view(images, c, h, w).float()
        at += c * h * w
        chunks.append(chunk.repeat_interleave(h1 // h, 2).repeat_interleave(w1 // w, 3).permute(0, 2, 3, 1).reshape(images * h1 * w1, c))
    flow.close()
    return chunks[0].contiguous(), torch.cat(chunks[1:], 1).contiguous()


class Prior:
    """context -> mean and log-scale: a projection into the stream, `depth` gated blocks, a projection out of it. values: instead of the last a table of
    that many values for each channel."""

    def __init__(self, n_in, n_out, width, hidden, depth, seed=0, values=None):
        gen = torch.Generator("cuda").manual_seed(seed)

        def weight(rows, cols, by=1.0):
            return (by / math.sqrt(cols) * torch.randn((rows, cols), generator=gen, device="cuda")).requires_grad_()

        def flat(n, value):
            return torch.full((n,), value, device="cuda").requires_grad_()

        def join():  # residual scale, gate, weights of the norms behind and before
            return [flat(1, 1.0 / math.sqrt(depth + 1)), flat(width, 1.0), flat(width, 1.0), flat(width, 1.0)]

        self.into, self.out, self.width = weight(width, n_in), weight(2 * n_out, width, 0.1), width
        self.joins = [join() for _ in range(depth + 1)]
        self.blocks = [(weight(2 * hidden, width), weight(width, hidden)) for _ in range(depth)]
        self.tables = [weight(values, width, 0.1) for _ in range(n_out)] if values else []

    def parameters(self):
        return [self.into, self.out] + [p for j in self.joins for p in j] + [w for b in self.blocks for w in b] + self.tables

    def train_trunk(self, context):
        """The last stream, and the codes that it is in for the backward pass."""
        x = context.bfloat16()
        h = torch.zeros((x.shape[0], self.width), device="cuda")
        h, u, codes = iodf.joined(h, iodf.projection(x, self.into, iodf.pack(x)), *self.joins[0])
        for (w1, w2), join, before in zip(self.blocks, self.joins[1:], self.joins):
            ab = iodf.projection(u, w1, codes, col_scale=before[3].detach())
            h, u, codes = iodf.joined(h, iodf.gated_projection(ab, w2), *join)
        return u, codes

    def train_pass(self, context):
        u, codes = self.train_trunk(context)
        return iodf.projection(u, self.out, codes, col_scale=self.joins[-1][3].detach()).float()

    def train_bits(self, context, value):
        """Bits a latent, whose values [rows, channels] count from 0 up, under the tables."""
        u, _ = self.train_trunk(context)
        return sum(iodf.classified(u, t, v).loss.mean() for t, v in zip(self.tables, value.t().contiguous())) / (math.log(2.0) * len(self.tables))

    @torch.no_grad()
    def infer_trunk(self, context):
        """The same stream, keeping nothing: for any number of rows, one among them."""
        x = context.bfloat16()
        h = torch.zeros((x.shape[0], self.width), device="cuda")
        h, u, _ = iodf.join(h, x @ self.into.bfloat16().t(), *self.joins[0], save=False, h_out=h)
        for (w1, w2), join in zip(self.blocks, self.joins[1:]):
            ab = u @ w1.bfloat16().t()
            half = ab.shape[1] // 2
            y, _ = iodf.glu(ab[:, :half], ab[:, half:], save=False)
            h, u, _ = iodf.join(h, y @ w2.bfloat16().t(), *join, save=False, h_out=h)
        return u

    @torch.no_grad()
    def infer(self, context):
        return (self.infer_trunk(context) @ self.out.bfloat16().t()).float()

    @torch.no_grad()
    def infer_bits(self, context, value):
        """Bits of each latent."""
        u = self.infer_trunk(context)
        return torch.stack([iodf.class_loss(u, t.bfloat16(), v).loss for t, v in zip(self.tables, value.t().contiguous())], 1) / math.log(2.0)


def bits(z, mean, log_scale):
    """Bits a latent under the discretised logistic distribution."""
    inv = torch.exp(-log_scale)
    mass = torch.sigmoid((z - mean + 0.5) * inv) - torch.sigmoid((z - mean - 0.5) * inv)
    return -torch.log2(mass.clamp_min(2.0 ** -24)).mean()


class Muon:
    """The blocks' weights by orthogonalised updates, those of one shape together; everything else by Adam."""

    def __init__(self, prior, rate, adam_rate):
        self.groups, self.rate = [[prior.into], [b[0] for b in prior.blocks], [b[1] for b in prior.blocks]], rate
        self.momenta = [[torch.zeros_like(w) for w in g] for g in self.groups]
        own = {id(w) for g in self.groups for w in g}
        self.rest = torch.optim.Adam([p for p in prior.parameters() if id(p) not in own], lr=adam_rate)

    def zero_grad(self):
        self.rest.zero_grad()
        for w in (w for g in self.groups for w in g):
            w.grad = None

    def step(self):
        self.rest.step()
        for weights, momenta in zip(self.groups, self.momenta):
            if weights:
                iodf.muon_step(weights, [w.grad for w in weights], momenta, self.rate)


def fit(model="paper_res32", images=64, width=512, hidden=1024, depth=4, steps=60, rate=2e-3, say=print, loss="logistic", optimiser="adam"):
    """Bits a level-1 latent before and after, and the bytes a row that the backward pass keeps of the blocks."""
    z, context = latents(model, images)
    context = context / context.std(0, keepdim=True).clamp_min(1.0)
    centre, spread = z.mean(0, keepdim=True), z.std(0, keepdim=True).clamp_min(0.5).log() - 0.55  # a logistic's scale is 0.55 of its deviation
    value = (z - z.min()).long()
    prior = Prior(context.shape[1], z.shape[1], width, hidden, depth, values=int(value.max()) + 1 if loss == "classes" else None)

    def loss_of(out):
        mean, log_scale = out.chunk(2, 1)
        return bits(z, centre + mean * spread.exp(), spread + log_scale)

    def train_loss():
        return prior.train_bits(context, value) if loss == "classes" else loss_of(prior.train_pass(context))

    def infer_loss():
        return float(prior.infer_bits(context, value).mean() if loss == "classes" else loss_of(prior.infer(context)))

    params = prior.parameters()
    update = Muon(prior, 0.02, rate) if optimiser == "muon" else torch.optim.Adam(params, lr=rate)
    first = infer_loss()
    for step in range(steps):
        now = train_loss()
        update.zero_grad()
        now.backward()
        update.step()
        if say and step % 10 == 0:
            say("step %3d: %.4f bits a latent" % (step, float(now.detach())))
    last = infer_loss()
    answer = (lambda n: prior.infer_bits(context[:n], value[:n])) if loss == "classes" else (lambda n: prior.infer(context[:n]))
    kept = (depth + 1) * 2 * width + depth * 2 * hidden
    return dict(first=first, last=last, rows=z.shape[0], kept_bytes_a_row=kept * 33 / 32, kept_in_16_bits=kept * 2, one_row=answer(1),
                all_rows=answer(z.shape[0]), prior=prior)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", default="paper_res32", choices=sorted(n for n, c in CONFIGS.items() if c.levels > 1))
    ap.add_argument("--images", type=int, default=64)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--depth", type=int, default=4)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--loss", default="logistic", choices=("logistic", "classes"))
    ap.add_argument("--optimiser", default="adam", choices=("adam", "muon"))
    a = ap.parse_args()
    r = fit(a.model, a.images, a.width, a.hidden, a.depth, a.steps, loss=a.loss, optimiser=a.optimiser)
    print("%d positions: %.4f -> %.4f bits a level-1 latent; the blocks keep %.0f bytes a position for the backward pass (%d in 16 bits)" % (
        r["rows"], r["first"], r["last"], r["kept_bytes_a_row"], r["kept_in_16_bits"]))
