"""Learners of a small language model that learn from their own data and from their consensus, on one GPU.

Each of n learners keeps a flat fp32 vector of parameters, a row of X [n, d]; the layers read their weights as views of the rows and write
gradients into views of the rows of G.  One iteration:

  1. the consensus model, the mean of the rows, answers each learner's batch: its k most probable next tokens (token_logprobs);
  2. each learner's forward pass: layer norm, a feed-forward block (GELU, then a projection with the residual added in its epilogue), layer norm, head;
  3. two losses, both by distill: the data's next token (one slot: cross entropy) and the consensus' top tokens at a temperature;
  4. the backward pass, which fills G;
  5. the averaging step X = mix(X) - lr G with a fresh randomized ring, the consensus distance in the same pass.

    python examples/consensus_distillation.py [--steps 200] [--learners 8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2002_01119_amd import layers, psgd  # noqa: E402

DEV = "cuda:0"
WIDTH, HIDDEN, VOCABULARY = 96, 256, 500
TAU, TOP, CONSENSUS_SHARE = 2.0, 8, 0.3
SHAPES = dict(norm1=(WIDTH,), shift1=(WIDTH,), up=(HIDDEN, WIDTH), up_bias=(HIDDEN,), down=(WIDTH, HIDDEN), down_bias=(WIDTH,),
              norm2=(WIDTH,), shift2=(WIDTH,), head=(VOCABULARY, WIDTH), head_bias=(VOCABULARY,))


def offsets():
    """Where each parameter starts in a flat vector (on 128-byte lines), and the vector's length."""
    at, d = {}, 0
    for name, shape in SHAPES.items():
        at[name] = d
        d += -(-math.prod(shape) // 32) * 32
    return at, d


def views(rows):
    """The parameters of all learners as [n, ...] views of the rows of an [n, d] tensor."""
    at, _ = offsets()
    n, pitch = rows.shape[0], rows.stride(0)
    out = {}
    for name, shape in SHAPES.items():
        strides = (shape[1], 1) if len(shape) == 2 else (1,)
        out[name] = rows.as_strided((n, *shape), (pitch, *strides), rows.storage_offset() + at[name])
    return out


def first_parameters(n, seed):
    """n learners that start apart."""
    _, d = offsets()
    X = torch.zeros((n, d), device=DEV)
    g = torch.Generator(device=DEV).manual_seed(seed)
    for name, p in views(X).items():
        if name.startswith("norm"):
            p.fill_(1.0)
        elif p.dim() == 3:
            p.normal_(0.0, p.shape[2] ** -0.5, generator=g)
    return X


class Model:
    """The layers of n learners over batches of t tokens, with the activations that the backward pass wants."""

    def __init__(self, n, t):
        new = lambda *shape: torch.empty(shape, device=DEV)  # noqa: E731
        self.h1, self.x2, self.h2 = (new(n, t, WIDTH) for _ in range(3))
        self.z, self.a = new(n, t, HIDDEN), new(n, t, HIDDEN)
        self.stats = [new(n, t) for _ in range(4)]
        self.logits = new(n, t, VOCABULARY)
        self.dh, self.dx2, self.dx = (new(n, t, WIDTH) for _ in range(3))
        self.da = new(n, t, HIDDEN)

    def forward(self, p, x):
        m1, r1, m2, r2 = self.stats
        layers.layer_norm(x, p["norm1"], p["shift1"], self.h1, mean=m1, rstd=r1)
        layers.linear(self.h1, p["up"], self.a, bias=p["up_bias"], act="gelu", z=self.z)
        layers.linear(self.a, p["down"], self.x2, bias=p["down_bias"], residual=x)
        layers.layer_norm(self.x2, p["norm2"], p["shift2"], self.h2, mean=m2, rstd=r2)
        layers.linear(self.h2, p["head"], self.logits, bias=p["head_bias"])
        return self.logits

    def backward(self, p, g, x, dlogits):
        m1, r1, m2, r2 = self.stats
        layers.linear_grad(dlogits, self.h2, p["head"], dx=self.dh, dw=g["head"], db=g["head_bias"])
        layers.layer_norm_grad(self.dh, self.x2, p["norm2"], m2, r2, self.dx2, g["norm2"], g["shift2"])
        layers.linear_grad(self.dx2, self.a, p["down"], dx=self.da, dw=g["down"], db=g["down_bias"])
        layers.linear_grad(self.da, self.h1, p["up"], dx=self.dh, dw=g["up"], db=g["up_bias"], act="gelu", z=self.z)
        layers.layer_norm_grad(self.dh, x, p["norm1"], m1, r1, self.dx, g["norm1"], g["shift1"], add=self.dx2)


class Run:
    def __init__(self, n=8, t=64, seed=0, lr=0.5):
        self.n, self.t, self.lr, self.k = n, t, lr, 0
        self.X = first_parameters(n, seed)
        self.G, self.mean = torch.zeros_like(self.X), torch.empty_like(self.X)
        self.zero = torch.zeros_like(self.X)
        self.students, self.teacher = Model(n, t), Model(n, t)
        self.gen = torch.Generator(device=DEV).manual_seed(seed + 1)
        # what there is to learn: a next token that two tables decide, told from the token's features
        self.features = torch.empty((VOCABULARY, WIDTH), device=DEV).normal_(generator=self.gen)
        self.following = torch.randint(0, VOCABULARY, (VOCABULARY, 2), generator=self.gen, device=DEV)
        self.nbr, self.w = torch.empty((n, 3), dtype=torch.int32, device=DEV), torch.empty((n, 3), device=DEV)
        self.step_count, self.seed = torch.zeros(1, dtype=torch.int64, device=DEV), seed
        self.distance = torch.zeros(1, dtype=torch.float64, device=DEV)
        new = lambda *shape, **kw: torch.empty(shape, device=DEV, **kw)  # noqa: E731
        self.logp, self.entropy = new(n, t), new(n, t)
        self.top, self.top_idx = new(n, t, TOP), new(n, t, TOP, dtype=torch.int32)
        self.losses = [new(n, t), new(n, t)]
        self.grads = [new(n, t, VOCABULARY), new(n, t, VOCABULARY)]
        self.one = torch.zeros((n, t, 1), device=DEV)

    def batch(self):
        now = torch.randint(0, VOCABULARY, (self.n, self.t), generator=self.gen, device=DEV)
        way = (torch.rand((self.n, self.t), generator=self.gen, device=DEV) < 0.8).long()
        return self.features[now].contiguous(), self.following[now].gather(2, 1 - way[:, :, None])[:, :, 0].int()

    def gradients(self, x, target):
        """Both losses of every learner and, in G, their gradient."""
        psgd.mix_full(self.X, self.mean, self.zero, 0.0)                       # every row: the mean
        layers.token_logprobs(self.teacher.forward(views(self.mean), x), target, self.logp, entropy=self.entropy, top_logp=self.top, top_idx=self.top_idx)
        p, g = views(self.X), views(self.G)
        logits = self.students.forward(p, x)
        weight = torch.full((self.n, self.t), (1.0 - CONSENSUS_SHARE) / self.t, device=DEV)
        layers.distill(logits, target[:, :, None], self.one, self.losses[0], weight=weight, dlogits=self.grads[0])
        weight = torch.full((self.n, self.t), CONSENSUS_SHARE / self.t, device=DEV)
        layers.distill(logits, self.top_idx, self.top, self.losses[1], tau=TAU, weight=weight, dlogits=self.grads[1])
        self.students.backward(p, g, x, self.grads[0].add_(self.grads[1]))

    def step(self):
        self.gradients(*self.batch())
        psgd.build_mixing_device(psgd.TOPO_RAND_RING, self.n, self.seed, self.nbr, self.w, step_dev=self.step_count, advance=1)
        psgd.mix_step(self.X, self.X, self.G, self.nbr, self.w, self.lr, cdist_out=self.distance)
        self.k += 1

    def report(self):
        """Mean cross entropy of the learners, of the consensus on the same tokens, and the distance between the learners."""
        own = float(self.losses[0].sum(1).mean()) / (1.0 - CONSENSUS_SHARE)
        return own, -float(self.logp.mean()), float(self.distance)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--learners", type=int, default=8)
    a = ap.parse_args()
    torch.cuda.set_device(0)
    run = Run(a.learners)
    for k in range(a.steps):
        run.step()
        if k % max(1, a.steps // 10) == 0 or k == a.steps - 1:
            print("step %4d  cross entropy: learners %.4f, consensus %.4f   distance %.4g" % ((k,) + run.report()), flush=True)
    if psgd.device_status():
        raise SystemExit("a kernel raised a flag")


if __name__ == "__main__":
    main()
