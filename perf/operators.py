"""Performance cases of the learners' layers and losses: what produces the gradients that the averaging step takes.

All n learners are computed at once: activations are [n, t, c] (t tokens of every learner), parameters are views of the rows of an
[n, d] array, one flat vector a learner, and gradients of parameters are written into views of the rows of another.  Kinds:

  norm          layer norm: y, mean and 1/deviation of every row
  norm_grad     its backward pass: the input's gradient (plus, with `extra`, the gradient that comes past the norm), and the gain's and bias's
  linear        y = act(x W' + b) + residual; with `extra` the residual, with `save` also z = x W' + b for the backward pass
  linear_grad   its backward pass: the gradients of x, W and b from those of y
  logprobs      log probability of a given token in every row, the row's entropy and the k most probable tokens
  distill       distillation from a teacher's k top logits: each row's loss and the gradient of the student's logits

Common fields: n learners, t tokens each, type of the activations, ptype of a norm's parameters (a linear layer's have the activations'
type), gtype of a norm's parameter gradients, off the column of the flat vectors at which the layer's parameters start, pitch the
columns that lie between an activation's rows, masked whether there are masked tokens, rows and vocabulary entries.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
EPS = 1e-5
DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
DEV = "cuda:0"


def _norm(kind, n, t, h, name=None, type=BF16, ptype=F32, gtype=F32, off=0, pitch=0, extra=False):
    c = dict(kind=kind, n=n, t=t, h=h, type=type, ptype=ptype, gtype=gtype, off=off, pitch=pitch, extra=extra)
    return dict(c, name=name) if name else c


def _linear(kind, n, t, i, o, name=None, type=BF16, act="none", bias=True, off=0, pitch=0, extra=False, save=False):
    c = dict(kind=kind, n=n, t=t, i=i, o=o, type=type, act=act, bias=bias, off=off, pitch=pitch, extra=extra, save=save)
    return dict(c, name=name) if name else c


def _tokens(kind, n, t, v, k, name=None, type=BF16, tau=1.0, pitch=0, masked=False):
    c = dict(kind=kind, n=n, t=t, v=v, k=k, type=type, tau=tau, pitch=pitch, masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token of each of eight learners: a call that costs its launch.
        _norm("norm", 8, 1, 512, "norm_n8_t1_h512", type=F32),
        # A training batch of four learners, parameters in the fp32 rows that are averaged.
        _norm("norm", 4, 4096, 4096, "norm_n4_t4096_h4096_bf16"),
        # Its backward pass at another width, bfloat16 gradients, the residual path's gradient added.
        _norm("norm_grad", 8, 4096, 2048, "norm_grad_n8_t4096_h2048_bf16", gtype=BF16, extra=True),
        # Odd sizes, parameters at an odd column, full precision.
        _norm("norm_grad", 16, 257, 1001, "norm_grad_n16_t257_h1001_odd", type=F32, off=77),
        # One new token for each of eight learners: the weights are read once.
        _linear("linear", 8, 1, 4096, 4096, "linear_n8_t1_4096x4096_bf16"),
        # First layer of a feed-forward block on a training batch, its pre-activations kept.
        _linear("linear", 4, 2048, 2048, 8192, "linear_n4_t2048_2048x8192_gelu_bf16", act="gelu", save=True),
        # The backward pass of such a layer.
        _linear("linear_grad", 4, 2048, 8192, 2048, "linear_grad_n4_t2048_8192x2048_silu_bf16", act="silu"),
        # Full precision, sizes that no tile divides, weights at an odd column.
        _linear("linear_grad", 3, 257, 1000, 771, "linear_grad_n3_t257_1000x771_odd", type=F32, act="relu", off=5),
        # One token sampled from a large vocabulary.
        _tokens("logprobs", 1, 1, 131072, 8, "logprobs_n1_t1_v131072_bf16"),
        # Scoring held-out text: padded vocabulary, ignored tokens, a row that the mask leaves empty.
        _tokens("logprobs", 8, 512, 32000, 20, "logprobs_n8_t512_v32000_masked", type=F32, masked=True),
        # Odd sizes, absent teacher slots, masked rows, a soft temperature.
        _tokens("distill", 16, 37, 10007, 16, "distill_n16_t37_v10007_masked", type=F32, tau=2.0, masked=True),
        # The largest: four learners' batches against 64 teacher logits a token.
        _tokens("distill", 4, 2048, 131072, 64, "distill_n4_t2048_v131072_bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(1, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)))))))


def _size(rng, lo, hi):
    """A size of the range: odd ones, multiples of eight and powers of two among them."""
    v = _log_int(rng, lo, hi)
    how = rng.random()
    if how < 0.35:
        return v | 1
    if how < 0.7:
        return max(8, v // 8 * 8) if hi >= 8 else v
    return min(hi, 1 << max(0, round(math.log2(v))))


def draw(rng):
    """A call of the same ranges: 1 .. 64 learners, one token to thousands, rows of 16 .. 16 384 activations or 100 .. 200 000 logits."""
    kind = rng.choice(["norm", "norm_grad", "linear", "linear", "linear_grad", "logprobs", "distill"])
    n = _log_int(rng, 1, 64)
    pitch = rng.choice([0, 0, 0, 8, 24, 3])
    off = rng.choice([0, 0, 64, 8, 7, 129])
    kind_of = rng.choice([F32, BF16, BF16])
    if kind in ("norm", "norm_grad"):
        h = _size(rng, 16, 16384)
        t = _size(rng, 1, max(1, min(16384, (1 << 26) // (n * h))))
        return _norm(kind, n, t, h, type=kind_of, ptype=rng.choice([F32, F32, BF16]), gtype=rng.choice([F32, BF16]), off=off, pitch=pitch,
                     extra=kind == "norm_grad" and rng.random() < 0.5)
    if kind in ("linear", "linear_grad"):
        n = min(n, 16)
        i, o = _size(rng, 16, 8192), _size(rng, 16, 8192)
        most = (5e11 if kind_of == BF16 else 1e11) / (4 if kind == "linear_grad" else 2) / (n * i * o)
        t = _size(rng, 1, max(1, min(8192, int(most))))
        act = rng.choice(["none", "relu", "gelu", "silu"])
        return _linear(kind, n, t, i, o, type=kind_of, act=act, bias=rng.random() < 0.7, off=off, pitch=pitch,
                       extra=kind == "linear" and rng.random() < 0.4, save=kind == "linear" and act != "none" and rng.random() < 0.5)
    v = _size(rng, 100, 200_000)
    t = _size(rng, 1, max(1, min(8192, (1 << 28) // (n * v))))
    k = _log_int(rng, 1, min(64, v // 2))
    return _tokens(kind, n, t, v, k, type=kind_of, tau=rng.choice([1.0, 2.0, 0.7]) if kind == "distill" else 1.0, pitch=pitch,
                   masked=rng.random() < 0.4)


# ------------------------------------------------------------------------------------------------ inputs
class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, type, mean=0.0, sigma=1.0):
        return torch.empty(shape, dtype=DTYPE[type], device=DEV).normal_(mean, sigma, generator=self.g)

    def ints(self, lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEV)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)


def _rows(case, c, type, draws=None, sigma=1.0):
    """An [n, t, c] activation whose rows lie `pitch` columns apart; drawn, or an output to be written."""
    shape = (case["n"], case["t"], c + case["pitch"])
    whole = draws.normal(shape, type, 0.0, sigma) if draws else torch.zeros(shape, dtype=DTYPE[type], device=DEV)
    return whole[:, :, :c]


def _flat(case, size, type):
    """Flat vectors of the n learners with a layer of `size` parameters at column `off`, and their number of columns."""
    d = case["off"] + size
    return torch.zeros((case["n"], d), dtype=DTYPE[type], device=DEV), d


def _prepare_norm(case, draws):
    n, t, h, off = case["n"], case["t"], case["h"], case["off"]
    x = _rows(case, h, case["type"], draws, 1.5)
    x += draws.normal((n, t, 1), case["type"], 0.0, 0.5)       # tokens differ in their mean
    flat, _ = _flat(case, 2 * h, case["ptype"])
    gain, bias = flat[:, off:off + h], flat[:, off + h:]
    gain.copy_(draws.normal((n, h), case["ptype"], 1.0, 0.1))
    bias.copy_(draws.normal((n, h), case["ptype"], 0.0, 0.1))
    s = dict(case=case, x=x, gain=gain, bias=bias)
    if case["kind"] == "norm":
        return dict(s, y=_rows(case, h, case["type"]), mean=torch.empty((n, t), device=DEV), rstd=torch.empty((n, t), device=DEV))
    xf = x.float()
    mean = xf.mean(2)
    s["mean"], s["rstd"] = mean, ((xf - mean[:, :, None]).square().mean(2) + EPS).rsqrt()
    s["dy"] = _rows(case, h, case["type"], draws, 1e-2)
    s["extra"] = _rows(case, h, case["type"], draws, 1e-2) if case["extra"] else None
    grads, _ = _flat(case, 2 * h, case["gtype"])
    return dict(s, dx=_rows(case, h, case["type"]), dgain=grads[:, off:off + h], dbias=grads[:, off + h:])


def _prepare_linear(case, draws):
    n, i, o, off, type = case["n"], case["i"], case["o"], case["off"], case["type"]

    def layer(flat, d):
        return flat.as_strided((n, o, i), (d, i, 1), off), flat[:, off + o * i:]

    w, b = layer(*_flat(case, o * i + o, type))
    w.copy_(draws.normal((n, o, i), type, 0.0, 1.0 / math.sqrt(i)))
    b.copy_(draws.normal((n, o), type, 0.0, 0.2))
    s = dict(case=case, x=_rows(case, i, type, draws), w=w, b=b if case["bias"] else None)
    if case["kind"] == "linear":
        s["residual"] = _rows(case, o, type, draws) if case["extra"] else None
        s["z"] = _rows(case, o, type) if case["save"] else None
        return dict(s, y=_rows(case, o, type))
    s["z"] = _rows(case, o, type, draws) if case["act"] != "none" else None
    s["dy"] = _rows(case, o, type, draws, 1e-2)
    dw, db = layer(*_flat(case, o * i + o, type))
    return dict(s, dx=_rows(case, i, type), dw=dw, db=db if case["bias"] else None)


def _prepare_tokens(case, draws):
    n, t, v, k = case["n"], case["t"], case["v"], case["k"]
    logits = _rows(case, v, case["type"], draws, 2.0)
    if case["masked"]:
        logits[:, :, v - v // 50:] = -math.inf                    # a vocabulary padded to its size
    s = dict(case=case, logits=logits)
    if case["kind"] == "logprobs":
        tokens = draws.ints(0, v - v // 50, (n, t))
        logits.scatter_add_(2, tokens[:, :, None], draws.normal((n, t, 1), case["type"], 4.0, 3.0))
        if case["masked"]:
            tokens[draws.uniform((n, t)) < 0.1] = -1
            logits[n - 1, t - 1] = -math.inf
        out = dict(logp=torch.empty((n, t), device=DEV), entropy=torch.empty((n, t), device=DEV),
                   top_logp=torch.empty((n, t, k), device=DEV), top_idx=torch.empty((n, t, k), dtype=torch.int32, device=DEV))
        return dict(s, tokens=tokens.int(), **out)
    first = draws.ints(0, v, (n, t, 1))
    step = draws.ints(1, max(2, v // k), (n, t, 1))
    idx = (first + step * torch.arange(k, device=DEV)) % v        # k different tokens
    top = (draws.normal((n, t, k), F32, 0.0, 2.0)).sort(2, descending=True).values + 6.0
    logits.scatter_add_(2, idx, (0.7 * top).to(logits.dtype))      # a student that has learned some of it
    weight = torch.full((n, t), 1.0 / t, device=DEV)
    if case["masked"]:
        idx = torch.where(draws.uniform((n, t, k)) < 0.1, -1, idx)
        idx = torch.where(torch.isneginf(logits.gather(2, idx.clamp(min=0))), -1, idx)
        if t > 4:
            idx[:, 0] = -1                                         # a row without any teacher slot
            weight[draws.uniform((n, t)) < 0.1] = 0.0
            logits[n - 1, t - 1] = math.nan                        # a padded row that nobody computed
            weight[n - 1, t - 1] = 0.0
    return dict(s, idx=idx.int(), top=top, weight=weight, loss=torch.empty((n, t), device=DEV), dlogits=_rows(case, v, case["type"]))


def prepare(case, seed):
    draws = _Draws(seed)
    if case["kind"].startswith("norm"):
        return _prepare_norm(case, draws)
    if case["kind"].startswith("linear"):
        return _prepare_linear(case, draws)
    return _prepare_tokens(case, draws)


# ------------------------------------------------------------------------------------------------ plain forms, in 32 bits
def _act(name, z):
    if name == "relu":
        return z * (z > 0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    p = 1.0 / (1.0 + torch.exp(-z))
    return p * (1.0 + z * (1.0 - p))


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(2, keepdim=True)
    c = x - mean
    rstd = (c.square().mean(2, keepdim=True) + EPS).rsqrt()
    y = c * rstd * s["gain"].float()[:, None] + s["bias"].float()[:, None]
    return {"y": y.to(s["x"].dtype), "mean": mean[:, :, 0], "rstd": rstd[:, :, 0]}


def _plain_norm_grad(s):
    case = s["case"]
    dy, rstd = s["dy"].float(), s["rstd"][:, :, None]
    xh = (s["x"].float() - s["mean"][:, :, None]) * rstd
    g = dy * s["gain"].float()[:, None]
    dx = rstd * (g - g.mean(2, keepdim=True) - xh * (g * xh).mean(2, keepdim=True))
    if s["extra"] is not None:
        dx = dx + s["extra"].float()
    out = DTYPE[case["gtype"]]
    return {"dx": dx.to(s["x"].dtype), "dgain": (dy * xh).sum(1).to(out), "dbias": dy.sum(1).to(out)}


def _plain_linear(s):
    case, type = s["case"], s["x"].dtype
    z = torch.matmul(s["x"].float(), s["w"].float().transpose(1, 2))
    if s["b"] is not None:
        z = z + s["b"].float()[:, None]
    y = _act(case["act"], z)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(type), "z": z.to(type) if s["z"] is not None else None}


def _plain_linear_grad(s):
    case, type = s["case"], s["x"].dtype
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _act_slope(case["act"], s["z"].float())
    return {"dx": torch.matmul(dz, s["w"].float()).to(type), "dw": torch.matmul(dz.transpose(1, 2), s["x"].float()).to(type),
            "db": dz.sum(1).to(type) if s["b"] is not None else None}


def _plain_logprobs(s):
    x, k = s["logits"].float(), s["case"]["k"]
    m = x.amax(2, keepdim=True)
    empty = torch.isneginf(m)
    c = x - torch.where(empty, 0.0, m)
    e = torch.exp(c)
    total = e.sum(2, keepdim=True)
    shift = torch.where(empty, 0.0, m + torch.log(total))
    entropy = torch.where(empty, 0.0, torch.log(total) - torch.where(e > 0, c * e, 0.0).sum(2, keepdim=True) / total)[:, :, 0]
    tokens = s["tokens"].long()
    logp = torch.where(tokens < 0, 0.0, (x.gather(2, tokens.clamp(min=0)[:, :, None]) - shift)[:, :, 0])
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF) * (1 << 32) - torch.arange(x.shape[2], device=x.device)
    idx = order.topk(k, 2).indices                                 # equal logits: the lowest index first
    return {"logp": logp, "entropy": entropy, "top_logp": x.gather(2, idx) - shift, "top_idx": idx.int()}


def _plain_distill(s):
    case = s["case"]
    tau, w, idx = case["tau"], s["weight"][:, :, None], s["idx"].long()
    off = (w == 0) | (idx < 0).all(2, keepdim=True)
    there = (idx >= 0) & ~off
    at = idx.clamp(min=0)
    a = torch.where(there, s["top"] / tau, -math.inf)
    a = a - torch.where(off, 0.0, a.amax(2, keepdim=True))
    p = torch.exp(a)
    total = torch.where(off, 1.0, p.sum(2, keepdim=True))
    p, logp = p / total, a - torch.log(total)
    x = torch.where(off, 0.0, s["logits"].float() / tau)
    c = x - x.amax(2, keepdim=True)
    e = torch.exp(c)
    mass = e.sum(2, keepdim=True)
    logq = c.gather(2, at) - torch.log(mass)
    loss = (w * tau * tau * torch.where(there, p * (logp - logq), 0.0).sum(2, keepdim=True))[:, :, 0]
    grad = torch.where(off, 0.0, w * tau * (e / mass)).scatter_add_(2, at, torch.where(there, -w * tau * p, 0.0))
    return {"loss": loss, "dlogits": grad.to(s["logits"].dtype)}


_PLAIN = dict(norm=_plain_norm, norm_grad=_plain_norm_grad, linear=_plain_linear, linear_grad=_plain_linear_grad,
              logprobs=_plain_logprobs, distill=_plain_distill)


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if not own:
        return _PLAIN[kind](s)
    from paper_2002_01119_amd import layers
    if kind == "norm":
        layers.layer_norm(s["x"], s["gain"], s["bias"], s["y"], EPS, mean=s["mean"], rstd=s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if kind == "norm_grad":
        layers.layer_norm_grad(s["dy"], s["x"], s["gain"], s["mean"], s["rstd"], s["dx"], s["dgain"], s["dbias"], add=s["extra"])
        return {"dx": s["dx"], "dgain": s["dgain"], "dbias": s["dbias"]}
    if kind == "linear":
        layers.linear(s["x"], s["w"], s["y"], bias=s["b"], act=case["act"], residual=s["residual"], z=s["z"])
        return {"y": s["y"], "z": s["z"]}
    if kind == "linear_grad":
        layers.linear_grad(s["dy"], s["x"], s["w"], dx=s["dx"], dw=s["dw"], db=s["db"], act=case["act"], z=s["z"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if kind == "logprobs":
        layers.token_logprobs(s["logits"], s["tokens"], s["logp"], entropy=s["entropy"], top_logp=s["top_logp"], top_idx=s["top_idx"])
        return {"logp": s["logp"], "entropy": s["entropy"], "top_logp": s["top_logp"], "top_idx": s["top_idx"]}
    layers.distill(s["logits"], s["idx"], s["top"], s["loss"], tau=case["tau"], weight=s["weight"], dlogits=s["dlogits"])
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def _size_of(type):
    return 4 if type == F32 else 2


def work(case):
    n, t, kind, e = case["n"], case["t"], case["kind"], _size_of(case["type"])
    rows = n * t
    if kind == "norm":
        h = case["h"]
        return {"bytes": 2 * rows * h * e + 2 * n * h * _size_of(case["ptype"]) + 8 * rows, "flops": 8 * rows * h}
    if kind == "norm_grad":
        h = case["h"]
        return {"bytes": (4 if case["extra"] else 3) * rows * h * e + n * h * (_size_of(case["ptype"]) + 2 * _size_of(case["gtype"])) + 8 * rows,
                "flops": 14 * rows * h}
    if kind == "linear":
        i, o = case["i"], case["o"]
        outs = 1 + case["extra"] + case["save"]
        return {"bytes": e * (rows * i + n * o * i + outs * rows * o + (n * o if case["bias"] else 0)), "flops": 2 * rows * i * o}
    if kind == "linear_grad":
        i, o = case["i"], case["o"]
        ins = 1 + (case["act"] != "none")
        return {"bytes": e * (2 * rows * i + 2 * n * o * i + ins * rows * o + (n * o if case["bias"] else 0)), "flops": 4 * rows * i * o}
    v, k = case["v"], case["k"]
    if kind == "logprobs":
        return {"bytes": rows * (v * e + 12 + 8 * k), "flops": 5 * rows * v}
    return {"bytes": rows * (2 * v * e + 8 + 8 * k), "flops": 6 * rows * v}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _exact_norm(s):
    x, n, t = s["x"].double(), s["case"]["n"], s["case"]["t"]
    var, mean = torch.var_mean(x, 2, correction=0)
    if s["case"]["kind"] == "norm":
        rstd = 1.0 / torch.sqrt(var + EPS)
        y = torch.addcmul(s["bias"].double().view(n, 1, -1), (x - mean.view(n, t, 1)) * rstd.view(n, t, 1), s["gain"].double().view(n, 1, -1))
        return {"y": y, "mean": mean, "rstd": rstd}
    # the backward pass is given its statistics; d y_j / d x_i = rstd gain_j (delta_ij - 1/h - xh_i xh_j / h)
    r = s["rstd"].double().view(n, t, 1)
    xh = (x - s["mean"].double().view(n, t, 1)).mul_(r)
    dy = s["dy"].double()
    up = dy * s["gain"].double().view(n, 1, -1)
    along = torch.linalg.vecdot(up, xh).div_(x.shape[2]).view(n, t, 1)
    dx = (up - up.sum(2, keepdim=True) / x.shape[2]).sub_(along * xh).mul_(r)
    if s["extra"] is not None:
        dx += s["extra"].double()
    return {"dx": dx, "dgain": (xh * dy).sum(1), "dbias": dy.sum(1)}


def _exact_linear(s):
    act, x, w = s["case"]["act"], s["x"].double(), s["w"].double()
    z = s["z"].double() if s["case"]["kind"] == "linear_grad" and s["z"] is not None else None
    if s["case"]["kind"] == "linear":
        z = torch.stack([a @ m.t() for a, m in zip(x, w)])
        if s["b"] is not None:
            z += s["b"].double().unsqueeze(1)
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        y, slope = z * cdf, cdf + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    elif act == "silu":
        sig = torch.sigmoid(z)
        y, slope = z * sig, sig + z * sig * torch.sigmoid(-z)
    elif act == "relu":
        y, slope = z.clamp(min=0.0), torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    else:
        y, slope = z, None
    if s["case"]["kind"] == "linear":
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return {"y": y, "z": z if s["z"] is not None else None}
    dz = s["dy"].double() if slope is None else s["dy"].double() * slope
    return {"dx": torch.stack([a @ m for a, m in zip(dz, w)]), "dw": torch.stack([a.t() @ b for a, b in zip(dz, x)]),
            "db": dz.sum(1) if s["b"] is not None else None}


def _exact_logprobs(s):
    n, t, k = s["case"]["n"], s["case"]["t"], s["case"]["k"]
    out = {"logp": [], "entropy": [], "top_logp": []}
    for x, token in zip(s["logits"], s["tokens"].long()):
        lq = torch.log_softmax(x.double(), 1).nan_to_num_(nan=-math.inf, neginf=-math.inf)
        out["logp"].append(torch.where(token < 0, 0.0, lq[torch.arange(t, device=DEV), token.clamp(min=0)]))
        out["entropy"].append(torch.special.entr(torch.exp(lq)).sum(1))
        out["top_logp"].append(lq.topk(k, 1).values)
    return {**{name: torch.stack(v) for name, v in out.items()}, "top_idx": None}


def _exact_distill(s):
    case, tau = s["case"], s["case"]["tau"]
    losses, grads = [], []
    for x, idx, top, w in zip(s["logits"], s["idx"].long(), s["top"].double(), s["weight"].double()):
        live = (w != 0) & (idx >= 0).any(1)
        lq = torch.log_softmax(x[live].double() / tau, 1)
        gone = idx[live] < 0
        lp = torch.log_softmax(top[live].div(tau).masked_fill(gone, -math.inf), 1)
        p, at = torch.exp(lp), idx[live].masked_fill(gone, 0)
        loss = torch.zeros(case["t"], dtype=torch.float64, device=DEV)
        loss[live] = w[live] * tau ** 2 * (p * (lp - lq.gather(1, at))).masked_fill(gone, 0.0).sum(1)
        g = torch.exp(lq)
        g.scatter_add_(1, at, -p)
        grad = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
        grad[live] = g * (tau * w[live])[:, None]
        losses.append(loss)
        grads.append(grad)
    return {"loss": torch.stack(losses), "dlogits": torch.stack(grads)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(s)
    if case["kind"].startswith("linear"):
        return _exact_linear(s)
    return _exact_logprobs(s) if case["kind"] == "logprobs" else _exact_distill(s)
