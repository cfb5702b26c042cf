"""Plain 64-bit CPU forms of the learners' layers and losses, and how far a kernel that sums in fp32 may be from them.

Each function returns (values, bounds): the bound of an element is what the roundings of the kernel's arithmetic can add up to, from the
magnitudes of the terms that enter it.  U is half a unit in the last place of fp32 at 1; HALF of bf16.  A sum of m fp32 terms in any order is off by at
most m U times the sum of their magnitudes.
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
FEW = 16                # roundings of the few operations that follow a sum


def f64(t):
    return None if t is None else t.detach().cpu().double()


def rounded(values, bounds, dtype):
    """The bounds with the output's own rounding."""
    return bounds + HALF[dtype] * values.abs() + 1e-38


def layer_norm(x, gain, bias, eps, dtype):
    x, gain, bias = f64(x), f64(gain), f64(bias)
    c = x.shape[2]
    mean = x.mean(2, keepdim=True)
    d = x - mean
    var = d.square().mean(2, keepdim=True)
    rstd = (var + eps).rsqrt()
    b_mean = (c + FEW) * U * x.abs().mean(2, keepdim=True)
    # a mean that is off by b shifts every difference by b and, to first order, not the variance
    b_rstd = rstd * (((c + FEW) * U) + 0.5 * b_mean ** 2 * rstd ** 2 + b_mean * U * rstd)
    h = d * rstd
    y = h * gain[:, None] + (0.0 if bias is None else bias[:, None])
    b_y = (b_mean * rstd + d.abs() * b_rstd + FEW * U * (h.abs() + x.abs() * rstd)) * gain.abs()[:, None] + FEW * U * y.abs()
    if bias is not None:
        b_y = b_y + FEW * U * bias.abs()[:, None]
    return (y, mean[:, :, 0], rstd[:, :, 0]), (rounded(y, b_y, dtype), b_mean[:, :, 0] + 1e-38, b_rstd[:, :, 0])


def layer_norm_grad(dy, x, gain, mean, rstd, add, dtype, gtype):
    dy, x, gain, add = f64(dy), f64(x), f64(gain), f64(add)
    m, r = f64(mean)[:, :, None], f64(rstd)[:, :, None]
    t, c = x.shape[1:]
    h, u = (x - m) * r, dy * gain[:, None]
    b_h = FEW * U * (x.abs() + m.abs()) * r
    mu, muh = u.mean(2, keepdim=True), (u * h).mean(2, keepdim=True)
    b_mu = (c + FEW) * U * u.abs().mean(2, keepdim=True)
    b_muh = ((c + FEW) * U * (u * h).abs() + u.abs() * b_h).mean(2, keepdim=True)
    dx = r * (u - mu - h * muh)
    b_dx = r * (FEW * U * (u.abs() + mu.abs() + (h * muh).abs()) + b_mu + h.abs() * b_muh + b_h * muh.abs())
    if add is not None:
        dx, b_dx = dx + add, b_dx + FEW * U * (dx.abs() + add.abs())
    dg, db = (dy * h).sum(1), dy.sum(1)
    b_dg = ((t + FEW) * U * (dy * h).abs() + dy.abs() * b_h).sum(1)
    b_db = (t + FEW) * U * dy.abs().sum(1)
    return (dx, dg, db), (rounded(dx, b_dx, dtype), rounded(dg, b_dg, gtype), rounded(db, b_db, gtype))


def act(name, z):
    if name == "relu":
        return z.clamp(min=0.0)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z * math.sqrt(0.5))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def act_slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "silu":
        return torch.sigmoid(z) * (1.0 + z * torch.sigmoid(-z))
    return torch.ones_like(z)


STEEPEST = 1.2          # of the activations' slopes (GELU 1.13, SiLU 1.10)


def linear(x, w, bias, name, residual, dtype):
    x, w, bias, residual = f64(x), f64(w), f64(bias), f64(residual)
    k = x.shape[2]
    z, mag = torch.matmul(x, w.transpose(1, 2)), torch.matmul(x.abs(), w.abs().transpose(1, 2))
    b_z = (k + FEW) * U * mag
    if bias is not None:
        z, b_z = z + bias[:, None], b_z + FEW * U * bias.abs()[:, None]
    y = act(name, z)
    b_y = STEEPEST * b_z + FEW * U * (z.abs() + y.abs())
    if residual is not None:
        y, b_y = y + residual, b_y + FEW * U * residual.abs()
    return (y, z), (rounded(y, b_y, dtype), rounded(z, b_z, dtype))


def linear_grad(dy, x, w, name, z, dtype):
    dy, x, w, z = f64(dy), f64(x), f64(w), f64(z)
    t, o = dy.shape[1:]
    dz = dy if name == "none" else dy * act_slope(name, z)
    # the slope's own roundings: its terms (a probability and z times a density or another) are at most 2 together
    b_dz = torch.zeros_like(dz) if name == "none" else FEW * U * dy.abs() * 2.0
    b_in = b_dz if name == "none" else b_dz + HALF[dtype] * dz.abs()          # rounded where it enters the products
    dx, dw, db = torch.matmul(dz, w), torch.matmul(dz.transpose(1, 2), x), dz.sum(1)
    b_dx = torch.matmul(b_in, w.abs()) + (o + FEW) * U * torch.matmul(dz.abs(), w.abs())
    b_dw = torch.matmul(b_in.transpose(1, 2), x.abs()) + (t + FEW) * U * torch.matmul(dz.abs().transpose(1, 2), x.abs())
    b_db = b_dz.sum(1) + (t + FEW) * U * dz.abs().sum(1)
    return (dx, dw, db), tuple(rounded(v, b, dtype) for v, b in ((dx, b_dx), (dw, b_dw), (db, b_db)))


# A softmax's sum: the exponential of a difference c is off by about (4 + |c|) U relative to itself and |c| exp(c) <= 0.37 exp(0), terms beyond count
# nothing; a lane adds up to 256 terms in a row, lanes are joined by ten further sums.
SOFTMAX = 300 * U


def logprobs(logits, tokens, k):
    x, tokens = f64(logits), tokens.detach().cpu().long()
    m = x.amax(2, keepdim=True)
    empty, bad = torch.isneginf(m), torch.isnan(m) | torch.isposinf(m)
    lq = torch.log_softmax(x - torch.where(empty, 0.0, m), 2)          # differences first: at 1e38 a sum of logarithms is lost in 64 bits too
    lq = torch.where(empty, -math.inf, torch.where(bad, math.nan, lq))
    n, t, v = x.shape
    got = lq.gather(2, tokens.clamp(0, v - 1)[:, :, None])[:, :, 0]
    logp = torch.where(tokens < 0, 0.0, torch.where(tokens >= v, math.nan, got))
    entropy = torch.where(bad, math.nan, torch.special.entr(torch.exp(lq)).sum(2, keepdim=True))[:, :, 0]
    # NaN first, then larger ones, equal ones by column: a stable sort
    key = torch.where(torch.isnan(x), math.inf, torch.where(torch.isposinf(x), 1e300, x)) + 0.0
    idx = torch.sort(key, dim=2, descending=True, stable=True).indices[:, :, :k]
    top = lq.gather(2, idx)
    b = lambda v: SOFTMAX + FEW * U * (v.abs() + m[:, :, 0:1].reshape(n, t, *([1] * (v.dim() - 2))).abs())  # noqa: E731
    return (logp, entropy, top, idx), (b(logp), SOFTMAX * (2.0 + 2.0 * entropy), b(top))


def distill(logits, idx, top, weight, tau, dtype):
    x, idx, top = f64(logits), idx.detach().cpu().long(), f64(top)
    n, t, v = x.shape
    weight = torch.ones(n, t, dtype=torch.float64) if weight is None else f64(weight)
    there = (idx >= 0) & (idx < v) & ~torch.isneginf(top)
    live = (weight != 0) & there.any(2)
    at = idx.clamp(0, v - 1)
    lp = torch.log_softmax(torch.where(there, top / tau, -math.inf), 2)
    x = torch.where(live[:, :, None], x, 0.0)
    lq = torch.log_softmax(x / tau, 2)
    p = torch.where(there & live[:, :, None], torch.exp(lp), 0.0)
    term = torch.where(p > 0, p * (lp - lq.gather(2, at)), 0.0)
    w = torch.where(live, weight, 0.0)
    loss = w * tau * tau * term.sum(2)
    q = torch.exp(lq)
    given = torch.zeros_like(q).scatter_add_(2, at, p)
    grad = (w * tau)[:, :, None] * (q - given)
    grad = torch.where(live[:, :, None], grad, 0.0)
    c = (x.amax(2, keepdim=True) - x).clamp(max=1e4) / tau
    span = (torch.where(there, top.abs(), 0.0).amax(2, keepdim=True) / tau)
    b_loss = w.abs() * tau * tau * (torch.where(p > 0, p * (lp.abs() + lq.gather(2, at).abs() + span), 0.0).sum(2) * SOFTMAX + SOFTMAX)
    b_grad = (w.abs() * tau)[:, :, None] * (q * (SOFTMAX + FEW * U * c) + given * (SOFTMAX + FEW * U * span))
    return (loss, grad), (b_loss, rounded(grad, torch.where(live[:, :, None], b_grad, 0.0), dtype))


def assert_within(got, want, bound, what=""):
    got = f64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN elsewhere"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities"
    over = (got - want).abs()[fine] - bound.expand_as(want)[fine]
    assert not over.numel() or float(over.max()) <= 0.0, "%s: %g over its bound, %d of %d values" % (what, float(over.max()), int((over > 0).sum()), over.numel())
