"""Layers and losses where they went wrong once: rows that hold NaN, sizes of zero, activations far from zero, teachers and temperatures at the ends of float."""
import math

import pytest

torch = pytest.importorskip("torch")
from oracle import layers_oracle as orc  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = math.inf, math.nan
DEV = "cuda:0"


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_01119_amd import layers as m
    m.load()
    torch.cuda.set_device(0)
    m.psgd.device_status()
    return m


def normal(shape, dtype, seed, sigma=1.0):
    return torch.empty(shape).normal_(0.0, sigma, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


# v: one lane's groups, several lanes, every number of lanes a row takes, rows with the batches' maxima left out
@pytest.mark.parametrize("v", [1, 5, 700, 5003, 40000, 400003])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_in_the_first_column_is_an_alternative(layers, dtype, v):
    """NaN counts as the largest, equal ones by ascending column: column 0 too, and a row of nothing but NaN."""
    n, t, k = 1, 5, min(v, 7)
    x = normal((n, t, v), dtype, v)
    x[0, 0, 0] = NAN
    x[0, 1] = NAN
    x[0, 2, 0] = x[0, 2, v - 1] = NAN
    x[0, 3, v // 2:] = -INF
    x[0, 3, 0] = NAN
    x[0, 4, 0] = INF
    tokens = torch.zeros((n, t), dtype=torch.int32, device=DEV)
    logp, ent = torch.empty((n, t), device=DEV), torch.empty((n, t), device=DEV)
    top, idx = torch.full((n, t, k), 7.0, device=DEV), torch.full((n, t, k), -7, dtype=torch.int32, device=DEV)
    layers.token_logprobs(x, tokens, logp, entropy=ent, top_logp=top, top_idx=idx)
    (w_logp, w_ent, w_top, w_idx), _ = orc.logprobs(x, tokens, k)
    assert torch.equal(idx.cpu().long(), w_idx)
    assert idx[0, 0, 0] == 0 and idx[0, 1].tolist() == list(range(k))
    assert torch.isnan(logp).all() and torch.isnan(ent).all() and torch.isnan(top).all()


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,i,o", [(3, 4, 0), (3, 0, 5), (0, 4, 5), (3, 0, 0), (0, 0, 5), (0, 4, 0), (40, 70, 0)])
def test_gradients_of_layers_with_sizes_of_zero(layers, act, dtype, t, i, o):
    """What is summed over nothing is zero, what has no element is left alone."""
    n = 2
    x, w = normal((n, t, i), dtype, 1), normal((n, o, i), dtype, 2)
    dy, z = normal((n, t, o), dtype, 3), normal((n, t, o), dtype, 4)
    full = lambda *shape: torch.full(shape, 7.0, dtype=dtype, device=DEV)  # noqa: E731
    y, zz, b = full(n, t, o), full(n, t, o), normal((n, o), dtype, 5)
    layers.linear(x, w, y, bias=b, act=act, z=zz)
    dx, dw, db = full(n, t, i), full(n, o, i), full(n, o)
    for asked in (dict(dx=dx, dw=dw, db=db), dict(dx=dx), dict(dw=dw), dict(db=db), {}):
        layers.linear_grad(dy, x, w, act=act, z=z if act != "none" else None, **asked)
    torch.cuda.synchronize()
    want, _ = orc.linear_grad(dy, x, w, act, z, dtype)
    for got, v in ((dx, want[0]), (dw, want[1])):
        assert torch.equal(orc.f64(got), v)
    bound = orc.linear_grad(dy, x, w, act, z, dtype)[1][2]
    orc.assert_within(db, want[2], bound, "db")
    assert layers.psgd.device_status() == 0


def grid(dtype, low, high):
    """Every sixteenth of a binary order from 2^-20 up, both signs, and steps of 2^-8 through the range; in the type."""
    k = torch.arange(16 * 20, dtype=torch.float64)
    fine = 2.0 ** (k / 16 - 20)
    z = torch.cat([fine, -fine, torch.arange(low, high, 2.0 ** -8, dtype=torch.float64), torch.zeros(1, dtype=torch.float64)])
    return z.to(dtype).to(DEV)


def of_kernels(layers, z, act, t):
    """act(z) by the forward pass and its slope by db of dy = 1, one token (t = 1) or one of the tiles' rows."""
    o = z.numel()
    x, w = torch.zeros((1, t, 1), dtype=z.dtype, device=DEV), torch.zeros((1, o, 1), dtype=z.dtype, device=DEV)
    y, db = torch.empty((1, t, o), dtype=z.dtype, device=DEV), torch.empty((1, o), dtype=z.dtype, device=DEV)
    layers.linear(x, w, y, bias=z[None], act=act)
    one = torch.ones((1, 1, o), dtype=z.dtype, device=DEV)
    layers.linear_grad(one, x[:, :1], w, db=db, act=act, z=z[None, None])
    torch.cuda.synchronize()
    assert all(torch.equal(y[0, 0].nan_to_num(7.0), r.nan_to_num(7.0)) for r in y[0])
    return orc.f64(y[0, 0]), orc.f64(db[0])


@pytest.mark.parametrize("t", [1, 9])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gelu_is_exact_to_a_few_places_everywhere(layers, dtype, t):
    """In float, from its operations: Phi to 12 U (a complementary error function of 8 U, its argument's two roundings, which z^2 multiplies), the
    density to (z^2 + 12) U.  In bf16 the terms may be off by 2^-12 of themselves, a sixteenth of what rounding the output costs."""
    z = grid(dtype, -14.0, 14.0)
    y, slope = of_kernels(layers, z, "gelu", t)
    z = orc.f64(z)
    phi = 0.5 * torch.special.erfc(-z * math.sqrt(0.5))
    density = z.abs() * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    off = orc.U if dtype == F32 else 0.0
    part = 0.0 if dtype == F32 else 2.0 ** -12
    b_phi, b_density = phi * (part + off * (12 + 2 * z * z)), density * (part + off * (12 + z * z))
    want, want_slope = orc.act("gelu", z), orc.act_slope("gelu", z)
    orc.assert_within(y, want, z.abs() * b_phi + 4 * off * want.abs() + orc.HALF[dtype] * want.abs() + 1e-36, "gelu")
    orc.assert_within(slope, want_slope, b_phi + b_density + 4 * off * want_slope.abs() + orc.HALF[dtype] * want_slope.abs() + 1e-36, "its slope")


@pytest.mark.parametrize("t", [1, 9])
def test_silu_of_floats_is_exact_to_a_few_places_everywhere(layers, t):
    """The exponential to 2 U, the sum, the quotient and the product to U each; what 1 - p of the slope loses is of p, not of itself."""
    z = grid(F32, -100.0, 100.0)
    y, slope = of_kernels(layers, z, "silu", t)
    z = orc.f64(z)
    p = torch.sigmoid(z)
    want, want_slope = orc.act("silu", z), orc.act_slope("silu", z)
    orc.assert_within(y, want, 8 * orc.U * want.abs() + 1e-36, "silu")
    orc.assert_within(slope, want_slope, 8 * orc.U * (want_slope.abs() + 2 * p * (1 + z.abs() * (p + torch.sigmoid(-z)))) + 1e-36, "its slope")


def check_distill(layers, x, idx, top, weight, tau):
    n, t, v = x.shape
    loss, alone, grad = torch.full((n, t), 7.0, device=DEV), torch.full((n, t), 7.0, device=DEV), torch.full((n, t, v), 7.0, dtype=x.dtype, device=DEV)
    layers.distill(x, idx, top, loss, tau=tau, weight=weight, dlogits=grad)
    layers.distill(x, idx, top, alone, tau=tau, weight=weight)
    torch.cuda.synchronize()
    (w_loss, w_grad), (b_loss, b_grad) = orc.distill(x, idx, top, weight, tau, x.dtype)
    return loss, alone, grad, w_loss, b_loss, w_grad, b_grad


# one way of holding a row after the other; the last is read again
@pytest.mark.parametrize("dtype,v", [(F32, 100), (BF16, 5003), (F32, 33001), (BF16, 140001)])
@pytest.mark.parametrize("tau", [0.5, 0.7, 3.0])
def test_a_teacher_at_the_ends_of_float(layers, dtype, v, tau):
    """Slots of the lowest and of the largest float are slots, also where dividing them by the temperature leaves the type: a teacher of nothing
    but the lowest value is uniform."""
    n, t, k = 1, 4, 6
    x = normal((n, t, v), dtype, 1)
    idx = torch.arange(3, 3 + k, dtype=torch.int32, device=DEV).expand(n, t, k).contiguous()
    top = normal((n, t, k), F32, 2)
    low = torch.finfo(F32).min
    top[0, 0] = low
    top[0, 1] = -low
    top[0, 2, 2:] = low
    idx[0, 3, 1:] = -1
    top[0, 3] = low
    loss, alone, grad, _, _, _, _ = check_distill(layers, x, idx, top, None, tau)
    # the same distributions from teachers in the middle of the range
    mild = top.clone()
    mild[0, 0] = mild[0, 1] = 0.0
    mild[0, 2, 2:] = -1e4
    mild[0, 3] = 0.0
    _, _, _, w_loss, b_loss, w_grad, b_grad = check_distill(layers, x, idx, mild, None, tau)
    orc.assert_within(loss, w_loss, b_loss, "loss")
    orc.assert_within(alone, w_loss, b_loss, "loss alone")
    orc.assert_within(grad, w_grad, b_grad, "dlogits")
    assert loss[0, 0] > 0.0 and grad[0, 3, 3] < 0.0


@pytest.mark.parametrize("dtype,v", [(F32, 100), (F32, 70001), (BF16, 140001)])
@pytest.mark.parametrize("tau", [1e28, 1e30, 1e35])
def test_masked_columns_at_a_very_high_temperature(layers, dtype, v, tau):
    """All that is not masked is alike then; a masked column stays out."""
    n, t, k = 1, 2, 4
    x = normal((n, t, v), dtype, 1)
    x[0, :, v // 3:] = -INF
    idx = torch.arange(1, 1 + k, dtype=torch.int32, device=DEV).expand(n, t, k).contiguous()
    top, weight = normal((n, t, k), F32, 2), torch.full((n, t), 1e-20, device=DEV)
    loss, alone, grad, w_loss, b_loss, w_grad, b_grad = check_distill(layers, x, idx, top, weight, tau)
    live = v // 3
    assert torch.isposinf(w_loss).all() or torch.allclose(w_loss, torch.full_like(w_loss, float(weight[0, 0]) * tau * tau * math.log(live / k)), rtol=1e-6)
    for got in (loss, alone):
        got = orc.f64(got)
        assert torch.equal(torch.isposinf(got), w_loss > torch.finfo(F32).max)
        fine = torch.isfinite(got)
        assert ((got - w_loss).abs() <= b_loss)[fine].all()
    orc.assert_within(grad, w_grad, b_grad, "dlogits")
    assert not grad[0, :, live:].any()


@pytest.mark.parametrize("tau", [2.0 ** -128, 4.0e-39, 2.0 ** -127])
def test_temperatures_whose_reciprocal_leaves_float_with_its_logarithms_base(layers, tau):
    """Refused, or right: 1 / tau may be a number where log2(e) / tau is none."""
    x = normal((1, 1, 50), F32, 1)
    idx, top = torch.tensor([[[3]]], dtype=torch.int32, device=DEV), torch.zeros((1, 1, 1), device=DEV)
    loss, grad = torch.empty((1, 1), device=DEV), torch.empty_like(x)
    try:
        layers.distill(x, idx, top, loss, tau=tau, dlogits=grad)
    except layers.psgd.PsgdError as e:
        assert "tau" in str(e)
        return
    assert not torch.isnan(loss).any() and not torch.isnan(grad).any()


@pytest.mark.parametrize("t", [1, 9])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_a_residual_that_cancels_the_activation(layers, act, dtype, t):
    """What is left is the activation's own error, which 32 bits hold to a few units of z whatever the output's type: 16 U |z|, as everywhere."""
    z = grid(dtype, -8.0, 8.0)
    o = z.numel()
    x, w = torch.zeros((1, t, 1), dtype=dtype, device=DEV), torch.zeros((1, o, 1), dtype=dtype, device=DEV)
    value = orc.act(act, orc.f64(z))
    r = (-value).to(dtype).to(DEV)
    y = torch.empty((1, t, o), dtype=dtype, device=DEV)
    layers.linear(x, w, y, bias=z[None], act=act, residual=r.expand(1, t, o))
    torch.cuda.synchronize()
    want = value + orc.f64(r)
    orc.assert_within(y[0, 0], want, orc.rounded(want, 16 * orc.U * orc.f64(z).abs(), dtype), "what is left")


# A launch counts its work items along one axis in 32 bits; what is beyond was never started, and nobody said so.
def all_alike(out, first):
    assert torch.equal(out, first.expand_as(out))


def test_more_rows_of_logits_than_one_launch_counts(layers):
    n, t, v = 512, (1 << 17) + 3, 8                             # 2^26 rows at four a workgroup of 256 are 2^32 work items
    x = normal((1, t, v), BF16, 1)
    tokens = (torch.arange(t, device=DEV) % v).int()[None]
    one, all_of = (torch.full((k, t), 7.0, device=DEV) for k in (1, n))
    layers.token_logprobs(x, tokens, one)
    layers.token_logprobs(x.expand(n, t, v), tokens.expand(n, t), all_of)
    all_alike(all_of, one)
    idx, top = tokens[:, :, None], torch.zeros((1, t, 1), device=DEV)
    grads = [torch.full((k, t, v), 7.0, dtype=BF16, device=DEV) for k in (1, n)]
    for k, loss, grad in zip((1, n), (one, all_of), grads):
        loss.fill_(7.0)
        layers.distill(x.expand(k, t, v), idx.expand(k, t, 1), top.expand(k, t, 1), loss, dlogits=grad)
    all_alike(all_of, one)
    all_alike(grads[1], grads[0])
    del grads
    all_of.fill_(7.0)
    layers.distill(x.expand(n, t, v), idx.expand(n, t, 1), top.expand(n, t, 1), all_of)
    all_alike(all_of, one)


def test_more_alternatives_rows_than_one_launch_counts(layers):
    n, t, v, k = 512, (1 << 15) + 1, 1028, 33                   # 2^24 rows of a workgroup of 256 each
    x, tokens = normal((1, t, v), BF16, 1), torch.zeros((1, t), dtype=torch.int32, device=DEV)
    outs = []
    for m in (1, n):
        logp, top, idx = torch.full((m, t), 7.0, device=DEV), torch.full((m, t, k), 7.0, device=DEV), torch.full((m, t, k), -7, dtype=torch.int32, device=DEV)
        layers.token_logprobs(x.expand(m, t, v), tokens.expand(m, t), logp, top_logp=top, top_idx=idx)
        outs.append((logp, top, idx))
    for one, all_of in zip(*outs):
        all_alike(all_of, one)



def test_more_tiles_than_one_launch_counts(layers):
    n, many, few = 512, (1 << 21) + 70, 20                      # 2^24 tiles of 64 x 64 and a workgroup of 256 each
    x, w = normal((1, many, 8), BF16, 1), normal((1, 1, 8), BF16, 2)
    bias = normal((1, 1), BF16, 3)
    ys = [torch.full((k, many, 1), 7.0, dtype=BF16, device=DEV) for k in (1, n)]
    for k, y in zip((1, n), ys):
        layers.linear(x.expand(k, many, 8), w.expand(k, 1, 8), y, bias=bias.expand(k, 1), act="silu")
    all_alike(ys[1], ys[0])
    del ys
    dy = normal((1, many, 1), BF16, 4)
    dxs = [torch.full((k, many, 1), 7.0, dtype=BF16, device=DEV) for k in (1, n)]
    for k, dx in zip((1, n), dxs):
        layers.linear_grad(dy.expand(k, many, 1), x[:, :, :1].expand(k, many, 1), w[:, :, :1].expand(k, 1, 1), dx=dx)
    all_alike(dxs[1], dxs[0])
    del dxs
    dy, x = normal((1, few, many), BF16, 5), normal((1, few, 1), BF16, 6)
    dws = [torch.full((k, many, 1), 7.0, dtype=BF16, device=DEV) for k in (1, n)]
    for k, dw in zip((1, n), dws):
        layers.linear_grad(dy.expand(k, few, many), x.expand(k, few, 1), w[:, :, :1].expand(k, many, 1), dw=dw)
    all_alike(dws[1], dws[0])


def test_more_outputs_of_one_token_than_one_launch_counts(layers):
    o = (1 << 28) + 100                                         # sixteen outputs a workgroup of 256; 64 sums of db a workgroup of 1024
    x, w = normal((1, 1, 8), BF16, 1), normal((1, 1, 8), BF16, 2).expand(1, o, 8)
    bias = normal((1, o), BF16, 3)
    y = torch.full((1, 1, o), 7.0, dtype=BF16, device=DEV)
    layers.linear(x, w, y, bias=bias)
    start = o - (1 << 20)
    for a, b in ((0, 1 << 20), (start, o)):                      # the first and the last, against a call for them alone
        part = torch.empty((1, 1, b - a), dtype=BF16, device=DEV)
        layers.linear(x, w[:, a:b], part, bias=bias[:, a:b])
        assert torch.equal(y[:, :, a:b], part)
    db = torch.full((1, o), 7.0, dtype=BF16, device=DEV)
    layers.linear_grad(y, x, w, db=db)
    assert torch.equal(db, y[:, 0])



def test_more_columns_of_a_norm_than_one_launch_counts(layers):
    c = (1 << 27) + 72                                           # 64 sums of dgain or dbias a workgroup of 1024
    x = normal((1, 1, 1024), BF16, 1).repeat(1, 1, c // 1024 + 1)[:, :, :c]
    mean, rstd = torch.zeros((1, 1), device=DEV), torch.ones((1, 1), device=DEV)
    gain = torch.ones((1, 1), dtype=BF16, device=DEV).expand(1, c).contiguous()
    dx, dgain, dbias = torch.empty_like(x), torch.full((1, c), 7.0, dtype=BF16, device=DEV), torch.full((1, c), 7.0, dtype=BF16, device=DEV)
    layers.layer_norm_grad(x, x, gain, mean, rstd, dx, dgain, dbias)
    assert torch.equal(dbias, x[:, 0])
    assert torch.equal(dgain, (x[:, 0].float() ** 2).to(BF16))
