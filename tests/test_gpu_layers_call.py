"""The layers' binding: the extension's short way against the long one, and what the short way does not answer."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_01119_amd import layers as m
    torch.cuda.set_device(0)
    m.load()
    assert m._short("layer_norm") is False and m._ext is not None       # bound; a call without arguments is not answered
    return m


def both(layers, monkeypatch, f):
    got = []
    for short in (True, False):
        with monkeypatch.context() as m:
            if not short:
                m.setattr(layers, "_short", lambda *a: False)
            else:
                real, answers = layers._short, []
                m.setattr(layers, "_short", lambda *a: answers.append(real(*a)) or answers[-1])
            out = f()
            torch.cuda.synchronize()
            got.append([v.clone() for v in out])
            if short:
                assert answers == [True] * len(answers) and answers
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,t", [(2, 3), (1, 1), (3, 70)])
def test_both_ways_give_the_same(layers, monkeypatch, dtype, n, t):
    g = torch.Generator(device="cuda:0").manual_seed(1)
    new = lambda *shape: torch.empty(shape, device="cuda:0").normal_(generator=g).to(dtype)  # noqa: E731
    out = lambda *shape, kind=dtype: torch.zeros(shape, device="cuda:0", dtype=kind)  # noqa: E731
    c, o, k = 136, 72, 5
    x, gain, bias, dy, w = new(n, t, c), new(n, c), new(n, c), new(n, t, c), new(n, o, c)
    mean, rstd = out(n, t, kind=F32), out(n, t, kind=F32)

    def norm():
        y = out(n, t, c)
        layers.layer_norm(x, gain, bias, y, 1e-5, mean=mean, rstd=rstd)
        return y, mean, rstd

    def norm_grad():
        dx, dg, db = out(n, t, c), out(n, c), out(n, c)
        layers.layer_norm_grad(dy, x, gain, mean, rstd, dx, dg, db, add=dy)
        return dx, dg, db

    def linear():
        y, z = out(n, t, o), out(n, t, o)
        layers.linear(x, w, y, bias=new(1, o).expand(n, o) * 0, act="gelu", residual=y * 0, z=z)
        return y, z

    def linear_grad():
        dx, dw, db = out(n, t, c), out(n, o, c), out(n, o)
        layers.linear_grad(x[:, :, :o], x, w, dx=dx, dw=dw, db=db, act="silu", z=x[:, :, o:2 * o] if 2 * o <= c else x[:, :, c - o:])
        return dx, dw, db

    def logprobs():
        logp, ent, top, idx = out(n, t, kind=F32), out(n, t, kind=F32), out(n, t, k, kind=F32), out(n, t, k, kind=torch.int32)
        layers.token_logprobs(x, torch.full((n, t), 3, dtype=torch.int32, device="cuda:0"), logp, entropy=ent, top_logp=top, top_idx=idx)
        return logp, ent, top, idx

    def distill():
        loss, d = out(n, t, kind=F32), out(n, t, c)
        idx = torch.arange(k, dtype=torch.int32, device="cuda:0").expand(n, t, k).contiguous()
        layers.distill(x, idx, idx.float(), loss, tau=2.0, weight=torch.ones((n, t), device="cuda:0"), dlogits=d)
        return loss, d

    for f in (norm, norm_grad, linear, linear_grad, logprobs, distill):
        both(layers, monkeypatch, f)


def test_what_is_not_in_order_is_refused_as_without_it(layers):
    x, gain = torch.zeros((2, 3, 8), device="cuda:0"), torch.ones((2, 8), device="cuda:0")
    y = torch.empty_like(x)
    with pytest.raises(ValueError, match="shape"):
        layers.layer_norm(x, gain[:1], None, y)
    with pytest.raises(ValueError, match="unit stride"):
        layers.layer_norm(x, gain.t().contiguous().t(), None, y)
    with pytest.raises(ValueError):
        layers.layer_norm(x.double(), gain, None, y)
    with pytest.raises(ValueError):
        layers.layer_norm(x.cpu(), gain, None, y)
    with pytest.raises(layers.psgd.PsgdError, match="overlap"):
        layers.layer_norm(x, gain, None, y.as_strided((2, 3, 8), (24, 4, 1)))
    with pytest.raises(layers.psgd.PsgdError, match="alike"):
        layers.layer_norm(x, gain, None, y.to(BF16))
    with pytest.raises(layers.psgd.PsgdError, match="eps"):
        layers.layer_norm(x, gain, None, y, -1.0)
    layers.layer_norm(x, gain, None, y, 1)                        # a whole number for eps goes the long way
    w = torch.zeros((2, 5, 8), device="cuda:0")
    with pytest.raises(layers.psgd.PsgdError, match="workspace"):
        layers.linear(torch.zeros((2, 17, 30000), device="cuda:0"), torch.zeros((2, 5, 30000), device="cuda:0"), torch.empty((2, 17, 5), device="cuda:0"),
                      workspace=torch.empty(16, dtype=torch.uint8, device="cuda:0"))
    with pytest.raises(layers.psgd.PsgdError, match="z is needed"):
        layers.linear_grad(torch.zeros((2, 3, 5), device="cuda:0"), x, w, dx=y, act="relu")
    with pytest.raises(layers.psgd.PsgdError, match="overlaps"):
        layers.linear(x, w, x[:, :, :5])
    with pytest.raises(layers.psgd.PsgdError, match="tau"):
        layers.distill(x, torch.zeros((2, 3, 1), dtype=torch.int32, device="cuda:0"), torch.zeros((2, 3, 1), device="cuda:0"), torch.empty((2, 3), device="cuda:0"), tau=0.0)
    torch.cuda.synchronize()
    assert layers.psgd.device_status() == 0
