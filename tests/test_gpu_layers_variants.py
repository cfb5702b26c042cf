"""Every kernel, tile and way of cutting a product that the layers' and losses' launch rules can choose, against their formulas in 64 bits, at sizes that nothing
divides (layers_shapes.py says what each runs, and test_layers_plan.py that it does)."""
import pytest

torch = pytest.importorskip("torch")
import layers_shapes as shapes  # noqa: E402
from oracle import layers_oracle as orc  # noqa: E402
from test_gpu_linear import layer, layers, rows, untouched  # noqa: E402, F401
from test_gpu_tokens import gen, logits_of, teacher, tokens_of  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DTYPE = {2: BF16, 4: F32}


def listed(table):
    return [pytest.param(DTYPE[size], *shape, id="%s-%s" % ("-".join(map(str, shape)), said.replace(" ", "-"))) for size in (2, 4) for shape, said in table[size]]


@pytest.mark.parametrize("dtype,n,t,i,o", listed(shapes.LINEAR))
def test_forward(layers, dtype, n, t, i, o):  # noqa: F811
    pitch, lead, off = (3, 1, 5) if (i + o) % 2 else (0, 0, 0)
    flat, w, b = layer(n, i, o, dtype, 1, off)
    x, r = rows(n, t, i, dtype, 3, pitch, lead), rows(n, t, o, dtype, 4, pitch)
    whole_y, whole_z = (torch.full((n, t, o + 2), 7.0, dtype=dtype, device="cuda:0") for _ in range(2))
    y, z = whole_y[:, :, 1:o + 1], whole_z[:, :, 1:o + 1]
    layers.linear(x, w, y, bias=b, act="gelu", residual=r, z=z)
    torch.cuda.synchronize()
    want, bound = orc.linear(x, w, b, "gelu", r, dtype)
    orc.assert_within(y, want[0], bound[0], "y")
    orc.assert_within(z, want[1], bound[1], "z")
    for whole in (whole_y, whole_z):        # nothing beside the columns is written
        assert (whole[:, :, 0] == 7.0).all() and (whole[:, :, o + 1] == 7.0).all()


@pytest.mark.parametrize("dtype,n,t,i,o", listed(shapes.GRAD))
def test_backward(layers, dtype, n, t, i, o):  # noqa: F811
    pitch, lead, off = (3, 1, 5) if (i + o) % 2 else (0, 0, 0)
    _, w, _ = layer(n, i, o, dtype, 1, off)
    x, dy, z = rows(n, t, i, dtype, 3, pitch, lead), rows(n, t, o, dtype, 4, pitch, lead), rows(n, t, o, dtype, 5, pitch)
    whole = torch.full((n, t, i + 2), 7.0, dtype=dtype, device="cuda:0")
    dx = whole[:, :, 1:i + 1]
    grads, dw, db = layer(n, i, o, dtype, None, off)
    layers.linear_grad(dy, x, w, dx=dx, dw=dw, db=db, act="silu", z=z)
    torch.cuda.synchronize()
    want, bound = orc.linear_grad(dy, x, w, "silu", z, dtype)
    for got, v, e, what in zip((dx, dw, db), want, bound, ("dx", "dw", "db")):
        orc.assert_within(got, v, e, what)
    untouched(grads, dw, db, off)
    assert (whole[:, :, 0] == 7.0).all() and (whole[:, :, i + 1] == 7.0).all()


def shared(count):
    """(learners, rows of a learner) of about `count` rows in all, few enough of a learner for a 64-bit form of them; the learners share their inputs."""
    return (count // 5, 5) if count >= 100 else (1, count)


@pytest.mark.parametrize("dtype,count,v,k", listed(shapes.LOGPROBS))
def test_logprobs(layers, dtype, count, v, k):  # noqa: F811
    n, t = shared(count)
    one, tokens = logits_of(1, t, v, dtype, v, 3, 1), tokens_of(1, t, v, 1)
    one[0, 1 % t] = one[0, 1 % t].round()                   # long runs of equal logits
    new = lambda *shape, kind=F32: torch.full(shape, 7, dtype=kind, device="cuda:0")  # noqa: E731
    logp, ent, top, idx = new(n, t), new(n, t), new(n, t, k), new(n, t, k, kind=torch.int32)
    layers.token_logprobs(one.expand(n, t, v), tokens.expand(n, t), logp, entropy=ent, top_logp=top, top_idx=idx)
    torch.cuda.synchronize()
    (w_logp, w_ent, w_top, w_idx), (b_logp, b_ent, b_top) = orc.logprobs(one, tokens, k)
    orc.assert_within(logp[:1], w_logp, b_logp, "logp")
    orc.assert_within(ent[:1], w_ent, b_ent, "entropy")
    assert torch.equal(idx[:1].cpu().long(), w_idx), "top_idx"
    orc.assert_within(top[:1], w_top, b_top, "top_logp")
    assert all(torch.equal(out, out[:1].expand_as(out)) for out in (logp, ent, top, idx))


@pytest.mark.parametrize("dtype,count,v,gradient", listed(shapes.DISTILL))
def test_distill(layers, dtype, count, v, gradient):  # noqa: F811
    n, t = (count // 4, 4) if count >= 100 else (1, count)
    k, tau = 16, 2.0
    one = logits_of(1, t, v, dtype, v, 3, 1)
    idx, top = teacher(1, t, v, k, 5, 0.1)
    weight = torch.rand((1, t), generator=gen(9)).to("cuda:0")
    loss = torch.full((n, t), 7.0, device="cuda:0")
    whole = torch.full((n, t, v + 2), 7.0, dtype=dtype, device="cuda:0") if gradient else None
    grad = whole[:, :, 1:v + 1] if gradient else None
    layers.distill(one.expand(n, t, v), idx.expand(n, t, k), top.expand(n, t, k), loss, tau=tau, weight=weight.expand(n, t).contiguous(), dlogits=grad)
    torch.cuda.synchronize()
    (w_loss, w_grad), (b_loss, b_grad) = orc.distill(one, idx, top, weight, tau, dtype)
    orc.assert_within(loss[:1], w_loss, b_loss, "loss")
    assert torch.equal(loss, loss[:1].expand_as(loss))
    if gradient:
        orc.assert_within(grad[:1], w_grad, b_grad, "dlogits")
        assert torch.equal(grad, grad[:1].expand_as(grad))
        assert (whole[:, :, 0] == 7.0).all() and (whole[:, :, v + 1] == 7.0).all()
