"""CPU-only checks of the layers' boundary: what the header declares is exported and bound, and calls that cannot be honoured are refused before
any device is touched.  Addresses here are numbers that nothing dereferences."""
import ctypes
import os
import re

import pytest

from paper_2002_01119_amd import layers, psgd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, I32 = layers.F32, layers.BF16, layers.I32


def test_every_declared_function_is_exported_and_bound():
    lib = layers.load()
    with open(os.path.join(ROOT, "include", "psgd_layers.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(psgd_[a-z0-9_]+)\s*\(", text)))
    assert declared == sorted(layers.EXPORTS)
    for name in declared:
        assert getattr(lib, name).argtypes is not None, name


class At:
    """Operands at made-up addresses, a mebi apart unless said otherwise."""

    def __init__(self):
        self.next = 1 << 40

    def __call__(self, learner, row=0, kind=F32, data=None):
        if data is None:
            data, self.next = self.next, self.next + (1 << 30)
        return layers.View(data, learner, row, kind)


def refused(rc, code, text):
    assert rc == code, (rc, psgd.last_error())
    assert text in psgd.last_error(), psgd.last_error()


N, T, C = 2, 3, 8
MEAN, RSTD = 1 << 60, (1 << 60) + 4096


def norm(lib, x=None, g=None, b=None, y=None, mean=MEAN, rstd=RSTD, n=N, t=T, c=C, eps=1e-5):
    at = At()
    x, g, y = x or at(T * C, C), g or at(C), y or at(T * C, C)
    return lib.psgd_layer_norm(x, g, b, y, mean, rstd, n, t, c, eps, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(n=0), psgd.EINVAL, "n=0"), (dict(n=513), psgd.EINVAL, "n=513"), (dict(t=-1), psgd.EINVAL, "negative"),
    (dict(c=1 << 31), psgd.EINVAL, "2^31"), (dict(eps=-1.0), psgd.EINVAL, "eps"), (dict(eps=float("nan")), psgd.EINVAL, "eps"),
    (dict(mean=None), psgd.EINVAL, "go together"),
    (dict(x=layers.View(1 << 40, 24, 8, BF16)), psgd.EINVAL, "alike"), (dict(x=layers.View(1 << 40, 24, 8, I32)), psgd.EINVAL, "alike"),
    (dict(g=layers.View(1 << 40, 8, 0, I32)), psgd.EINVAL, "gain"), (dict(b=layers.View(1 << 41, 8, 0, BF16)), psgd.EINVAL, "alike"),
    (dict(x=layers.View(None, 24, 8, F32)), psgd.EINVAL, "null"), (dict(x=layers.View((1 << 40) + 2, 24, 8, F32)), psgd.EALIGN, "aligned"),
    (dict(x=layers.View(1 << 50, -24, 8, F32)), psgd.EINVAL, "negative"), (dict(x=layers.View(1 << 40, 1 << 48, 8, F32)), psgd.EINVAL, "too large"),
    (dict(y=layers.View(1 << 50, 24, 0, F32)), psgd.EALIAS, "rows of the output y"), (dict(y=layers.View(1 << 50, 0, 8, F32)), psgd.EALIAS, "rows of the output y"),
    (dict(y=layers.View((1 << 40) + 4, 24, 8, F32)), psgd.EALIAS, "y overlaps x"), (dict(y=layers.View((1 << 40) + (1 << 30), 24, 8, F32)), psgd.EALIAS, "y overlaps gain"),
    (dict(mean=(1 << 40) + 8), psgd.EALIAS, "mean overlaps x"), (dict(rstd=MEAN + 4), psgd.EALIAS, "mean overlaps rstd"),
])
def test_layer_norm_refusals(change, code, text):
    refused(norm(layers.load(), **change), code, text)


def norm_grad(lib, n=N, t=T, c=C, workspace=1 << 61, size=1 << 20, **over):
    at = At()
    v = dict(dy=at(T * C, C), x=at(T * C, C), gain=at(C), add=None, dx=at(T * C, C), dgain=at(C), dbias=at(C))
    v.update(over)
    return lib.psgd_layer_norm_grad(v["dy"], v["x"], v["gain"], MEAN, RSTD, v["add"], v["dx"], v["dgain"], v["dbias"], n, t, c, workspace, size, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(workspace=None), psgd.EINVAL, "workspace"), (dict(size=64), psgd.EINVAL, "workspace"), (dict(workspace=(1 << 61) + 8), psgd.EINVAL, "workspace"),
    (dict(dx=layers.View((1 << 40) + 32, 24, 8, F32)), psgd.EALIAS, "dx overlaps dy"),
    (dict(dx=layers.View((1 << 40) + (1 << 30), 24, 8, F32)), psgd.EALIAS, "dx overlaps x"),
    (dict(dgain=layers.View(1 << 50, 0, 0, F32)), psgd.EALIAS, "rows of the output dgain"),
    (dict(dgain=layers.View(1 << 50, 20, 0, F32), dbias=layers.View((1 << 50) + 28, 20, 0, F32)), psgd.EALIAS, "dgain overlaps dbias"),
    (dict(dbias=layers.View(1 << 50, 8, 0, BF16)), psgd.EINVAL, "alike"), (dict(workspace=1 << 40), psgd.EALIAS, "workspace overlaps dy"),
])
def test_layer_norm_grad_refusals(change, code, text):
    refused(norm_grad(layers.load(), **change), code, text)


def test_layers_in_the_rows_of_one_array_are_apart():
    """Gradients of gain and bias side by side in one row, learners a row apart: no overlap, so the refusal is another."""
    rc = norm_grad(layers.load(), dgain=layers.View(1 << 50, 20, 0, F32), dbias=layers.View((1 << 50) + 32, 20, 0, F32), workspace=None)
    refused(rc, psgd.EINVAL, "workspace")


def linear(lib, act=0, n=N, t=T, i=4, o=5, workspace=None, size=0, **over):
    at = At()
    v = dict(x=at(T * 4, 4), w=at(20, 4), bias=None, residual=None, y=at(T * 5, 5), z=None)
    v.update(over)
    return lib.psgd_linear(v["x"], v["w"], v["bias"], v["residual"], v["y"], v["z"], act, n, t, i, o, workspace, size, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(act=4), psgd.EINVAL, "act=4"), (dict(act=-1), psgd.EINVAL, "act=-1"), (dict(n=0), psgd.EINVAL, "n=0"), (dict(i=-4), psgd.EINVAL, "negative"),
    (dict(w=layers.View(1 << 50, 20, 4, BF16)), psgd.EINVAL, "alike"), (dict(bias=layers.View(1 << 50, 5, 0, I32)), psgd.EINVAL, "alike"),
    (dict(y=layers.View(1 << 50, 15, 4, F32)), psgd.EALIAS, "rows of the output y"), (dict(y=layers.View(1 << 40, 15, 5, F32)), psgd.EALIAS, "y overlaps x"),
    (dict(z=layers.View((1 << 40) + 2 * (1 << 30), 15, 5, F32)), psgd.EALIAS, "z overlaps y"),
    (dict(residual=layers.View((1 << 40) + 2 * (1 << 30) + 4, 15, 5, F32)), psgd.EALIAS, "y overlaps residual"),
    (dict(x=layers.View((1 << 50) + 1, 12, 4, F32)), psgd.EALIGN, "x is not aligned"),
])
def test_linear_refusals(change, code, text):
    refused(linear(layers.load(), **change), code, text)


def linear_grad(lib, act=0, n=N, t=T, i=4, o=5, **over):
    at = At()
    v = dict(dy=at(T * 5, 5), z=None, x=at(T * 4, 4), w=at(20, 4), dx=at(T * 4, 4), dw=at(20, 4), db=at(5))
    v.update(over)
    return lib.psgd_linear_grad(v["dy"], v["z"], v["x"], v["w"], v["dx"], v["dw"], v["db"], act, n, t, i, o, None, 0, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(act=2), psgd.EINVAL, "z is needed"), (dict(dx=layers.View(1 << 40, 12, 4, F32)), psgd.EALIAS, "dx overlaps dy"),
    (dict(dw=layers.View(1 << 50, 0, 4, F32)), psgd.EALIAS, "rows of the output dw"), (dict(db=layers.View(1 << 50, 4, 0, F32)), psgd.EALIAS, "rows of the output db"),
    (dict(dw=layers.View(1 << 50, 24, 4, F32), db=layers.View((1 << 50) + 76, 24, 0, F32)), psgd.EALIAS, "dw overlaps db"),
    (dict(db=layers.View(1 << 50, 5, 0, BF16)), psgd.EINVAL, "alike"),
])
def test_linear_grad_refusals(change, code, text):
    refused(linear_grad(layers.load(), **change), code, text)


V, K = 50, 4
OUT = 1 << 60


def logprobs(lib, n=N, t=T, v=V, k=K, logp=OUT, entropy=OUT + 1024, top=OUT + 2048, idx=OUT + 8192, **over):
    at = At()
    o = dict(logits=at(T * V, V), tokens=at(T, 1, I32))
    o.update(over)
    return lib.psgd_token_logprobs(o["logits"], o["tokens"], logp, entropy, top, idx, k, n, t, v, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(k=65), psgd.EINVAL, "k=65"), (dict(k=-1), psgd.EINVAL, "k=-1"), (dict(v=3), psgd.EINVAL, "k=4"), (dict(v=0, k=0), psgd.EINVAL, "no column"),
    (dict(k=0), psgd.EINVAL, "go with k"), (dict(idx=None), psgd.EINVAL, "go with k"), (dict(logp=None), psgd.EINVAL, "logp is needed"),
    (dict(tokens=layers.View(1 << 50, 3, 1, F32)), psgd.EINVAL, "int32"), (dict(n=512, t=1 << 23), psgd.EINVAL, "n * t"),
    (dict(entropy=OUT), psgd.EALIAS, "entropy overlaps logp"), (dict(logp=1 << 40), psgd.EALIAS, "logp overlaps logits"),
    (dict(idx=OUT + 2049), psgd.EALIGN, "top_idx is not aligned"),
])
def test_token_logprobs_refusals(change, code, text):
    refused(logprobs(layers.load(), **change), code, text)


def distill(lib, n=N, t=T, v=V, k=K, tau=1.0, loss=OUT, weight=None, **over):
    at = At()
    o = dict(logits=at(T * V, V), idx=at(T * K, K, I32), top=at(T * K, K), dlogits=at(T * V, V))
    o.update(over)
    return lib.psgd_distill(o["logits"], o["idx"], o["top"], weight, loss, o["dlogits"], tau, k, n, t, v, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(k=0), psgd.EINVAL, "k=0"), (dict(k=1025), psgd.EINVAL, "k=1025"), (dict(tau=0.0), psgd.EINVAL, "tau"), (dict(tau=-1.0), psgd.EINVAL, "tau"),
    (dict(tau=float("inf")), psgd.EINVAL, "tau"), (dict(tau=float("nan")), psgd.EINVAL, "tau"), (dict(tau=1e-45), psgd.EINVAL, "tau"),
    (dict(loss=None), psgd.EINVAL, "loss is needed"),
    (dict(idx=layers.View(1 << 50, 12, 4, F32)), psgd.EINVAL, "int32"), (dict(top=layers.View(1 << 50, 12, 4, BF16)), psgd.EINVAL, "float"),
    (dict(dlogits=layers.View(1 << 50, 150, 50, BF16)), psgd.EINVAL, "alike"), (dict(dlogits=layers.View((1 << 40) + 4, 150, 50, F32)), psgd.EALIAS, "dlogits overlaps logits"),
    (dict(dlogits=layers.View(1 << 50, 150, 40, F32)), psgd.EALIAS, "rows of the output dlogits"), (dict(weight=OUT), psgd.EALIAS, "loss overlaps weight"),
])
def test_distill_refusals(change, code, text):
    refused(distill(layers.load(), **change), code, text)


def test_workspaces_of_nothing():
    lib = layers.load()
    assert lib.psgd_layer_norm_grad_workspace(0, 1, 1) == 0 and lib.psgd_layer_norm_grad_workspace(1, 1, 0) == 0
    assert lib.psgd_layer_norm_grad_workspace(4, 10, 100) % 256 == 0 and lib.psgd_layer_norm_grad_workspace(4, 10, 100) >= 4 * 2 * 100 * 4


def test_binding_refuses_host_tensors_and_shapes():
    torch = pytest.importorskip("torch")
    x, g = torch.zeros(2, 3, 8), torch.zeros(2, 8)
    with pytest.raises(ValueError, match="GPU"):
        layers.layer_norm(x, g, None, torch.zeros(2, 3, 8))
    for bad in (dict(x=torch.zeros(3, 8)), dict(gain=torch.zeros(8)), dict(y=torch.zeros(2, 3, 9)), dict(x=x.double()), dict(mean=torch.zeros(2, 3).double()),
                dict(x=torch.zeros(2, 8, 3).transpose(1, 2)), dict(x=None)):
        with pytest.raises(ValueError):
            layers.layer_norm(**{**dict(x=x, gain=g, bias=None, y=torch.zeros(2, 3, 8)), **bad})
    w, y = torch.zeros(2, 5, 8), torch.zeros(2, 3, 5)
    with pytest.raises(ValueError, match="act"):
        layers.linear(x, w, y, act="tanh")
    for bad in (dict(w=torch.zeros(2, 5, 7)), dict(w=torch.zeros(1, 5, 8)), dict(y=torch.zeros(2, 3, 4)), dict(z=torch.zeros(2, 3, 4)), dict(workspace=torch.zeros(4))):
        with pytest.raises(ValueError):
            layers.linear(**{**dict(x=x, w=w, y=y), **bad})
    logp, tok = torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32)
    for bad in (dict(tokens=tok.long()), dict(tokens=tok[:, :2]), dict(logp=torch.zeros(6, 1)[:5]), dict(top_logp=torch.zeros(2, 3, 4))):
        with pytest.raises(ValueError):
            layers.token_logprobs(**{**dict(logits=x, tokens=tok, logp=logp), **bad})
    idx, top = torch.zeros(2, 3, 4, dtype=torch.int32), torch.zeros(2, 3, 4)
    for bad in (dict(top_idx=idx[:, :, 0]), dict(top_logit=top[:, :, :2]), dict(loss=torch.zeros(5)), dict(dlogits=torch.zeros(2, 3, 7))):
        with pytest.raises(ValueError):
            layers.distill(**{**dict(logits=x, top_idx=idx, top_logit=top, loss=logp), **bad})
    assert ctypes.sizeof(layers.View) == 32
