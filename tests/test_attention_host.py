"""CPU-only checks of the attention blocks' boundary: what the header declares is exported and bound, and calls that cannot be honoured are refused before any
device is touched.  Addresses here are numbers that nothing dereferences."""
import ctypes
import os
import re

import pytest

from paper_2002_01119_amd import attention, layers, psgd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, I32 = layers.F32, layers.BF16, layers.I32
View, Cache = layers.View, attention.Cache


def test_every_declared_function_is_exported_and_bound():
    lib = attention.load()
    with open(os.path.join(ROOT, "include", "psgd_attention.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(psgd_[a-z0-9_]+)\s*\(", text)))
    assert declared == sorted(attention.EXPORTS)
    for name in declared:
        assert getattr(lib, name).argtypes is not None, name
    assert ctypes.sizeof(Cache) == 40


def place(k):
    return (1 << 40) + (k << 32)


def refused(rc, code, text):
    assert rc == code, (rc, psgd.last_error())
    assert text in psgd.last_error(), psgd.last_error()


N, T, HEADS, KV, HEAD = 2, 6, 4, 2, 8
CQ, CK = HEADS * HEAD, KV * HEAD


def wide(k, kind=F32):
    return View(place(k), T * CQ, CQ, kind)


def narrow(k, kind=F32):
    return View(place(k), T * CK, CK, kind)


def flat(k, kind=F32):
    return View(place(k), HEAD, 0, kind)


def qk(lib, heads=HEADS, kv=KV, head=HEAD, rotary=HEAD, pairs=0, base=10000.0, eps=1e-6, n=N, t=T, **over):
    v = dict(q=wide(1), k=narrow(2), positions=None, q_gain=flat(3), k_gain=flat(4), q_out=wide(5), k_out=narrow(6))
    v.update(over)
    return lib.psgd_qk_norm_rope(v["q"], v["k"], v["positions"], v["q_gain"], v["k_gain"], v["q_out"], v["k_out"], heads, kv, head, rotary, pairs, base, eps, n, t, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(n=0), psgd.EINVAL, "n=0"), (dict(n=513), psgd.EINVAL, "n=513"), (dict(t=-1), psgd.EINVAL, "negative"), (dict(t=1 << 31), psgd.EINVAL, "2^31"),
    (dict(head=0), psgd.EINVAL, "head=0"), (dict(head=257), psgd.EINVAL, "head=257"), (dict(heads=-1), psgd.EINVAL, "heads=-1"), (dict(heads=1 << 30), psgd.EINVAL, "2^31"),
    (dict(rotary=3), psgd.EINVAL, "rotary=3"), (dict(rotary=10), psgd.EINVAL, "rotary=10"), (dict(rotary=-2), psgd.EINVAL, "rotary=-2"), (dict(pairs=2), psgd.EINVAL, "pairs=2"),
    (dict(base=0.0), psgd.EINVAL, "base"), (dict(base=0.99), psgd.EINVAL, "base"), (dict(base=float("nan")), psgd.EINVAL, "base"), (dict(base=float("inf")), psgd.EINVAL, "base"), (dict(base=5e-324), psgd.EINVAL, "base"),
    (dict(eps=-1.0), psgd.EINVAL, "eps"), (dict(eps=float("inf")), psgd.EINVAL, "eps"), (dict(q=None), psgd.EINVAL, "null operand"), (dict(k_out=None), psgd.EINVAL, "null operand"),
    (dict(k_gain=None), psgd.EINVAL, "go together"), (dict(q=wide(1, BF16)), psgd.EINVAL, "alike"), (dict(k=narrow(2, I32)), psgd.EINVAL, "alike"),
    (dict(q_gain=flat(3, BF16)), psgd.EINVAL, "alike"), (dict(q_gain=flat(3, I32), k_gain=flat(4, I32)), psgd.EINVAL, "alike"),
    (dict(positions=View(place(7), 6, 1, F32)), psgd.EINVAL, "int32"), (dict(positions=View(place(7) + 2, 6, 1, I32)), psgd.EALIGN, "positions"),
    (dict(positions=View(None, 6, 1, I32)), psgd.EINVAL, "null"), (dict(q=View(place(1) + 1, T * CQ, CQ, F32)), psgd.EALIGN, "q is not aligned"),
    (dict(k=View(place(2), -1, CK, F32)), psgd.EINVAL, "negative"), (dict(q_out=View(place(5), T * CQ, CQ - 1, F32)), psgd.EALIAS, "rows of the output q_out"),
    (dict(q_out=View(place(1) + 4, T * CQ, CQ, F32)), psgd.EALIAS, "q_out overlaps q"), (dict(k_out=wide(1)), psgd.EALIAS, "k_out overlaps q"),
    (dict(k_out=View(place(5) + 64, T * CK, CK, F32)), psgd.EALIAS, "q_out overlaps k_out"), (dict(q_out=wide(3)), psgd.EALIAS, "q_out overlaps q_gain"),
])
def test_qk_norm_rope_refusals(change, code, text):
    refused(qk(attention.load(), **change), code, text)


def qk_grad(lib, heads=HEADS, kv=KV, n=N, t=T, workspace=1 << 61, size=1 << 20, **over):
    v = dict(dq_out=wide(1), dk_out=narrow(2), q=wide(3), k=narrow(4), positions=None, q_gain=flat(5), k_gain=flat(6), dq=wide(7), dk=narrow(8), dq_gain=flat(9), dk_gain=flat(10))
    v.update(over)
    return lib.psgd_qk_norm_rope_grad(v["dq_out"], v["dk_out"], v["q"], v["k"], v["positions"], v["q_gain"], v["k_gain"], v["dq"], v["dk"], v["dq_gain"], v["dk_gain"],
                                      heads, kv, HEAD, HEAD, 0, 10000.0, 1e-6, n, t, workspace, size, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(q=None), psgd.EINVAL, "null operand"), (dict(dk=None), psgd.EINVAL, "null operand"), (dict(workspace=None), psgd.EINVAL, "workspace"),
    (dict(size=64), psgd.EINVAL, "workspace"), (dict(workspace=(1 << 61) + 8), psgd.EINVAL, "workspace"), (dict(dq_gain=flat(9, BF16)), psgd.EINVAL, "alike"),
    (dict(dq=wide(3)), psgd.EALIAS, "dq overlaps q"), (dict(dq=View(place(1) + 8, T * CQ, CQ, F32)), psgd.EALIAS, "dq overlaps dq_out"),
    (dict(dk_gain=flat(9)), psgd.EALIAS, "dq_gain overlaps dk_gain"), (dict(dq_gain=flat(5)), psgd.EALIAS, "dq_gain overlaps q_gain"),
    (dict(dk=wide(7)), psgd.EALIAS, "dq overlaps dk"), (dict(workspace=place(3)), psgd.EALIAS, "workspace overlaps q"), (dict(dq_gain=View(place(9), 4, 0, F32)), psgd.EALIAS, "rows of the output dq_gain"),
])
def test_qk_norm_rope_grad_refusals(change, code, text):
    refused(qk_grad(attention.load(), **change), code, text)


def forward(lib, heads=HEADS, kv=KV, head=HEAD, window=0, sinks=0, scale=0.5, sequences=0, n=N, t=T, lse=1 << 60, **over):
    v = dict(q=wide(1), k=narrow(2), v=narrow(3), starts=None, out=wide(4))
    v.update(over)
    return lib.psgd_attention(v["q"], v["k"], v["v"], v["starts"], v["out"], lse, heads, kv, head, window, sinks, scale, sequences, n, t, None)


STARTS = View(place(9), 3, 0, I32)
SHAPE = [
    (dict(n=0), psgd.EINVAL, "n=0"), (dict(t=-1), psgd.EINVAL, "negative"), (dict(t=(1 << 31) - 5), psgd.EINVAL, "2^31"), (dict(kv=3), psgd.EINVAL, "kv=3"), (dict(kv=0), psgd.EINVAL, "kv=0"),
    (dict(heads=0), psgd.EINVAL, "heads=0"), (dict(head=0), psgd.EINVAL, "head=0"), (dict(head=257), psgd.EINVAL, "head=257"), (dict(window=-1), psgd.EINVAL, "window=-1"),
    (dict(sinks=-1, window=5), psgd.EINVAL, "sinks=-1"), (dict(sinks=2), psgd.EINVAL, "window=0 with sinks=2"), (dict(scale=float("nan")), psgd.EINVAL, "scale"),
    (dict(scale=float("inf")), psgd.EINVAL, "scale"), (dict(sequences=-1), psgd.EINVAL, "sequences=-1"), (dict(sequences=2), psgd.EINVAL, "without starts"),
    (dict(starts=STARTS), psgd.EINVAL, "sequences=0 with starts"), (dict(starts=View(place(9), 3, 0, F32), sequences=2), psgd.EINVAL, "int32"),
    (dict(starts=View(place(9) + 2, 3, 0, I32), sequences=2), psgd.EALIGN, "starts"), (dict(k=narrow(2, BF16)), psgd.EINVAL, "alike"), (dict(q=None), psgd.EINVAL, "null operand"),
    (dict(v=View(None, T * CK, CK, F32)), psgd.EINVAL, "null pointer"), (dict(q=View(place(1), T * CQ, -CQ, F32)), psgd.EINVAL, "negative"),
]


@pytest.mark.parametrize("change,code,text", SHAPE + [
    (dict(out=wide(1)), psgd.EALIAS, "out overlaps q"), (dict(out=View(place(4), T * CQ, 8, F32)), psgd.EALIAS, "rows of the output out"), (dict(lse=place(1)), psgd.EALIAS, "lse overlaps q"),
    (dict(lse=place(4)), psgd.EALIAS, "out overlaps lse"), (dict(out=View(place(9), T * CQ, CQ, F32), starts=STARTS, sequences=2), psgd.EALIAS, "out overlaps starts"),
    (dict(lse=(1 << 60) + 2), psgd.EALIGN, "lse"),
])
def test_attention_refusals(change, code, text):
    refused(forward(attention.load(), **change), code, text)


def backward(lib, heads=HEADS, kv=KV, head=HEAD, window=0, sinks=0, scale=0.5, sequences=0, n=N, t=T, lse=1 << 60, workspace=1 << 61, size=1 << 20, **over):
    v = dict(dout=wide(10), q=wide(1), k=narrow(2), v=narrow(3), starts=None, out=wide(4), dq=wide(11), dk=narrow(12), dv=narrow(13))
    v.update(over)
    return lib.psgd_attention_grad(v["dout"], v["q"], v["k"], v["v"], v["out"], lse, v["starts"], v["dq"], v["dk"], v["dv"], heads, kv, head, window, sinks, scale, sequences,
                                   n, t, workspace, size, None)


@pytest.mark.parametrize("change,code,text", SHAPE + [
    (dict(lse=None), psgd.EINVAL, "lse is needed"), (dict(workspace=None), psgd.EINVAL, "workspace"), (dict(size=100), psgd.EINVAL, "workspace"),
    (dict(workspace=(1 << 61) + 16), psgd.EINVAL, "workspace"), (dict(dq=wide(10)), psgd.EALIAS, "dq overlaps dout"), (dict(dk=narrow(2)), psgd.EALIAS, "dk overlaps k"),
    (dict(dv=narrow(12)), psgd.EALIAS, "dk overlaps dv"), (dict(workspace=place(11)), psgd.EALIAS, "workspace overlaps dq"), (dict(dk=View(place(11) + 4, T * CK, CK, F32)), psgd.EALIAS, "dq overlaps dk"),
])
def test_attention_grad_refusals(change, code, text):
    refused(backward(attention.load(), **change), code, text)


def test_gradients_side_by_side_in_one_array_are_apart():
    """Column slices of one [n, t, (heads + 2 kv) head] array: no overlap, so the refusal is another."""
    w = CQ + 2 * CK
    rc = backward(attention.load(), dq=View(place(11), T * w, w, F32), dk=View(place(11) + 4 * CQ, T * w, w, F32), dv=View(place(11) + 4 * (CQ + CK), T * w, w, F32), workspace=None)
    refused(rc, psgd.EINVAL, "workspace")


B, SLOTS = 3, 10


def cache(k, kind=F32):
    return Cache(place(k), B * SLOTS * CK, SLOTS * CK, CK, kind)


def step(lib, heads=HEADS, kv=KV, head=HEAD, window=0, sinks=0, scale=0.5, n=N, b=B, slots=SLOTS, **over):
    v = dict(q=View(place(1), B * CQ, CQ, F32), k=View(place(2), B * CK, CK, F32), v=View(place(3), B * CK, CK, F32), ck=cache(4), cv=cache(5), lengths=View(place(6), B, 1, I32),
             out=View(place(7), B * CQ, CQ, F32))
    v.update(over)
    return lib.psgd_attention_step(v["q"], v["k"], v["v"], v["ck"], v["cv"], v["lengths"], v["out"], heads, kv, head, window, sinks, scale, n, b, slots, None, 0, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(n=0), psgd.EINVAL, "n=0"), (dict(b=-1), psgd.EINVAL, "negative"), (dict(kv=3), psgd.EINVAL, "kv=3"), (dict(head=300), psgd.EINVAL, "head=300"), (dict(slots=0), psgd.EINVAL, "slots=0"),
    (dict(slots=(1 << 30) + 1), psgd.EINVAL, "slots"), (dict(sinks=1), psgd.EINVAL, "sinks=1"), (dict(window=-2), psgd.EINVAL, "window=-2"), (dict(scale=float("nan")), psgd.EINVAL, "scale"),
    (dict(lengths=View(place(6), B, 1, F32)), psgd.EINVAL, "int32"), (dict(lengths=None), psgd.EINVAL, "null operand"), (dict(ck=cache(4, BF16)), psgd.EINVAL, "alike"),
    (dict(b=1 << 30, n=512), psgd.EINVAL, "n * b * heads"), (dict(ck=Cache(None, 240, 80, 16, F32)), psgd.EINVAL, "cache_k is a null"), (dict(cv=Cache(place(5) + 1, 480, 160, 16, F32)), psgd.EALIGN, "cache_v"),
    (dict(cv=Cache(place(5), 480, -160, 16, F32)), psgd.EINVAL, "negative"), (dict(ck=Cache(place(4), 480, 160, 15, F32)), psgd.EALIAS, "rows of cache_k"),
    (dict(ck=Cache(place(4), 0, 160, 16, F32)), psgd.EALIAS, "rows of cache_k"), (dict(ck=Cache(place(4), 1 << 50, 160, 16, F32)), psgd.EINVAL, "too large"),
    (dict(cv=cache(4)), psgd.EALIAS, "cache_k overlaps cache_v"), (dict(cv=Cache(place(4) + 4 * 8, 480, 160, 16, F32)), psgd.EALIAS, "cache_k overlaps cache_v"),
    (dict(out=View(place(4), B * CQ, CQ, F32)), psgd.EALIAS, "overlaps out"), (dict(out=View(place(1), B * CQ, CQ, F32)), psgd.EALIAS, "out overlaps q"), (dict(q=View(place(4), 0, 0, F32)), psgd.EALIAS, "cache_k overlaps q"),
])
def test_attention_step_refusals(change, code, text):
    refused(step(attention.load(), **change), code, text)


@pytest.mark.parametrize("strides,apart,meet", [
    ((960, 320, 32), 16, False), ((960, 320, 32), 15, True), ((960, 320, 32), 17, True),             # rows side by side
    ((960, 32, 96), 16, False), ((32, 64, 320), 16, False), ((32, 64, 320), 8, True),                # sequences or learners innermost
    ((960, 320, 16), 160, False), ((960, 320, 16), 144, True),                                      # a sequence's keys, then its values
])
def test_caches_between_each_others_rows(strides, apart, meet):
    lib = attention.load()
    rc = step(lib, ck=Cache(place(4), *strides, F32), cv=Cache(place(4) + 4 * apart, *strides, F32), out=View(place(4), B * CQ, CQ, F32))
    refused(rc, psgd.EALIAS, "cache_k overlaps cache_v") if meet else refused(rc, psgd.EALIAS, "cache_k overlaps out")


def dropout(lib, p=0.5, n=N, t=T, c=8, step_dev=None, **over):
    v = dict(x=View(place(1), T * 8, 8, F32), residual=None, y=View(place(2), T * 8, 8, F32))
    v.update(over)
    return lib.psgd_dropout(v["x"], v["residual"], v["y"], p, 1, 2, step_dev, n, t, c, None)


@pytest.mark.parametrize("change,code,text", [
    (dict(p=-0.1), psgd.EINVAL, "p="), (dict(p=1.1), psgd.EINVAL, "p="), (dict(p=float("nan")), psgd.EINVAL, "p="), (dict(n=0), psgd.EINVAL, "n=0"), (dict(c=-1), psgd.EINVAL, "negative"),
    (dict(n=512, t=1 << 23), psgd.EINVAL, "n * t"), (dict(x=None), psgd.EINVAL, "null operand"), (dict(y=View(place(2), T * 8, 8, BF16)), psgd.EINVAL, "alike"),
    (dict(residual=View(place(3), T * 8, 8, I32)), psgd.EINVAL, "alike"), (dict(y=View(place(1) + 4, T * 8, 8, F32)), psgd.EALIAS, "y overlaps x"),
    (dict(residual=View(place(2) + 4, T * 8, 8, F32)), psgd.EALIAS, "y overlaps residual"), (dict(y=View(place(2), T * 8, 7, F32)), psgd.EALIAS, "rows of the output y"),
    (dict(step_dev=(1 << 50) + 4), psgd.EALIGN, "step_dev"), (dict(step_dev=place(2) + 8), psgd.EALIAS, "y overlaps step_dev"),
])
def test_dropout_refusals(change, code, text):
    refused(dropout(attention.load(), **change), code, text)


def test_workspaces_of_nothing():
    lib = attention.load()
    assert lib.psgd_qk_norm_rope_grad_workspace(0, 1, 64) == 0 and lib.psgd_qk_norm_rope_grad_workspace(1, 1, 257) == 0
    assert lib.psgd_qk_norm_rope_grad_workspace(4, 10, 100) % 256 == 0 and lib.psgd_qk_norm_rope_grad_workspace(4, 10, 100) >= 4 * 2 * 100 * 4
    assert lib.psgd_attention_grad_workspace(4, 2, 64, 0, 0, 0, 0, 5) == 0 and lib.psgd_attention_grad_workspace(4, 2, 64, 0, 0, 0, 2, 0) == 0
    assert lib.psgd_attention_grad_workspace(4, 2, 64, 0, 0, 0, 2, 100) >= 2 * 4 * 100 * 4
    big = 2 ** 31 - 1                                      # sizes that would overflow, each refused before they are multiplied
    for sizes in ((big, big, 64, 0, 0, 0, 256, 5), (4, 2, 64, -1, 0, 0, 2, 100), (4, 2, 64, 0, 3, 0, 2, 100), (4, 2, 64, 8, 1, big, 2, 100), (4, 2, 64, 8, 1, 1, 2, big),
                  (1 << 22, 1 << 22, 1, 1 << 15, 1 << 15, 1 << 20, 512, 1 << 16)):
        assert lib.psgd_attention_grad_workspace(*sizes) == 0
    assert 0 < lib.psgd_attention_grad_workspace(1 << 10, 1 << 10, 256, 1 << 15, 1 << 15, 1 << 20, 1, 1 << 16) < 1 << 40
    assert lib.psgd_attention_step_workspace(4, 2, 64, 0, 0, 1, 0, 9) == 0 and lib.psgd_attention_step_workspace(4, 2, 64, 0, 0, 1, 1, 1 << 31) == 0


def test_binding_refuses_host_tensors_and_shapes():
    torch = pytest.importorskip("torch")
    q, k, g = torch.zeros(2, 3, 32), torch.zeros(2, 3, 16), torch.zeros(2, 8)
    with pytest.raises(ValueError, match="GPU"):
        attention.qk_norm_rope(q, k, q, k, 4, 2)
    for bad in (dict(heads=5), dict(heads=0), dict(kv=3), dict(k=q), dict(q_gain=g[:, :7], k_gain=g), dict(positions=torch.zeros(2, 3)), dict(positions=torch.zeros(2, 4, dtype=torch.int32)),
                dict(q=q.double()), dict(q_out=torch.zeros(2, 3, 31)), dict(q=torch.zeros(2, 32, 3).transpose(1, 2)), dict(pairs="other"), dict(k=None)):
        with pytest.raises(ValueError):
            attention.qk_norm_rope(**{**dict(q=q, k=k, q_out=q, k_out=k, heads=4, kv=2), **bad})
    starts = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        attention.attention(q, k, k, q.clone(), 4, 2, starts=starts)
    for bad in (dict(lse=torch.zeros(2, 4)), dict(lse=torch.zeros(2, 4, 3).double()), dict(starts=starts.long()), dict(starts=starts[:1]), dict(starts=starts[:, :1]), dict(out=k), dict(v=None)):
        with pytest.raises(ValueError):
            attention.attention(**{**dict(q=q, k=k, v=k, out=q, heads=4, kv=2), **bad})
    c = torch.zeros(2, 3, 9, 16)
    lengths = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        attention.attention_step(q, k, k, c, c.clone(), lengths, q.clone(), 4, 2)
    for bad in (dict(cache_k=c[0]), dict(cache_k=c[:, :, :8]), dict(cache_v=c[:, :2]), dict(cache_k=c.double()), dict(cache_v=torch.zeros(2, 3, 16, 9).transpose(2, 3)), dict(lengths=lengths.long()),
                dict(lengths=lengths[:, :2]), dict(cache_k=c[:, :, :0], cache_v=c[:, :, :0])):
        with pytest.raises(ValueError):
            attention.attention_step(**{**dict(q=q, k=k, v=k, cache_k=c, cache_v=c, lengths=lengths, out=q, heads=4, kv=2), **bad})
    with pytest.raises(ValueError, match="GPU"):
        attention.dropout(q, q, 0.5, 1)
    for bad in (dict(y=k), dict(residual=k), dict(x=q[0])):
        with pytest.raises(ValueError):
            attention.dropout(**{**dict(x=q, y=q, p=0.5, seed=1), **bad})
