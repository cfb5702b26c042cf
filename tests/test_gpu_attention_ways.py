"""Ways that the attention blocks' calls can go beside the usual one: tiles straight to LDS or through registers, the binding's short way or its long one, two calls at
the same time, a process's first calls inside a captured graph, arrays whose offsets pass 32 bits."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
from oracle import attention_oracle as orc  # noqa: E402
from test_gpu_attention import check, cuts, normal, within  # noqa: E402
import test_gpu_attention_step as step_tests  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16, NAN = torch.float32, torch.bfloat16, float("nan")


@pytest.fixture(scope="module")
def attention():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_01119_amd import attention as m
    m.load()
    torch.cuda.set_device(0)
    return m


def slices(n, t, heads, kv, head, dtype, lead, seed=None):
    """q, k and v of one array that begins `lead` elements behind a multiple of 16 bytes."""
    width = (heads + 2 * kv) * head
    a = torch.full((lead + n * t * width,), NAN, dtype=dtype, device="cuda:0")[lead:].view(n, t, width)
    if seed is not None:
        a.copy_(normal(a.shape, dtype, seed))
    return (a,) + a.split((heads * head, kv * head, kv * head), 2)


@pytest.mark.parametrize("t,window,sinks", [(300, 0, 0), (700, 90, 5)])
@pytest.mark.parametrize("head", [16, 32, 64, 96, 128, 136, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_either_way_to_the_tiles(attention, t, window, sinks, head, dtype):
    """Which way a tile goes depends on alignment alone, and what comes out does not: the same bits, parts of tiles and first tokens' among them."""
    n, heads, kv = 2, 4, 2
    starts = cuts([[0, t - 50, t], [3, 3, t - 1]])
    dout = normal((n, t, heads * head), dtype, 2)
    got = []
    for lead in (0, 1):
        _, q, k, v = slices(n, t, heads, kv, head, dtype, lead, 1)
        out, lse = torch.full((n, t, heads * head), NAN, dtype=dtype, device="cuda:0"), torch.full((n, heads, t), NAN, device="cuda:0")
        d, dq, dk, dv = slices(n, t, heads, kv, head, dtype, lead)
        attention.attention(q, k, v, out, heads, kv, lse=lse, starts=starts, window=window, sinks=sinks)
        attention.attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, starts=starts, window=window, sinks=sinks)
        got.append([torch.nan_to_num(x, 777.0) for x in (out, lse, d)])
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("head", [16, 32, 64, 96, 128, 136, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_either_way_to_the_steps_tiles(attention, head, dtype):
    n, b, heads, kv, slots = 1, 3, 6, 2, 700
    lengths = cuts([[650, 31, 699]])
    q, k, v = normal((n, b, heads * head), dtype, 1), normal((n, b, kv * head), dtype, 2), normal((n, b, kv * head), dtype, 3)
    got = []
    for lead in (0, 1):
        ck, cv = (torch.empty(lead + n * b * slots * kv * head, dtype=dtype, device="cuda:0")[lead:].view(n, b, slots, kv * head) for _ in range(2))
        ck.copy_(normal(ck.shape, dtype, 4))
        cv.copy_(normal(cv.shape, dtype, 5))
        out = torch.empty((n, b, heads * head), dtype=dtype, device="cuda:0")
        attention.attention_step(q, k, v, ck, cv, lengths, out, heads, kv)
        got.append((out, ck.clone(), cv.clone()))
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("n", [15, 16])
@pytest.mark.parametrize("lead", [0, 1])
@pytest.mark.parametrize("head", [24, 64, 80, 128, 144])
def test_tiles_of_either_height(attention, head, lead, n):
    """16 heads of 260 tokens are 720 tiles of 128 rows for 15 learners, which go in tiles of half of them, and 768 for 16, which go whole."""
    starts = cuts([[0, 64 + i, 120, 120, 259] for i in range(n)])
    check(attention, n, 260, 16, 2, head, BF16, window=100, sinks=3, starts=starts, lead=lead, backward=False)


def test_short_way_and_long_way(attention, monkeypatch):
    """Every call makes the same bits either way, and the short way is the one that is taken."""
    n, t, heads, kv, head, slots = 2, 90, 4, 2, 32, 40
    _, q, k, v = slices(n, t, heads, kv, head, BF16, 0, 1)
    pos, starts, lengths = torch.arange(n * t, dtype=torch.int32, device="cuda:0").view(n, t), cuts([[0, 30, 90], [5, 5, 80]]), cuts([[3, 39], [-1, 70]])
    gq, gk = normal((n, head), F32, 6), normal((n, head), F32, 7)
    counter = torch.tensor([3], device="cuda:0")

    def calls(**more):
        new = lambda like: torch.full_like(like, NAN)  # noqa: E731
        made = {}
        qr, kr, dqr, dkr = new(q.contiguous()), new(k.contiguous()), new(q.contiguous()), new(k.contiguous())
        attention.qk_norm_rope(q, k, qr, kr, heads, kv, positions=pos, q_gain=gq, k_gain=gk, eps=1e-5, rotary=16, base=1e5, pairs="neighbours", **more)
        dgq, dgk = new(gq), new(gk)
        attention.qk_norm_rope_grad(qr, kr, q, k, dqr, dkr, heads, kv, positions=pos, q_gain=gq, k_gain=gk, dq_gain=dgq, dk_gain=dgk, eps=1e-5, rotary=16, base=1e5,
                                    pairs="neighbours", **more)
        out, lse, dq, dk, dv = new(qr), torch.full((n, heads, t), NAN, device="cuda:0"), new(qr), new(kr), new(kr)
        attention.attention(qr, kr, v, out, heads, kv, lse=lse, starts=starts, window=20, sinks=2, scale=0.3, **more)
        attention.attention_grad(out, qr, kr, v, out, lse, dq, dk, dv, heads, kv, starts=starts, window=20, sinks=2, scale=0.3, **more)
        ck, cv = normal((n, 2, slots, kv * head), BF16, 8), normal((n, 2, slots, kv * head), BF16, 9)
        token = new(qr[:, :2])
        attention.attention_step(qr[:, :2], kr[:, :2], v[:, :2], ck, cv, lengths, token, heads, kv, window=30, sinks=4, scale=0.3, **more)
        y = new(qr)
        attention.dropout(qr, y, 0.3, -5, step=2 ** 63 + 1, residual=q.contiguous(), step_dev=counter, **more)
        made = (qr, kr, dqr, dkr, dgq, dgk, out, lse, dq, dk, dv, ck, cv, token, y)
        return [torch.nan_to_num(x, 777.0) for x in made]

    assert attention._ext is not None or attention._bind() is None
    taken = []
    real = attention._short
    monkeypatch.setattr(attention, "_short", lambda name, *args: (taken.append((name, real(name, *args))), taken[-1][1])[1])
    short = calls()
    assert taken == [(name, True) for name in ("qk_norm_rope", "qk_norm_rope_grad", "attention", "attention_grad", "attention_step", "dropout")]
    with_stream = calls(stream=torch.cuda.current_stream())
    monkeypatch.setattr(attention, "_short", lambda name, *args: False)
    long = calls()
    for a, b, c in zip(short, long, with_stream):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_two_calls_at_once(attention):
    """Two streams, each with its own workspace, many times over: neither sees the other."""
    n, t, heads, kv, head = 1, 600, 4, 1, 64
    sides = []
    for s in range(2):
        _, q, k, v = slices(n, t, heads, kv, head, BF16, 0, 10 + s)
        out, lse, dout = torch.empty((n, t, heads * head), dtype=BF16, device="cuda:0"), torch.empty((n, heads, t), device="cuda:0"), normal((n, t, heads * head), BF16, 20 + s)
        d = slices(n, t, heads, kv, head, BF16, 0)
        ck, cv, token = normal((n, 1, t, kv * head), BF16, 30 + s), normal((n, 1, t, kv * head), BF16, 40 + s), torch.empty((n, 1, heads * head), dtype=BF16, device="cuda:0")
        rooms = [torch.empty(size, dtype=torch.uint8, device="cuda:0") for size in (attention.attention_grad_workspace(heads, kv, head, n, t), attention.attention_step_workspace(
            heads, kv, head, n, 1, t))]
        sides.append((q, k, v, out, lse, dout, d, ck, cv, token, rooms, torch.cuda.Stream()))
    lengths = cuts([[t - 1]])

    def work(side, stream):
        q, k, v, out, lse, dout, (_, dq, dk, dv), ck, cv, token, rooms, _ = side
        attention.attention(q, k, v, out, heads, kv, lse=lse, stream=stream)
        attention.attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, workspace=rooms[0], stream=stream)
        attention.attention_step(q[:, :1], k[:, :1], v[:, :1], ck, cv, lengths, token, heads, kv, workspace=rooms[1], stream=stream)

    want = []
    for side in sides:
        work(side, None)
        want.append([x.clone() for x in (side[3], side[4], side[6][0], side[9])])
    torch.cuda.synchronize()
    for _ in range(10):
        for side in sides:
            for x in (side[3], side[6][0], side[9]):
                x.fill_(NAN)
        torch.cuda.synchronize()
        for side in sides:
            work(side, side[11])
        torch.cuda.synchronize()
        for side, w in zip(sides, want):
            for x, y in zip((side[3], side[4], side[6][0], side[9]), w):
                assert torch.equal(x, y)


_FIRST_CALLS = """
import torch
from paper_2002_01119_amd import attention, psgd
torch.cuda.set_device(0)
n, t, heads, kv, head = 2, 300, 4, 2, 128
draw = lambda *shape: torch.randn(shape, device="cuda:0").bfloat16()
q, k, v, do = draw(n, t, heads * head), draw(n, t, kv * head), draw(n, t, kv * head), draw(n, t, heads * head)
ck, cv = draw(n, 3, 600, kv * head), draw(n, 3, 600, kv * head)
starts = torch.tensor([[0, 100, 300], [5, 5, 299]], dtype=torch.int32, device="cuda:0")
lengths = torch.tensor([[0, 599, 300], [-1, 40, 600]], dtype=torch.int32, device="cuda:0")
gain, counter = torch.ones(n, head, device="cuda:0"), torch.zeros(1, dtype=torch.int64, device="cuda:0")
outs = [torch.empty_like(x) for x in (q, k, q, q, k, v, q, k, q)] + [torch.empty(n, heads, t, device="cuda:0"), torch.empty_like(gain), torch.empty_like(gain), torch.empty_like(q[:, :3])]
qr, kr, o, dq, dk, dv, dqi, dki, y, lse, dgq, dgk, token = outs
rooms = [torch.empty(256 + s, dtype=torch.uint8, device="cuda:0") for s in (attention.qk_norm_rope_grad_workspace(n, t, head), attention.attention_grad_workspace(heads, kv, head, n, t, 60, 3, 2),
         attention.attention_step_workspace(heads, kv, head, n, 3, 600))]
def calls():
    attention.qk_norm_rope(q, k, qr, kr, heads, kv, q_gain=gain, k_gain=gain)
    attention.attention(qr, kr, v, o, heads, kv, lse=lse, starts=starts, window=60, sinks=3)
    attention.attention_grad(do, qr, kr, v, o, lse, dq, dk, dv, heads, kv, starts=starts, window=60, sinks=3, workspace=rooms[1])
    attention.qk_norm_rope_grad(dq, dk, q, k, dqi, dki, heads, kv, q_gain=gain, k_gain=gain, dq_gain=dgq, dk_gain=dgk, workspace=rooms[0])
    attention.attention_step(q[:, :3], k[:, :3], v[:, :3], ck, cv, lengths, token, heads, kv, workspace=rooms[2])
    attention.dropout(o, y, 0.1, 4, residual=q, step_dev=counter)
for x in outs:
    x.zero_()
torch.cuda.synchronize()
g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
with torch.cuda.graph(g, stream=s):                     # the first calls of the process, with more than 64 KB of LDS and the status word
    calls()
got = []
for _ in range(3):
    for x in outs:
        x.zero_()
    g.replay()
    torch.cuda.synchronize()
    got.append([x.clone() for x in outs])
for x in outs:
    x.zero_()
calls()
torch.cuda.synchronize()
same = lambda a, b: torch.equal(torch.nan_to_num(a, 777.0), torch.nan_to_num(b, 777.0))
assert all(same(a, b) for r in got for a, b in zip(r, outs))
assert psgd.device_status() == 2                        # the length that does not fit
print("captured first calls match")
"""


def test_first_calls_of_a_process_under_capture(attention):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "match" in r.stdout, r.stderr[-2000:]


@pytest.fixture
def far():
    """Room of 2^32 elements and some."""
    room = torch.empty((1 << 32) + (1 << 22), dtype=BF16, device="cuda:0")
    yield room
    del room
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,learner,row", [(2, (1 << 31) + 4096, 2048), (1, 0, (1 << 25) + 64)])
def test_offsets_beyond_32_bits(attention, far, n, learner, row):
    """The second learner, or the later tokens, lie more than 2^31 elements behind the first."""
    t, heads, kv, head = 100, 4, 2, 64
    q, k, v, dq, dk, dv, out, dout = (far.as_strided((n, t, c * head), (learner, row, 1), at) for c, at in
                                      ((heads, 0), (kv, 256), (kv, 384), (heads, 512), (kv, 768), (kv, 896), (heads, 1024), (heads, 1280)))
    for i, x in enumerate((q, k, v, dout)):
        x.copy_(normal(x.shape, BF16, i))
    for x in (dq, dk, dv, out):
        x.fill_(NAN)
    lse = torch.empty((n, heads, t), device="cuda:0")
    attention.qk_norm_rope(q, k, q, k, heads, kv)
    attention.attention(q, k, v, out, heads, kv, lse=lse, window=30, sinks=2)
    attention.attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, window=30, sinks=2)
    want, bound = orc.attention(q, k, v, None, heads, kv, 30, 2, head ** -0.5, BF16)
    within(out, want[0], bound[0], "out")
    want, bound = orc.attention_grad(dout, q, k, v, out, lse, None, heads, kv, 30, 2, head ** -0.5, BF16)
    for got, w, b, what in zip((dq, dk, dv), want, bound, ("dq", "dk", "dv")):
        within(got, w, b, what)
    near = out.contiguous()
    attention.dropout(out, dq, 0.5, 3, residual=q)
    other = torch.empty_like(near)
    attention.dropout(near, other, 0.5, 3, residual=q.contiguous())
    assert torch.equal(dq, other)


@pytest.mark.parametrize("strides", [(1 << 31, 256), (1024, 1 << 22)])
def test_caches_beyond_32_bits(attention, far, strides):
    """A cache whose later sequence, or whose later slots, lie more than 2^31 elements behind its first."""
    b, heads, kv, head, slots = 2, 4, 2, 64, 600
    ck, cv = (far.as_strided((1, b, slots, kv * head), (0,) + strides + (1,), at) for at in (0, 128))
    for i, x in enumerate((ck, cv)):
        x.copy_(normal(x.shape, BF16, i))
    step_tests.check(attention, torch.tensor([[599, 40]], dtype=torch.int32, device="cuda:0"), heads, kv, head, slots, BF16, garbage=False, caches=(ck, cv))
