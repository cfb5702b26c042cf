"""Causal attention in packed sequences, with windows and first tokens that stay visible, forward and backward, against its formula in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
from oracle import attention_oracle as orc  # noqa: E402
from oracle.layers_oracle import assert_within  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


@pytest.fixture(scope="module")
def attention():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_01119_amd import attention as m
    m.load()
    torch.cuda.set_device(0)
    return m


def normal(shape, dtype, seed, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.empty(shape).normal_(0.0, sigma, generator=g)).to(dtype).to("cuda:0")


def projected(n, t, heads, kv, head, dtype, seed=None, pitch=0, lead=0, sigma=1.0):
    """q, k and v as column slices of one array; drawn, or NaN to be written."""
    width = (heads + 2 * kv) * head + pitch
    whole = torch.full((lead + n * t * width,), NAN, dtype=dtype, device="cuda:0")
    a = whole[lead:].view(n, t, width)
    if seed is not None:
        a.copy_(normal(a.shape, dtype, seed, sigma))
    return a, a[:, :, :heads * head], a[:, :, heads * head:(heads + kv) * head], a[:, :, (heads + kv) * head:(heads + 2 * kv) * head]


def cuts(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda:0")


def within(got, want, bound, what):
    """Rows of no sequence are NaN on both sides: they were NaN before."""
    assert_within(got, want, bound, what)


def check(attention, n, t, heads, kv, head, dtype, window=0, sinks=0, starts=None, pitch=0, lead=0, scale=None, backward=True, sigma=1.0, again=False):
    _, q, k, v = projected(n, t, heads, kv, head, dtype, 1, pitch, lead, sigma)
    out = torch.full((n, t, heads * head + pitch), NAN, dtype=dtype, device="cuda:0")[:, :, :heads * head]
    lse = torch.full((n, heads, t), NAN, device="cuda:0")
    how = dict(starts=starts, window=window, sinks=sinks, scale=scale)
    s = head ** -0.5 if scale is None else scale
    attention.attention(q, k, v, out, heads, kv, lse=lse, **how)
    want, bound = orc.attention(q, k, v, None if starts is None else starts.cpu(), heads, kv, window, sinks, s, dtype)
    within(out, want[0], bound[0], "out")
    within(lse, want[1], bound[1], "lse")
    if not backward:
        return
    dout = normal((n, t, heads * head), dtype, 2)
    runs = []
    for _ in range(2 if again else 1):
        a, dq, dk, dv = projected(n, t, heads, kv, head, dtype, None, pitch, lead)
        attention.attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, **how)
        runs.append(torch.nan_to_num(a, 12345.0))
    assert torch.equal(runs[0], runs[-1])                                       # the same bits again
    want, bound = orc.attention_grad(dout, q, k, v, out, lse, None if starts is None else starts.cpu(), heads, kv, window, sinks, s, dtype)
    for got, w, b, what in zip((dq, dk, dv), want, bound, ("dq", "dk", "dv")):
        within(got, w, b, what)
    assert torch.isnan(a[:, :, (heads + 2 * kv) * head:]).all()


# one row, a tile, either side of its edges, several
LENGTHS = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 257]


@pytest.mark.parametrize("t", LENGTHS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lengths(attention, t, dtype):
    check(attention, 1, t, 2, 1, 64, dtype)


@pytest.mark.parametrize("head", [1, 7, 8, 16, 33, 50, 64, 72, 80, 96, 127, 128, 136, 200, 255, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_heads_of_any_width(attention, head, dtype):
    pitch, lead = (3, 1) if head % 2 else (0, 0)
    check(attention, 2, 150, 2, 2, head, dtype, window=70, sinks=3, pitch=pitch, lead=lead)


@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1), (4, 2), (6, 3), (5, 5), (16, 2), (9, 1)])
@pytest.mark.parametrize("n", [1, 4])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_heads_and_learners(attention, heads, kv, n, dtype):
    check(attention, n, 90, heads, kv, 32, dtype, again=True)


WINDOWS = [(1, 0), (1, 1), (2, 1), (16, 0), (17, 4), (63, 0), (64, 1), (65, 64), (100, 65), (128, 4), (150, 129), (299, 1), (300, 7), (1 << 31, 5)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("head,dtype", [(64, F32), (128, BF16), (64, BF16), (256, BF16), (200, F32)])
def test_windows(attention, window, sinks, head, dtype):
    check(attention, 1, 300, 2, 1, head, dtype, window=min(window, 2 ** 31 - 1), sinks=sinks)


PACKED = [
    [[0, 200]], [[0, 100, 200]], [[0, 1, 2, 3, 200]], [[0, 0, 0, 130, 130, 200, 200]], [[5, 64, 128, 190]], [[0, 63, 127, 191, 199]],
    [[7, 7, 7]], [[199, 200]], [[0, 0]], [[200, 200]], [list(range(0, 201))], [[0] * 70 + [90] * 70 + [200] * 3],
]


@pytest.mark.parametrize("rows", PACKED, ids=[str(i) for i in range(len(PACKED))])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 2)])
@pytest.mark.parametrize("head,dtype", [(64, F32), (128, BF16), (256, F32), (256, BF16)])
def test_packed_sequences(attention, rows, window, sinks, head, dtype):
    check(attention, 1, 200, 2, 1, head, dtype, window=window, sinks=sinks, starts=cuts(rows))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sequences_of_each_learner(attention, dtype):
    starts = cuts([[0, 50, 180, 300], [0, 0, 299, 300], [10, 20, 30, 40]])
    check(attention, 3, 300, 4, 2, 64, dtype, starts=starts)
    check(attention, 3, 300, 4, 2, 64, dtype, starts=cuts([[0, 70, 290]]).expand(3, 3), window=40)     # the same of all learners


def test_more_sequences_than_a_wavefront_looks_at(attention):
    g = torch.Generator().manual_seed(3)
    rows = torch.sort(torch.randint(0, 1001, (2, 400), generator=g), 1).values.to(torch.int32).to("cuda:0")
    check(attention, 2, 1000, 2, 1, 64, F32, starts=rows)
    check(attention, 2, 1000, 2, 1, 64, BF16, starts=rows, window=5, sinks=1)


@pytest.mark.parametrize("n,kv,t,window", [(8, 1, 700, 0), (4, 2, 1030, 0), (3, 3, 513, 200), (1, 1, 2100, 129)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_tiles(attention, n, kv, t, window, dtype):
    """Numbers of learners and key heads that dies share evenly and others."""
    check(attention, n, t, 2 * kv, kv, 64, dtype, window=window, sinks=3 if window else 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scales_and_sharp_rows(attention, dtype):
    for scale in (0.0, -0.3, 1.0, 3.0):
        check(attention, 1, 130, 2, 1, 64, dtype, scale=scale)
    check(attention, 1, 260, 1, 1, 128, dtype, sigma=6.0)                # scores of hundreds: rows look at one token


@pytest.mark.parametrize("bad", [NAN, float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nothing_passes_from_one_sequence_to_another(attention, bad, dtype):
    """Garbage in rows of no sequence and in another sequence."""
    n, t, heads, kv, head = 1, 300, 2, 1, 64
    starts = cuts([[20, 90, 170, 280]])
    a, q, k, v = projected(n, t, heads, kv, head, dtype, 1)
    clean = a.clone()
    for rows in (slice(0, 20), slice(90, 170), slice(280, 300)):
        a[:, rows] = bad
    outs = []
    for x in (clean, a):
        qq, kk, vv = x[:, :, :128], x[:, :, 128:192], x[:, :, 192:256]
        out, lse = torch.zeros((n, t, heads * head), dtype=dtype, device="cuda:0"), torch.zeros((n, heads, t), device="cuda:0")
        attention.attention(qq, kk, vv, out, heads, kv, lse=lse, starts=starts)
        dout = normal(out.shape, dtype, 5)
        if x is a:
            dout[:, 90:170] = bad
            dout[:, :20] = bad
        d, dq, dk, dv = projected(n, t, heads, kv, head, dtype)
        attention.attention_grad(dout, qq, kk, vv, out, lse, dq, dk, dv, heads, kv, starts=starts)
        outs.append((out, lse.transpose(1, 2).contiguous(), d))
    for rows in (slice(20, 90), slice(170, 280)):
        for x, y in zip(*outs):
            assert torch.equal(x[:, rows], y[:, rows])
    for x in outs[1][:2]:
        assert (x[:, :20] == 0).all() and (x[:, 280:] == 0).all()


def test_starts_out_of_order_raise_the_flag(attention):
    from paper_2002_01119_amd import psgd
    psgd.device_status(clear=True)
    n, t, heads, kv, head = 1, 64, 1, 1, 32
    _, q, k, v = projected(n, t, heads, kv, head, F32, 1)
    out = torch.zeros((n, t, head), device="cuda:0")
    attention.attention(q, k, v, out, heads, kv, starts=cuts([[0, 32, 64]]))
    assert psgd.device_status() == 0
    for rows in ([0, 40, 20], [-1, 64, 64], [0, 30, 65]):
        attention.attention(q, k, v, out, heads, kv, starts=cuts([rows]))
        assert psgd.device_status(clear=True) == 2
        assert psgd.device_status() == 0


@pytest.mark.parametrize("dtype,head", [(F32, 64), (BF16, 128), (BF16, 64)])
def test_gradients_are_those_of_differences(attention, dtype, head):
    """Against differences of the oracle in 64 bits: not the same derivation."""
    n, t, heads, kv, window, sinks = 1, 40, 2, 1, 20, 2
    starts = cuts([[0, 30, 40]])
    _, q, k, v = projected(n, t, heads, kv, head, dtype, 1)
    out, lse = torch.empty((n, t, heads * head), dtype=dtype, device="cuda:0"), torch.empty((n, heads, t), device="cuda:0")
    attention.attention(q, k, v, out, heads, kv, lse=lse, starts=starts, window=window, sinks=sinks)
    dout = normal(out.shape, dtype, 2)
    dq, dk, dv = torch.empty_like(out), torch.empty((n, t, kv * head), dtype=dtype, device="cuda:0"), torch.empty((n, t, kv * head), dtype=dtype, device="cuda:0")
    attention.attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, starts=starts, window=window, sinks=sinks)

    def value(q, k, v):
        (o, _), _ = orc.attention(q, k, v, starts.cpu(), heads, kv, window, sinks, head ** -0.5, torch.float64)
        return float((o * dout.cpu().double()).sum())

    orc.HALF[torch.float64] = 0.0
    base = [x.cpu().double() for x in (q, k, v)]
    for i, d in enumerate((dq, dk, dv)):
        way = normal(base[i].shape, F32, 20 + i).cpu().double()
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + 1e-4 * way, base[i] - 1e-4 * way
        slope, terms = (value(*up) - value(*down)) / 2e-4, d.cpu().double() * way
        # the gradient's elements are each off by a few halves of their type (as test_lengths bounds them), with either sign; D too, from the rounded out
        assert abs(slope - float(terms.sum())) <= (3e-2 if dtype == BF16 else 1e-5) * float(terms.abs().sum())


def test_other_strides_and_streams(attention):
    """Heads' arrays of their own, tokens outermost, inputs shared by learners, a stream that is not the current one."""
    n, t, heads, kv, head = 3, 140, 4, 2, 64
    q = normal((t, n, heads * head), BF16, 1).transpose(0, 1)
    k, v = normal((1, t, kv * head), BF16, 2).expand(n, t, kv * head), normal((1, t, kv * head), BF16, 3).expand(n, t, kv * head)
    out = torch.full((t, n, heads * head), NAN, dtype=BF16, device="cuda:0").transpose(0, 1)
    lse = torch.empty((n, heads, t), device="cuda:0")
    dout = normal((n, t, heads * head), BF16, 4)
    dq = torch.empty((t, n, heads * head), dtype=BF16, device="cuda:0").transpose(0, 1)
    dk, dv = (torch.empty((n, t, kv * head), dtype=BF16, device="cuda:0") for _ in range(2))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    attention.attention(q, k, v, out, heads, kv, lse=lse, stream=stream)
    attention.attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, stream=stream)
    torch.cuda.synchronize()
    want, bound = orc.attention(q, k, v, None, heads, kv, 0, 0, head ** -0.5, BF16)
    within(out, want[0], bound[0], "out")
    want, bound = orc.attention_grad(dout, q, k, v, out, lse, None, heads, kv, 0, 0, head ** -0.5, BF16)
    for got, w, b, what in zip((dq, dk, dv), want, bound, ("dq", "dk", "dv")):
        within(got, w, b, what)


def test_captured_and_replayed(attention):
    n, t, heads, kv, head = 2, 260, 4, 2, 64
    a, q, k, v = projected(n, t, heads, kv, head, BF16, 1)
    out, lse, dout = torch.empty((n, t, heads * head), dtype=BF16, device="cuda:0"), torch.empty((n, heads, t), device="cuda:0"), normal((n, t, heads * head), BF16, 2)
    d, dq, dk, dv = projected(n, t, heads, kv, head, BF16)
    starts = cuts([[0, 100, 260], [0, 20, 250]])
    room = torch.empty(attention.attention_grad_workspace(heads, kv, head, n, t, sequences=2), dtype=torch.uint8, device="cuda:0")

    def calls():
        attention.attention(q, k, v, out, heads, kv, lse=lse, starts=starts, window=50, sinks=2)
        attention.attention_grad(dout, q, k, v, out, lse, dq, dk, dv, heads, kv, starts=starts, window=50, sinks=2, workspace=room)

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (3, 4, 5):
        a.copy_(normal(a.shape, BF16, seed))
        starts.copy_(cuts([[0, 10 * seed, 260], [seed, 200, 255]]))              # other sequences, the same launch
        for x in (out, d):
            x.fill_(NAN)
        calls()
        want = [x.clone() for x in (out, lse, d)]
        for x in (out, d):
            x.fill_(NAN)
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((out, lse, d), want):
            assert torch.equal(torch.nan_to_num(got, 777.0), torch.nan_to_num(w, 777.0))
