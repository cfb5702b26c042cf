"""Attention of one new token of each sequence against its cache, against its formula in 64 bits."""
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


def numbers(rows):
    return torch.tensor(rows, dtype=torch.int32, device="cuda:0")


def check(attention, lengths, heads, kv, head, slots, dtype, window=0, sinks=0, scale=None, sigma=1.0, garbage=True, caches=None):
    """Slots that no visible position lies in hold NaN."""
    n, b = lengths.shape
    a = normal((n, b, (heads + 2 * kv) * head + 3), dtype, 1, sigma)
    q, k, v = a[:, :, :heads * head], a[:, :, heads * head:(heads + kv) * head], a[:, :, (heads + kv) * head:(heads + 2 * kv) * head]
    ck, cv = caches or (normal((n, b, slots, kv * head), dtype, 2 + i, sigma) for i in range(2))
    if garbage:
        for i in range(n):
            for r in range(b):
                p = int(lengths[i, r])
                seen = {orc.slot_of(j, sinks, slots) for j in range(p) if not window or p - j < window or j < sinks} if p < slots or (window and slots >= sinks + window) else set()
                rest = [s for s in range(slots) if s not in seen]
                ck[i, r, rest], cv[i, r, rest] = NAN, NAN
    out = torch.full((n, b, heads * head), NAN, dtype=dtype, device="cuda:0")
    want, bound, wk, wv = orc.attention_step(q, k, v, ck, cv, lengths, heads, kv, window, sinks, head ** -0.5 if scale is None else scale, dtype)
    attention.attention_step(q, k, v, ck, cv, lengths, out, heads, kv, window=window, sinks=sinks, scale=scale)
    assert_within(out, want, bound, "out")
    for got, w, what in ((ck, wk, "cache_k"), (cv, wv, "cache_v")):
        assert torch.equal(torch.nan_to_num(got.cpu(), 777.0), torch.nan_to_num(w, 777.0)), what


@pytest.mark.parametrize("length", [0, 1, 15, 16, 31, 32, 33, 127, 128, 129, 255, 300, 511])
@pytest.mark.parametrize("head,dtype", [(64, F32), (128, BF16)])
def test_lengths(attention, length, head, dtype):
    check(attention, numbers([[length]]), 4, 2, head, 512, dtype)


@pytest.mark.parametrize("head", [1, 8, 16, 33, 50, 64, 72, 80, 96, 127, 128, 136, 200, 255, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_heads_of_any_width(attention, head, dtype):
    check(attention, numbers([[70, 3, -1], [0, 149, 64]]), 4, 2, head, 150, dtype)


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (5, 1), (16, 1), (17, 1), (40, 1), (64, 2), (6, 3)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_heads(attention, heads, kv, dtype):
    check(attention, numbers([[40, 90], [0, 199]]), heads, kv, 32, 200, dtype)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (16, 0), (17, 4), (64, 1), (100, 65), (128, 4)])
@pytest.mark.parametrize("more", [0, 1, 37])
@pytest.mark.parametrize("head,dtype", [(64, F32), (64, BF16), (128, BF16)])
def test_rings(attention, window, sinks, more, head, dtype):
    """Caches of sinks + window rows and a few more, lengths far beyond them."""
    slots = sinks + window + more
    lengths = numbers([[0, sinks, window, slots - 1, slots], [slots + 1, 2 * slots, 1000, 1001, max(0, sinks - 1)]])
    check(attention, lengths, 4, 2, head, slots, dtype, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_window_on_a_cache_that_is_no_ring(attention, dtype):
    check(attention, numbers([[0, 5, 49, 30]]), 2, 1, 64, 50, dtype, window=60, sinks=4)
    check(attention, numbers([[0, 5, 7]]), 2, 1, 64, 8, dtype, window=11, sinks=37)         # fewer rows than first tokens


@pytest.mark.parametrize("n,b,length,slots", [(1, 1, 4999, 5000), (1, 2, 3000, 5000), (4, 60, 200, 256), (1, 1, 9, 20000), (2, 3, 1023, 1024)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_parts(attention, n, b, length, slots, dtype):
    """One part, several, and parts that hold nothing."""
    g = torch.Generator().manual_seed(4)
    lengths = (length - torch.randint(0, min(length, 50) + 1, (n, b), generator=g)).to(torch.int32).to("cuda:0")
    check(attention, lengths, 2, 1, 64, slots, dtype, garbage=slots < 2000)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scales_and_sharp_rows(attention, dtype):
    for scale in (0.0, -0.3, 2.0):
        check(attention, numbers([[100]]), 2, 1, 64, 128, dtype, scale=scale)
    check(attention, numbers([[100, 600]]), 2, 1, 128, 700, dtype, sigma=6.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_other_strides(attention, dtype):
    """Keys and values of one array, side by side in a row, row by row, and heads' sequences outermost; lengths of any stride."""
    n, b, slots, kv, head = 2, 3, 60, 2, 32
    lengths = numbers([[[10, 0], [59, 0], [0, 0]], [[33, 0], [34, 0], [35, 0]]])[:, :, 0]
    both = normal((n, b, slots, 2 * kv * head), dtype, 5)
    check(attention, lengths, 4, kv, head, slots, dtype, caches=(both[..., :kv * head], both[..., kv * head:]))
    both = normal((n, b, slots, 2, kv * head), dtype, 6)
    check(attention, lengths, 4, kv, head, slots, dtype, caches=(both[..., 0, :], both[..., 1, :]))
    both = normal((2, slots, b, n, kv * head), dtype, 7).permute(0, 3, 2, 1, 4)
    check(attention, lengths, 4, kv, head, slots, dtype, caches=(both[0], both[1]))


def test_lengths_that_do_not_fit_raise_the_flag(attention):
    from paper_2002_01119_amd import psgd
    psgd.device_status(clear=True)
    n, b, heads, kv, head, slots = 1, 4, 4, 2, 64, 16
    q, k = normal((n, b, heads * head), F32, 1), normal((n, b, kv * head), F32, 2)
    ck, cv = normal((n, b, slots, kv * head), F32, 3), normal((n, b, slots, kv * head), F32, 4)
    before, out = ck.clone(), torch.full((n, b, heads * head), 5.0, device="cuda:0")
    attention.attention_step(q, k, k, ck, cv, numbers([[15, 16, -7, 2 ** 31 - 1]]), out, heads, kv)
    assert psgd.device_status(clear=True) == 2
    assert torch.isfinite(out[0, 0]).all() and torch.isnan(out[0, 1]).all() and (out[0, 2] == 5.0).all() and torch.isnan(out[0, 3]).all()
    assert torch.equal(ck[0, 1:], before[0, 1:]) and torch.equal(ck[0, 0, :15], before[0, 0, :15]) and torch.equal(ck[0, 0, 15], k[0, 0])


def test_steps_are_the_rows_of_attention(attention):
    """A sequence fed token by token through a ring of its window against the forward pass over all of it."""
    n, t, heads, kv, head, window, sinks = 2, 90, 4, 2, 64, 20, 3
    a = normal((n, t, (heads + 2 * kv) * head), F32, 1)
    q, k, v = a.split((heads * head, kv * head, kv * head), 2)
    out, lse = torch.empty((n, t, heads * head), device="cuda:0"), torch.empty((n, heads, t), device="cuda:0")
    attention.attention(q, k, v, out, heads, kv, lse=lse, window=window, sinks=sinks)
    caches = [torch.full((n, 1, window + sinks, kv * head), NAN, device="cuda:0") for _ in range(2)]
    lengths, steps = torch.zeros((n, 1), dtype=torch.int32, device="cuda:0"), torch.empty_like(out)
    for i in range(t):
        row = slice(i, i + 1)
        attention.attention_step(q[:, row], k[:, row], v[:, row], *caches, lengths, steps[:, row], heads, kv, window=window, sinks=sinks)
        lengths += 1
    want, bound = orc.attention(q, k, v, None, heads, kv, window, sinks, head ** -0.5, F32)
    assert_within(out, want[0], bound[0], "out")
    assert_within(steps, want[0], bound[0], "steps")


def test_captured_and_replayed(attention):
    """One graph for every step: lengths live on the device."""
    n, b, heads, kv, head, slots = 2, 2, 8, 2, 64, 3000
    a = normal((n, b, (heads + 2 * kv) * head), BF16, 1)
    q, k, v = a.split((heads * head, kv * head, kv * head), 2)
    caches = [normal((n, b, slots, kv * head), BF16, 2 + i) for i in range(2)]
    out, lengths = torch.empty((n, b, heads * head), dtype=BF16, device="cuda:0"), numbers([[2000, 5], [-1, 2900]])
    need = attention.attention_step_workspace(heads, kv, head, n, b, slots)
    assert need > 0
    room = torch.empty(need, dtype=torch.uint8, device="cuda:0")

    def call():
        attention.attention_step(q, k, v, *caches, lengths, out, heads, kv, workspace=room)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        a.copy_(normal(a.shape, BF16, 10 + i))
        lengths += 7
        kept = [c.clone() for c in caches]
        out.fill_(3.0)
        call()
        want, after = out.clone(), [c.clone() for c in caches]
        for c, x in zip(caches, kept):
            c.copy_(x)
        out.fill_(3.0)
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(c, x) for c, x in zip(caches, after))
