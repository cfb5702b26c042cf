"""Dropout from a counter, against the generator in 64-bit integers."""
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


def normal(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.empty(shape).normal_(0.0, 1.0, generator=g)).to(dtype).to("cuda:0")


SEED = 0xFEDCBA9876543210


@pytest.mark.parametrize("n,t,c", [(1, 1, 1), (1, 1, 3), (2, 3, 4), (2, 3, 5), (3, 7, 8), (1, 5, 9), (4, 33, 257), (8, 1, 4096), (2, 130, 1000), (512, 2, 13), (1, 3000, 31)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_values(attention, n, t, c, dtype, residual, p):
    x = normal((n, t, c + 3), dtype, 1)[:, :, :c]
    r = normal((n, t, c), dtype, 2) if residual else None
    whole = torch.full((n, t, c + 5), NAN, dtype=dtype, device="cuda:0")
    attention.dropout(x, whole[:, :, :c], p, SEED, step=12345, residual=r)
    assert_within(whole[:, :, :c], *orc.dropout(x, r, p, SEED, 12345, dtype), "y")
    assert torch.isnan(whole[:, :, c:]).all()


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -18, 2.0 ** -16, 0.25, 0.9999999, 1 - 2.0 ** -16])
def test_probabilities(attention, p):
    x, r = normal((2, 40, 300), F32, 1), normal((2, 40, 300), F32, 2)
    y = torch.empty_like(x)
    attention.dropout(x, y, p, 7, step=3, residual=r)
    assert_within(y, *orc.dropout(x, r, p, 7, 3, F32), "y")
    if p < 2.0 ** -17:
        assert torch.equal(y, x + r)
    if p == 1.0:
        assert torch.equal(y, r)


def test_share_and_independence(attention):
    """The share that is kept, and that seeds, steps, learners and neighbours do not go together: five deviations of a binomial."""
    n, t, c, p = 2, 512, 1024, 0.25
    x = torch.ones((n, t, c), device="cuda:0")
    masks = []
    for seed, step in ((1, 0), (1, 1), (2, 0), (1, 2)):
        y = torch.empty_like(x)
        attention.dropout(x, y, p, seed, step=step)
        masks.append(y != 0)
        assert torch.equal(y[masks[-1]].unique(), torch.tensor([65536.0 / 49152.0], device="cuda:0"))
    count = n * t * c
    for m in masks:
        assert abs(float(m.double().mean()) - 0.75) < 5 * (0.1875 / count) ** 0.5
    both = lambda a, b: abs(float((a & b).double().mean()) - 0.5625) < 5 * (0.5625 * 0.4375 / a.numel()) ** 0.5  # noqa: E731
    assert all(both(a, b) for i, a in enumerate(masks) for b in masks[:i])
    m = masks[0]
    assert both(m[0], m[1]) and both(m[:, 1:], m[:, :-1]) and both(m[:, :, 1:], m[:, :, :-1]) and both(m[:, :, 4:], m[:, :, :-4])


def test_dropped_elements_are_zero_whatever_they_hold(attention):
    x = normal((1, 20, 64), BF16, 1)
    kept, _ = orc.dropped(1, 20, 64, 0.5, 9, 0)
    x[~kept.to("cuda:0")] = NAN
    y = torch.empty_like(x)
    attention.dropout(x, y, 0.5, 9)
    assert torch.isfinite(y).all() and (y[~kept.to("cuda:0")] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_backward(attention, dtype):
    x, r = normal((2, 9, 77), dtype, 1), normal((2, 9, 77), dtype, 2)
    want, bound = orc.dropout(x, r, 0.3, 5, 6, dtype)
    a, b, y = x.clone(), r.clone(), torch.empty_like(x)
    attention.dropout(a, a, 0.3, 5, step=6, residual=r)
    attention.dropout(x, b, 0.3, 5, step=6, residual=b)
    attention.dropout(x, y, 0.3, 5, step=6, residual=r)
    assert torch.equal(a, y) and torch.equal(b, y)
    assert_within(y, want, bound, "y")
    # the gradient of sum(y w): the same mask on w; and against differences, exact for a linear map
    w, dx = normal((2, 9, 77), dtype, 3), torch.empty_like(x)
    attention.dropout(w, dx, 0.3, 5, step=6)
    kept, scale = orc.dropped(2, 9, 77, 0.3, 5, 6)
    assert torch.equal(dx.cpu() != 0, kept & (w.cpu() != 0))
    up = torch.empty((2, 9, 77), device="cuda:0")
    down = torch.empty_like(up)
    attention.dropout(x.float() + 1.0, up, 0.3, 5, step=6)
    attention.dropout(x.float(), down, 0.3, 5, step=6)
    assert float(((up - down).cpu() - kept * scale).abs().max()) <= 8 * 2.0 ** -24 * 8     # few roundings of values below 8


def test_rows_of_any_stride_and_a_shared_input(attention):
    x = normal((1, 1, 100), F32, 1).expand(3, 5, 100)
    y = torch.empty((5, 3, 100), device="cuda:0").transpose(0, 1)
    attention.dropout(x, y, 0.4, 1)
    assert_within(y, *orc.dropout(x, None, 0.4, 1, 0, F32), "y")


def test_a_captured_call_draws_a_new_mask_for_each_replay(attention):
    x = normal((2, 30, 64), F32, 1)
    y, step = torch.empty_like(x), torch.zeros(1, dtype=torch.int64, device="cuda:0")
    attention.dropout(x, y, 0.5, 11, step=4, step_dev=step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attention.dropout(x, y, 0.5, 11, step=4, step_dev=step)
        step += 1
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert_within(y, *orc.dropout(x, None, 0.5, 11, 4 + i, F32), "y")


def test_more_rows_than_a_launch_counts(attention):
    """Rows in several launches: 2^30 groups of 16 bytes a launch, here of one column each."""
    n, t = 2, 3 << 28
    x = torch.ones((1, 1, 1), dtype=BF16, device="cuda:0").expand(n, t, 1)
    y = torch.empty((n, t, 1), dtype=BF16, device="cuda:0")
    attention.dropout(x, y, 0.5, 3)
    step, golden = 0, 0x9E3779B97F4A7C15
    import numpy as np
    for row in (0, 1, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, n * t - 1):
        with np.errstate(over="ignore"):
            z = np.uint64((3 ^ ((step + 1) * golden & (1 << 64) - 1))) + np.uint64((row + 1) * golden & (1 << 64) - 1)
            z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
            z = z ^ (z >> np.uint64(31))
        assert float(y.view(-1)[row]) == (2.0 if int(z) & 65535 < 32768 else 0.0)
    assert abs(float((y != 0).sum(dtype=torch.int64)) / (n * t) - 0.5) < 5 * 0.5 / (n * t) ** 0.5
