"""An attention block of several learners put together as a training step has it - linear layer, norms and rotation, attention, linear layer, dropout and the
residual - with parameters in rows of X and gradients in rows of G, against autograd in 64 bits; then the averaging step on those rows; and the block serving
token by token."""
import pytest

torch = pytest.importorskip("torch")
from oracle import attention_oracle as orc  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
N, T, C, HEADS, KV, HEAD = 3, 70, 40, 4, 2, 16
Q, K = HEADS * HEAD, KV * HEAD
WINDOW, SINKS, P, SEED, STEP = 20, 2, 0.2, 77, 5


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_01119_amd import attention, layers, psgd
    attention.load()
    torch.cuda.set_device(0)
    return attention, layers, psgd


def parameters(X):
    """Views of the rows of [n, d]: w_qkv, q_gain, k_gain, w_out."""
    at = [0]

    def take(*shape):
        size = 1
        for s in shape:
            size *= s
        v = X.as_strided((X.shape[0],) + shape, (X.stride(0), shape[1], 1) if len(shape) == 2 else (X.stride(0), 1), X.storage_offset() + at[0])
        at[0] += size
        return v
    return take(Q + 2 * K, C), take(HEAD), take(HEAD), take(C, Q)


SIZE = (Q + 2 * K) * C + 2 * HEAD + C * Q


def made(dtype):
    g = torch.Generator().manual_seed(3)
    X = torch.empty(N, SIZE + 5).normal_(0.0, 1.0, generator=g)
    for p, sigma, mean in zip(parameters(X), (C ** -0.5, 0.2, 0.2, Q ** -0.5), (0.0, 1.0, 1.0, 0.0)):
        p.copy_(torch.empty(p.shape).normal_(mean, sigma, generator=g))
    x, dy = (torch.empty(N, T, C).normal_(0.0, 1.0, generator=g).to(dtype).to("cuda:0") for _ in range(2))
    starts = torch.tensor([[0, 30, 70], [0, 0, 70], [0, 69, 70]], dtype=torch.int32, device="cuda:0")
    row = torch.arange(T)
    first = torch.stack([torch.where(row < s[1], s[0], s[1]) for s in starts.cpu()])
    positions = (row - first).to(torch.int32).to("cuda:0")
    return X.to(dtype).to("cuda:0"), x, dy, starts, positions


def forward(mods, X, x, starts, positions):
    attention, layers, _ = mods
    dtype = x.dtype
    w, gq, gk, wo = parameters(X)
    a, b = torch.empty((N, T, Q + 2 * K), dtype=dtype, device="cuda:0"), torch.empty((N, T, Q + K), dtype=dtype, device="cuda:0")
    layers.linear(x, w, a)
    q, k, v = a.split((Q, K, K), 2)
    qr, kr = b.split((Q, K), 2)
    attention.qk_norm_rope(q, k, qr, kr, HEADS, KV, positions=positions, q_gain=gq, k_gain=gk)
    o, lse = torch.empty((N, T, Q), dtype=dtype, device="cuda:0"), torch.empty((N, HEADS, T), device="cuda:0")
    attention.attention(qr, kr, v, o, HEADS, KV, lse=lse, starts=starts, window=WINDOW, sinks=SINKS)
    z, y = torch.empty((N, T, C), dtype=dtype, device="cuda:0"), torch.empty((N, T, C), dtype=dtype, device="cuda:0")
    layers.linear(o, wo, z)
    attention.dropout(z, y, P, SEED, step=STEP, residual=x)
    return a, qr, kr, o, lse, y


def backward(mods, X, G, x, dy, starts, positions, kept):
    attention, layers, _ = mods
    a, qr, kr, o, lse, _ = kept
    w, gq, gk, wo = parameters(X)
    dw, dgq, dgk, dwo = parameters(G)
    dz, do, da, dx = (torch.empty_like(t) for t in (dy, o, a, dy))
    attention.dropout(dy, dz, P, SEED, step=STEP)
    layers.linear_grad(dz, o, wo, dx=do, dw=dwo)
    q, k, v = a.split((Q, K, K), 2)
    dq, dk, dv = da.split((Q, K, K), 2)
    attention.attention_grad(do, qr, kr, v, o, lse, dq, dk, dv, HEADS, KV, starts=starts, window=WINDOW, sinks=SINKS)
    attention.qk_norm_rope_grad(dq, dk, q, k, dq, dk, HEADS, KV, positions=positions, q_gain=gq, k_gain=gk, dq_gain=dgq, dk_gain=dgk)
    layers.linear_grad(da, x, w, dx=dx, dw=dw)
    return dx + dy


def reference(X, x, starts, positions, kept):
    """The block in 64 bits, from tensors that carry gradients."""
    w, gq, gk, wo = parameters(X)
    a = x @ w.transpose(1, 2)

    def turned(u, gain):
        u = u.unflatten(2, (-1, HEAD))
        u = u * (u.square().mean(3, keepdim=True) + 1e-6).rsqrt() * gain[:, None, None]
        f = positions.double()[:, :, None, None] * 10000.0 ** (-2.0 * torch.arange(HEAD // 2).double() / HEAD)
        p, s = u[..., :HEAD // 2], u[..., HEAD // 2:]
        return torch.cat((p * f.cos() - s * f.sin(), s * f.cos() + p * f.sin()), 3)

    q, k, v = turned(a[:, :, :Q], gq), turned(a[:, :, Q:Q + K], gk), a[:, :, Q + K:].unflatten(2, (KV, HEAD))
    rows = []
    for i in range(N):
        seen = torch.zeros(T, T, dtype=torch.bool)
        for lo, hi in orc.sequences(starts[i].tolist(), T):
            seen[lo:hi, lo:hi] = orc.visible(hi - lo, WINDOW, SINKS)
        heads = []
        for h in range(HEADS):
            z = (q[i, :, h] @ k[i, :, h * KV // HEADS].T * HEAD ** -0.5).masked_fill(~seen, -float("inf"))
            heads.append(torch.softmax(z, 1) @ v[i, :, h * KV // HEADS])
        rows.append(torch.cat(heads, 1))
    z = torch.stack(rows) @ wo.transpose(1, 2)
    mask, scale = kept
    return x + torch.where(mask, z * scale, 0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_training_step(mods, dtype):
    psgd = mods[2]
    X, x, dy, starts, positions = made(dtype)
    G = torch.zeros_like(X)
    kept = forward(mods, X, x, starts, positions)
    dx = backward(mods, X, G, x, dy, starts, positions, kept)
    X64, x64 = X.cpu().double().requires_grad_(), x.cpu().double().requires_grad_()
    y64 = reference(X64, x64, starts.cpu(), positions.cpu(), orc.dropped(N, T, C, P, SEED, STEP))
    y64.backward(dy.cpu().double())
    # six operators in a row, each off by a few halves of its type (their own tests bound them): 2^-8 or 2^-24 times the square root of the sums' lengths, of
    # which a relative distance of the whole takes the mean; a mistake in any of them is a hundred times that
    near = 4e-2 if dtype == BF16 else 1e-5
    for got, want, what in ((kept[5], y64.detach(), "y"), (dx, x64.grad, "dx"), (G[:, :SIZE], X64.grad[:, :SIZE], "G")):
        far = float((got.cpu().double() - want).norm() / want.norm())
        assert far <= near, (what, far)
    assert (G[:, SIZE:] == 0).all()
    if dtype == F32:
        nbr, w = psgd.build_mixing(psgd.TOPO_RING, N)
        out = torch.empty_like(X)
        psgd.mix_step(X, out, G, torch.from_numpy(nbr).to("cuda:0"), torch.from_numpy(w).to("cuda:0"), 0.1)
        assert torch.isfinite(out).all()


def test_serving_token_by_token(mods):
    """The same block without dropout, fed a token at a time: the rows of the whole, from caches that are rings of the window."""
    attention, layers, _ = mods
    X, x, _, _, _ = made(F32)
    w, gq, gk, wo = parameters(X)
    a = torch.empty((N, T, Q + 2 * K), device="cuda:0")
    layers.linear(x, w, a)
    q, k, v = a.split((Q, K, K), 2)
    qr, kr, whole = torch.empty((N, T, Q), device="cuda:0"), torch.empty((N, T, K), device="cuda:0"), torch.empty((N, T, Q), device="cuda:0")
    attention.qk_norm_rope(q, k, qr, kr, HEADS, KV, q_gain=gq, k_gain=gk)
    attention.attention(qr, kr, v, whole, HEADS, KV, window=WINDOW, sinks=SINKS)
    caches = [torch.empty((N, 1, WINDOW + SINKS, K), device="cuda:0") for _ in range(2)]
    lengths, tok = torch.zeros((N, 1), dtype=torch.int32, device="cuda:0"), torch.empty((N, 1, Q + 2 * K), device="cuda:0")
    out = torch.empty((N, 1, Q), device="cuda:0")
    for i in range(T):
        layers.linear(x[:, i:i + 1], w, tok)
        q1, k1, v1 = tok.split((Q, K, K), 2)
        attention.qk_norm_rope(q1, k1, q1, k1, HEADS, KV, positions=lengths, q_gain=gq, k_gain=gk)
        attention.attention_step(q1, k1, v1, *caches, lengths, out, HEADS, KV, window=WINDOW, sinks=SINKS)
        # both sides are fp32 all the way: sums of 40, 16 and 22 terms in another order
        assert float((out[:, 0] - whole[:, i]).abs().max()) <= 1e-5 * float(whole[:, i].abs().max())
        lengths += 1
