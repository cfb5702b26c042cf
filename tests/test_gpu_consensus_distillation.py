"""The example that runs the layers, the losses and the averaging step together: its gradients against automatic ones in 64 bits, and that the
learners learn."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def demo():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    spec = importlib.util.spec_from_file_location("consensus_distillation", os.path.join(ROOT, "examples", "consensus_distillation.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(p, x):
    f = torch.nn.functional
    norm = lambda v, g, b: f.layer_norm(v, (v.shape[-1],)) * p[g][:, None] + p[b][:, None]  # noqa: E731
    product = lambda v, w: torch.matmul(v, p[w].transpose(1, 2)) + p[w + "_bias"][:, None]  # noqa: E731
    h = f.gelu(product(norm(x, "norm1", "shift1"), "up"))
    x = x + product(h, "down")
    return product(norm(x, "norm2", "shift2"), "head")


def test_gradients_are_those_of_the_whole(demo):
    run = demo.Run(n=3, t=10, seed=4)
    for _ in range(3):
        run.step()
    x, target = run.batch()
    run.gradients(x, target)
    torch.cuda.synchronize()
    X = run.X.detach().cpu().double().requires_grad_(True)
    p, x64 = demo.views(X), x.cpu().double()
    logq = torch.log_softmax(plain_logits(p, x64), 2)
    loss = -(1.0 - demo.CONSENSUS_SHARE) / run.t * logq.gather(2, target.cpu().long()[:, :, None]).sum()
    with torch.no_grad():
        mean = X.mean(0, keepdim=True).expand_as(X).contiguous()
        teacher = plain_logits(demo.views(mean), x64)
        top = teacher.topk(demo.TOP, 2)
        share = torch.softmax(top.values / demo.TAU, 2)
    logq = torch.log_softmax(plain_logits(p, x64) / demo.TAU, 2).gather(2, top.indices)
    loss = loss + demo.CONSENSUS_SHARE / run.t * demo.TAU ** 2 * (share * (torch.log(share) - logq)).sum()
    loss.backward()
    assert torch.equal(run.top_idx.cpu().long(), top.indices)
    total = float(run.losses[0].sum() + run.losses[1].sum())
    assert abs(total - loss.item()) <= 1e-5 * abs(loss.item())
    # fp32 throughout, sums of at most 500 terms through six layers: 1e-5 of the whole gradient's size
    got = run.G.cpu().double()
    assert torch.linalg.norm(got - X.grad) <= 1e-5 * torch.linalg.norm(X.grad)


def test_learners_learn_and_agree(demo):
    run = demo.Run(n=4, t=64, seed=1)
    run.step()
    first = run.report()
    for _ in range(150):
        run.step()
    last = run.report()
    assert first[0] > 0.95 * math.log(demo.VOCABULARY)
    assert last[0] < 0.6 * first[0] and last[1] < 0.6 * first[1] and last[2] < first[2], (first, last)
    from paper_2002_01119_amd import psgd
    assert psgd.device_status() == 0
