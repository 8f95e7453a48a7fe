"""The training step that the operators make up with the all-reduce (paper_2303_06324_amd/example_step.py): against torch's own gradients
and an update in 64 bits, the same on every rank, and replayed from a graph with eager work in between."""
import numpy as np
import pytest

from oracle import step as st

pytestmark = pytest.mark.gpu


def _trainer(**kw):
    from paper_2303_06324_amd import example_step as ex
    return ex.Trainer(ranks=4, rows=24, hidden=64, vocab=501, **kw)


def test_first_step_against_torch():
    """The gradient of the mean over all ranks' tokens by torch's autograd in 64 bits on the same bf16 parameters.  Logits, their gradient and
    the bucket are bf16 (2^-8 of their size each), the reduction rounds once a rank: the gradient as a whole is within 2 % of its norm."""
    import torch
    t = _trainer()
    before = [r.params.double().cpu() for r in t.ranks]
    w = t.ranks[0].copies.double().cpu().requires_grad_()
    vocab, hidden = 501, 64
    cut = vocab * hidden
    total, count = 0.0, sum(float(r.weight.sum()) for r in t.ranks)
    for r in t.ranks:
        z = r.hidden.double().cpu() @ w[:cut].view(vocab, hidden).t() + w[cut:]
        logp = torch.log_softmax(z, 1).gather(1, r.targets.cpu()[:, None])[:, 0]
        old, a = r.old.double().cpu(), r.advantage.double().cpu()
        ratio = torch.exp(logp - old)
        pg = -torch.minimum(ratio * a, ratio.clamp(0.8, 1.28) * a)
        d = old - logp
        total = total + (r.weight.double().cpu() * (pg + 0.01 * (torch.exp(d) - d - 1))).sum() / count
    total.backward()
    t.step()
    torch.cuda.synchronize()
    got = t.ranks[0].reduced.double().cpu()
    assert float((got - w.grad).norm() / w.grad.norm()) < 0.02
    total = float(total.detach())
    assert abs(t.loss() - total) < 0.02 * (abs(total) + 0.05)
    norm = st.grad_norm([got.numpy()])
    assert abs(float(t.ranks[0].norm) - norm) < 1e-6 * norm
    f = st.clip_factor(norm, 1.0)
    p, _, _ = st.adamw(before[0].numpy(), got.numpy(), 0.0 * got.numpy(), 0.0 * got.numpy(), 1, 1e-3, 0.9, 0.95, 1e-8, 0.01, f)
    assert np.abs(t.ranks[0].params.double().cpu().numpy() - p).max() < 1e-8 + 2.0 ** -22 * np.abs(p).max()
    for r in t.ranks[1:]:
        assert torch.equal(r.params, t.ranks[0].params) and torch.equal(r.copies, t.ranks[0].copies) and torch.equal(r.norm, t.ranks[0].norm)


def test_replayed_from_a_graph():
    """Replays with the program's own work and waits in between give what eager steps give, bit for bit."""
    import torch
    eager, replayed = _trainer(seed=5), _trainer(seed=5)
    eager.step()
    replayed.step()
    graph = replayed.capture()          # (capturing runs nothing)
    assert int(replayed.step_no) == 1
    for k in range(6):
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        x = torch.randn(1000, device="cuda").square().sum()
        assert float(x) > 0 and int(replayed.step_no) == int(eager.step_no) == k + 2
        for a, b in zip(eager.ranks, replayed.ranks):
            assert torch.equal(a.params, b.params) and torch.equal(a.m, b.m) and torch.equal(a.v, b.v) and torch.equal(a.copies, b.copies), k
            assert torch.equal(a.loss, b.loss) and torch.equal(a.sums, b.sums) and torch.equal(a.norm, b.norm), k
            assert torch.equal(a.params, eager.ranks[0].params)


def test_training_lowers_the_loss():
    t = _trainer(seed=9, lr=3e-3)
    t.step()
    first = t.loss()
    for _ in range(15):
        t.step()
    assert t.loss() < first - 0.01
