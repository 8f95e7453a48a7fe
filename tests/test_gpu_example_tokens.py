"""The training step from tokens to the update (paper_2303_06324_amd/example_tokens.py): against torch's own gradients in 64 bits, the same on every
rank, and replayed from a graph with eager work in between."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _trainer(**kw):
    from paper_2303_06324_amd import example_tokens as ex
    return ex.Trainer(ranks=4, **{**dict(rows=70, dim=72, vocab=501), **kw})


def test_first_step_against_torch():
    """The gradient of the mean over all ranks' tokens by torch's autograd in 64 bits on the same bf16 parameters.  Embeddings, norms, the hidden states' gradients and the
    bucket are bf16 (2^-8 of their size each, eight roundings one behind the other at most), the reduction rounds once a rank: within 3 % of its norm."""
    import torch
    t = _trainer()
    dim, vocab = 72, 501
    w = t.ranks[0].copies.double().cpu().requires_grad_()
    table, weight, bias = w[:vocab * dim].view(vocab, dim), w[vocab * dim:vocab * dim + dim], w[vocab * dim + dim:]
    total, count = 0.0, sum(float(r.valid.sum()) for r in t.ranks)
    for r in t.ranks:
        x = table[r.tokens.cpu()] * math.sqrt(dim)
        d = x - x.mean(1, keepdim=True)
        y = d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * weight + bias
        logp = torch.log_softmax(y @ table.t(), 1)
        on = r.targets.cpu() >= 0
        total = total - logp[on].gather(1, r.targets.cpu()[on][:, None]).sum() / count
    total.backward()
    t.step()
    torch.cuda.synchronize()
    total = float(total.detach())
    assert abs(t.loss() - total) < 0.01 * total
    for a, b in ((0, vocab * dim), (vocab * dim, vocab * dim + dim), (vocab * dim + dim, w.numel())):
        got, want = t.ranks[0].reduced.double().cpu()[a:b], w.grad[a:b]
        assert float((got - want).norm() / want.norm()) < 0.03
    for r in t.ranks[1:]:
        assert torch.equal(r.params, t.ranks[0].params) and torch.equal(r.copies, t.ranks[0].copies) and torch.equal(r.norm, t.ranks[0].norm)


@pytest.mark.parametrize("rows,dim", [(70, 72), (300, 128), (700, 64)])
def test_replayed_from_a_graph(rows, dim):
    """Replays with the program's own work and waits in between give what eager steps give, bit for bit."""
    import torch
    eager, replayed = _trainer(seed=5, rows=rows, dim=dim), _trainer(seed=5, rows=rows, dim=dim)
    eager.step()
    replayed.step()
    graph = replayed.capture()          # (capturing runs nothing)
    assert int(replayed.step_no) == 1
    for k in range(5):
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        x = torch.randn(1000, device="cuda").square().sum()
        assert float(x) > 0 and int(replayed.step_no) == int(eager.step_no) == k + 2
        for a, b in zip(eager.ranks, replayed.ranks):
            assert torch.equal(a.params, b.params) and torch.equal(a.m, b.m) and torch.equal(a.v, b.v) and torch.equal(a.copies, b.copies), k
            assert torch.equal(a.loss, b.loss) and torch.equal(a.sums, b.sums) and torch.equal(a.norm, b.norm) and torch.equal(a.grads, b.grads), k
            assert torch.equal(a.params, eager.ranks[0].params)
