"""A data-parallel training step on R virtual ranks, as the library's calls make it up:

    logits of every rank's tokens (torch)  ->  policy_loss: loss and gradient of the logits
    ->  gradients of the parameters into the rank's bucket (torch)  ->  all-reduce of the buckets (collective_noalloc)
    ->  grad_norm of the reduced bucket  ->  adamw, which clips by it

The policy is one linear layer over given hidden states, in bf16 with fp32 parameters and moments.  Everything goes onto one stream
and allocates nothing, so the step can be captured into a HIP graph.  `python -m paper_2303_06324_amd.example_step` trains for a
few steps, eagerly and by replays of the graph, and checks that all ranks end with the same parameters.
"""
from __future__ import annotations

import torch

import paper_2303_06324_amd as dfx


class Rank:
    """What one virtual rank holds: its tokens, and parameters, gradients and moments, each flat with the layer's tensors in it."""

    def __init__(self, seed: int, rows: int, hidden: int, vocab: int, init: torch.Tensor):
        gen = torch.Generator("cuda").manual_seed(seed)
        dev = {"device": "cuda"}
        self.rows, self.vocab = rows, vocab
        self.hidden = torch.empty(rows, hidden, dtype=torch.bfloat16, **dev).normal_(generator=gen)
        self.targets = torch.randint(0, vocab, (rows,), generator=gen, **dev)
        self.weight = (torch.rand(rows, generator=gen, **dev) < 0.8).float()
        self.advantage = torch.empty(rows, **dev).normal_(generator=gen)
        self.old = torch.zeros(rows, **dev)
        n = init.numel()
        self.params = init.clone()
        self.copies = init.to(torch.bfloat16)
        self.grads = torch.zeros(n, dtype=torch.bfloat16, **dev)       # the bucket
        self.reduced = torch.zeros(n, dtype=torch.bfloat16, **dev)
        self.m, self.v = torch.zeros(n, **dev), torch.zeros(n, **dev)
        cut = vocab * hidden
        self.w, self.b = self.copies[:cut].view(vocab, hidden), self.copies[cut:]
        self.gw, self.gb = self.grads[:cut].view(vocab, hidden), self.grads[cut:]
        self.logits = torch.empty(rows, vocab, dtype=torch.bfloat16, **dev)
        self.logp, self.loss, self.sums = torch.empty(rows, **dev), torch.empty(rows, **dev), torch.empty(5, **dev)
        self.count, self.total, self.scale = torch.empty(4, **dev), torch.empty(4, **dev), torch.empty((), **dev)
        self.norm = torch.empty((), **dev)
        nbytes = dfx.policy_loss_workspace(rows, vocab, dfx.BF16)
        self.work, self.work_bytes = torch.empty(nbytes, dtype=torch.uint8, **dev), nbytes

        def named(flat, kind):
            at = flat.data_ptr()
            return dfx.TensorList([(at, cut, kind), (at + cut * flat.element_size(), n - cut, kind)])

        self.lists = {"p": named(self.params, dfx.F32), "m": named(self.m, dfx.F32), "v": named(self.v, dfx.F32),
                      "g": named(self.reduced, dfx.BF16), "copy": named(self.copies, dfx.BF16)}

    def forward(self):
        torch.mm(self.hidden, self.w.t(), out=self.logits)
        self.logits.add_(self.b)

    def score(self, stream: int, out: torch.Tensor):
        """Log-probabilities of the targets under the present parameters."""
        self.forward()
        dfx.policy_loss(self.rows, self.vocab, dfx.BF16, self.logits.data_ptr(), self.targets.data_ptr(), weight=self.weight.data_ptr(),
                        logp=out.data_ptr(), workspace=self.work.data_ptr(), workspace_bytes=self.work_bytes, stream=stream)

    def backward(self, stream: int):
        """Loss, the logits' gradient in the logits' place, and the parameters' gradients in the bucket."""
        self.forward()
        z = self.logits.data_ptr()
        dfx.policy_loss(self.rows, self.vocab, dfx.BF16, z, self.targets.data_ptr(), old_logp=self.old.data_ptr(),
                        ref_logp=self.old.data_ptr(), advantage=self.advantage.data_ptr(), weight=self.weight.data_ptr(),
                        scale=self.scale.data_ptr(), logp=self.logp.data_ptr(), loss=self.loss.data_ptr(), sums=self.sums.data_ptr(), grad=z,
                        clip_high=0.28, kl_coef=0.01, workspace=self.work.data_ptr(), workspace_bytes=self.work_bytes, stream=stream)
        torch.mm(self.logits.t(), self.hidden, out=self.gw)
        torch.sum(self.logits, 0, out=self.gb)

    def update(self, config, stream: int):
        dfx.grad_norm(self.lists["g"], self.norm.data_ptr(), stream=stream)
        dfx.adamw(self.lists["p"], self.lists["g"], self.lists["m"], self.lists["v"], config, copies=self.lists["copy"],
                  norm=self.norm.data_ptr(), stream=stream)


class Trainer:
    def __init__(self, ranks: int = 8, rows: int = 64, hidden: int = 256, vocab: int = 2011, seed: int = 0, lr: float = 1e-3):
        init = torch.empty(vocab * hidden + vocab, device="cuda").normal_(0.0, 0.05, generator=torch.Generator("cuda").manual_seed(seed))
        self.ranks = [Rank(seed + 1 + r, rows, hidden, vocab, init) for r in range(ranks)]
        self.step_no = torch.zeros((), dtype=torch.int32, device="cuda")
        self.config = dfx.AdamWConfig(lr=lr, beta2=0.95, weight_decay=0.01, step_dev=self.step_no.data_ptr(), max_norm=1.0)
        stream = torch.cuda.current_stream().cuda_stream
        for r in self.ranks:                    # the tokens were sampled under the first parameters
            r.score(stream, r.old)

    def _all_reduce(self, sends, recvs, kind: int, stream: int):
        rc = dfx.collective_noalloc(len(sends), dfx.ALLREDUCE, sends[0].numel(), kind, dfx.SUM, 0, [t.data_ptr() for t in sends],
                                    [t.data_ptr() for t in recvs], 0, stream)
        if rc != dfx.OK:
            raise dfx.DfxError(rc, "dfx_collective_noalloc")

    def step(self):
        """One step on the current stream."""
        stream = torch.cuda.current_stream().cuda_stream
        self.step_no.add_(1)
        for r in self.ranks:                    # the loss is a mean over all ranks' tokens
            torch.sum(r.weight, 0, out=r.count[0])
        self._all_reduce([r.count for r in self.ranks], [r.total for r in self.ranks], dfx.F32, stream)
        for r in self.ranks:
            torch.reciprocal(r.total[0], out=r.scale)
            r.backward(stream)
        self._all_reduce([r.grads for r in self.ranks], [r.reduced for r in self.ranks], dfx.BF16, stream)
        for r in self.ranks:
            r.update(self.config, stream)

    def loss(self) -> float:
        return float(sum(r.sums[0] for r in self.ranks) / sum(r.sums[4] for r in self.ranks))

    def capture(self) -> "torch.cuda.CUDAGraph":
        """The step as a graph; it has to have run eagerly before."""
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            self.step()
        return graph


def main():
    for what in ("eager", "graph"):
        t = Trainer()
        t.step()
        print(what, "step 1: loss %.4f" % t.loss(), flush=True)
        run = t.step if what == "eager" else t.capture().replay
        for k in range(2, 21):
            run()
            if k % 5 == 0:
                torch.cuda.synchronize()
                print(what, "step %d: loss %.4f norm %.4f" % (k, t.loss(), float(t.ranks[0].norm)), flush=True)
        assert all(torch.equal(r.params, t.ranks[0].params) for r in t.ranks)
    print("all ranks hold the same parameters")


if __name__ == "__main__":
    main()
