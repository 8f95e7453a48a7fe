"""A data-parallel training step from tokens to the update, on R virtual ranks, as the library's calls make it up:

    tokens  ->  embed  ->  layer_norm  ->  vocab_loss against the next tokens: loss, gradients of the hidden states and of the table
    ->  layer_norm_grad  ->  embed_grad onto the table's gradient  ->  all-reduce of the bucket (collective_noalloc)
    ->  grad_norm of the reduced bucket  ->  adamw, which clips by it

The model is what lies at a language model's two ends and nothing in between: a table of embeddings that is the head's weight as well, and a
layer norm, in bf16 with fp32 parameters and moments.  Everything goes onto one stream and allocates nothing, so the step can be captured into a
HIP graph.  `python -m paper_2303_06324_amd.example_tokens` trains for a few steps, eagerly and by replays of the graph, and checks that
all ranks end with the same parameters.
"""
from __future__ import annotations

import math

import torch

import paper_2303_06324_amd as dfx


class Rank:
    """What one virtual rank holds: its text, and parameters, gradients and moments, each flat with the model's tensors in it."""

    def __init__(self, text: torch.Tensor, dim: int, vocab: int, init: torch.Tensor):
        dev = {"device": "cuda"}
        self.rows, self.dim, self.vocab = text.numel(), dim, vocab
        self.tokens = text.clone()
        self.targets = torch.cat([text[1:], torch.full((1,), -1, dtype=torch.int64, **dev)])      # the last token has none behind it
        n = init.numel()
        self.params = init.clone()
        self.copies = init.to(torch.bfloat16)
        self.grads = torch.zeros(n, dtype=torch.bfloat16, **dev)       # the bucket
        self.reduced = torch.zeros(n, dtype=torch.bfloat16, **dev)
        self.m, self.v = torch.zeros(n, **dev), torch.zeros(n, **dev)
        cut = vocab * dim
        self.places = (0, cut, cut + dim)      # of the table, the norm's weight and its bias
        self.x, self.y, self.dy = (torch.empty(self.rows, dim, dtype=torch.bfloat16, **dev) for _ in range(3))
        self.loss, self.sums = torch.empty(self.rows, **dev), torch.empty(2, **dev)
        self.count, self.total, self.scale = torch.empty(4, **dev), torch.empty(4, **dev), torch.empty((), **dev)
        self.valid = (self.targets >= 0).float()
        self.norm = torch.empty((), **dev)
        sizes = (dfx.vocab_loss_workspace(self.rows, dim, vocab, dfx.BF16, grad=True), dfx.layer_norm_grad_workspace(self.rows, dim, dfx.BF16),
                 dfx.embed_grad_workspace(self.rows, dim, vocab, dfx.BF16))
        self.work = torch.empty(max(sizes), dtype=torch.uint8, **dev)      # one behind the other: one workspace for all

        def named(flat, kind):
            ends = self.places[1:] + (n,)
            return dfx.TensorList([(flat.data_ptr() + a * flat.element_size(), b - a, kind) for a, b in zip(self.places, ends)])

        self.lists = {"p": named(self.params, dfx.F32), "m": named(self.m, dfx.F32), "v": named(self.v, dfx.F32),
                      "g": named(self.reduced, dfx.BF16), "copy": named(self.copies, dfx.BF16)}

    def step(self, stream: int):
        """Loss and all gradients, in the bucket."""
        rows, dim, vocab = self.rows, self.dim, self.vocab
        table, weight, bias = (self.copies[a:].data_ptr() for a in self.places)
        g_table, g_weight, g_bias = (self.grads[a:].data_ptr() for a in self.places)
        work = {"workspace": self.work.data_ptr(), "workspace_bytes": self.work.numel(), "stream": stream}
        x, y, dy, tokens = self.x.data_ptr(), self.y.data_ptr(), self.dy.data_ptr(), self.tokens.data_ptr()
        dfx.embed(rows, dim, vocab, dfx.BF16, tokens, table, x, scale=math.sqrt(dim), stream=stream)
        dfx.layer_norm(rows, dim, dfx.BF16, x, y, weight=weight, bias=bias, stream=stream)
        dfx.vocab_loss(rows, dim, vocab, dfx.BF16, y, table, self.targets.data_ptr(), scale=self.scale.data_ptr(), loss=self.loss.data_ptr(),
                       sums=self.sums.data_ptr(), grad_hidden=dy, grad_weight=g_table, **work)
        dfx.layer_norm_grad(rows, dim, dfx.BF16, x, dy, dy, weight=weight, grad_weight=g_weight, grad_bias=g_bias, **work)
        dfx.embed_grad(rows, dim, vocab, dfx.BF16, tokens, dy, g_table, scale=math.sqrt(dim), accumulate=True, **work)

    def update(self, config, stream: int):
        dfx.grad_norm(self.lists["g"], self.norm.data_ptr(), stream=stream)
        dfx.adamw(self.lists["p"], self.lists["g"], self.lists["m"], self.lists["v"], config, copies=self.lists["copy"],
                  norm=self.norm.data_ptr(), stream=stream)


class Trainer:
    def __init__(self, ranks: int = 8, rows: int = 256, dim: int = 128, vocab: int = 2011, seed: int = 0, lr: float = 3e-3):
        gen = torch.Generator("cuda").manual_seed(seed)
        init = torch.empty(vocab * dim + 2 * dim, device="cuda").normal_(0.0, 0.05, generator=gen)
        init[vocab * dim:] = 0.0
        init[vocab * dim:vocab * dim + dim] = 1.0
        follow = torch.randperm(vocab, generator=gen, device="cuda")      # the text: a token has one that mostly follows it
        self.ranks = []
        for _ in range(ranks):
            text = [torch.randint(0, vocab, (1,), generator=gen, device="cuda")]
            noise = torch.rand(rows, generator=gen, device="cuda") < 0.2
            other = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
            for k in range(1, rows):
                text.append(torch.where(noise[k], other[k:k + 1], follow[text[-1]]))
            self.ranks.append(Rank(torch.cat(text), dim, vocab, init))
        self.step_no = torch.zeros((), dtype=torch.int32, device="cuda")
        self.config = dfx.AdamWConfig(lr=lr, beta2=0.95, weight_decay=0.01, step_dev=self.step_no.data_ptr(), max_norm=1.0)

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
            torch.sum(r.valid, 0, out=r.count[0])
        self._all_reduce([r.count for r in self.ranks], [r.total for r in self.ranks], dfx.F32, stream)
        for r in self.ranks:
            torch.reciprocal(r.total[0], out=r.scale)
            r.step(stream)
        self._all_reduce([r.grads for r in self.ranks], [r.reduced for r in self.ranks], dfx.BF16, stream)
        for r in self.ranks:
            r.update(self.config, stream)

    def loss(self) -> float:
        return float(sum(r.sums[0] for r in self.ranks) / sum(r.sums[1] for r in self.ranks))

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
        for k in range(2, 41):
            run()
            if k % 10 == 0:
                torch.cuda.synchronize()
                print(what, "step %d: loss %.4f norm %.4f" % (k, t.loss(), float(t.ranks[0].norm)), flush=True)
        assert all(torch.equal(r.params, t.ranks[0].params) for r in t.ranks)
    print("all ranks hold the same parameters")


if __name__ == "__main__":
    main()
