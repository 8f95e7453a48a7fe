"""The operators at the two ends of a language model on streams of their own, and as graphs that are replayed at once.

Last of all: streams share a few hardware queues, and which of them a later context's daemon gets depends on the streams that the process has used.  A copy to the host
that lands behind a daemon that does not leave by itself (quit_idle_us = 0) waits until it is stopped, so that tests which look at results beside one run before this.
"""
import pytest

from tests.test_gpu_ends import EPS, _dfx, _t

pytestmark = pytest.mark.gpu


def test_ends_on_other_streams():
    """Two streams at once, each with its own memory, behind work that makes their inputs; then as two graphs, replayed together with eager work between."""
    torch, td = _t()
    dfx, kinds = _dfx()
    rows, dim, vocab = 200, 192, 1100
    kind = kinds["bf16"]

    class Side:
        def __init__(self, seed):
            gen = torch.Generator("cuda").manual_seed(seed)
            new = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")
            self.tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
            self.targets = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
            self.source = torch.randn(vocab, dim, generator=gen, device="cuda")
            self.table, self.x, self.h, self.dh, self.dx = new(vocab, dim), new(rows, dim), new(rows, dim), new(rows, dim), new(rows, dim)
            self.gt, self.gw, self.gb = (new(*s, dtype=torch.float32) for s in ((vocab, dim), (dim,), (dim,)))
            self.logp = new(rows, dtype=torch.float32)
            sizes = (dfx.embed_grad_workspace(rows, dim, vocab, kind), dfx.layer_norm_grad_workspace(rows, dim, kind), dfx.vocab_loss_workspace(rows, dim, vocab, kind, True))
            self.work = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
            self.sizes = sizes
            self.stream = torch.cuda.Stream()

        def run(self):
            s = torch.cuda.current_stream().cuda_stream
            self.table.copy_(self.source)
            dfx.embed(rows, dim, vocab, kind, self.tokens.data_ptr(), self.table.data_ptr(), self.x.data_ptr(), scale=3.0, stream=s)
            dfx.layer_norm(rows, dim, kind, self.x.data_ptr(), self.h.data_ptr(), eps=EPS, stream=s)
            dfx.vocab_loss(rows, dim, vocab, kind, self.h.data_ptr(), self.table.data_ptr(), self.targets.data_ptr(), logp=self.logp.data_ptr(), grad_hidden=self.dh.data_ptr(),
                           grad_weight=self.gt.data_ptr(), grad_dtype=dfx.F32, workspace=self.work[2].data_ptr(), workspace_bytes=self.sizes[2], stream=s)
            dfx.layer_norm_grad(rows, dim, kind, self.x.data_ptr(), self.dh.data_ptr(), self.dx.data_ptr(), grad_weight=self.gw.data_ptr(), grad_bias=self.gb.data_ptr(), grad_dtype=dfx.F32,
                                eps=EPS, workspace=self.work[1].data_ptr(), workspace_bytes=self.sizes[1], stream=s)
            dfx.embed_grad(rows, dim, vocab, kind, self.tokens.data_ptr(), self.dx.data_ptr(), self.gt.data_ptr(), out_dtype=dfx.F32, scale=3.0, accumulate=True,
                           workspace=self.work[0].data_ptr(), workspace_bytes=self.sizes[0], stream=s)

        def outputs(self):
            return [self.logp, self.gt, self.gw, self.gb, self.dx]

    sides = [Side(90), Side(91)]
    want = []
    for side in sides:
        side.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in side.outputs()])

    def clear():
        for side in sides:
            for t in side.outputs() + [side.table, side.x, side.h]:
                t.zero_()
        torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        for side, w in zip(sides, want):
            for a, b in zip(side.outputs(), w):
                assert torch.equal(a, b)

    clear()
    for _ in range(3):
        for side in sides:
            with torch.cuda.stream(side.stream):
                side.run()
    same()
    graphs = []
    for side in sides:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            side.run()
    for _ in range(4):
        clear()
        for side, graph in zip(sides, graphs):
            with torch.cuda.stream(side.stream):
                graph.replay()
        same()
        sides[0].run()                         # eager work between
        same()
