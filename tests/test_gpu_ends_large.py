"""The operators at the two ends of a language model where offsets pass 32 bits, rows are very long or far apart, and vocabularies take several pieces by themselves.

What is looked for is a wrong address, which is as wrong as can be.  References in 64 bits by torch, in parts.  Bounds, u = 2^-24, H half a step of the type: a logit by an addition's 2 u of the sum of magnitudes each and
2^-22 of 32-bit products; logp by twice the largest of them, and (48 + V / 256 + 3 log V + 8) u; the gradients, by the norm of a row or of a matrix, 2 H (dz and the result, rounded) and 2^-10 (the sums in 32 bits and
the logits' errors, which are far below it here) of the norm of the sums of magnitudes, half the type's smallest step for each of a row's elements, and f16's of dz, 2^-40, of the sum of what it multiplies."""
import math

import pytest

from tests.test_gpu_ends import _dfx, _t, _work
from tests.test_gpu_step import HALF, TINY, U

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _give_back():
    """What the tests behind these find free is what was."""
    yield
    torch, _ = _t()
    torch.cuda.empty_cache()


def _room(gib):
    torch, _ = _t()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip("does not fit")


def _fill(rows, dim, stride, dt, std, gen):
    """Rows so far apart, in memory that is not all written: (memory, view)."""
    torch, td = _t()
    mem = torch.empty((rows - 1) * stride + dim if rows else 0, dtype=td[dt], device="cuda")
    view = torch.as_strided(mem, (rows, dim), (stride, 1))
    step = max(1, (1 << 27) // dim)
    for a in range(0, rows, step):
        view[a:a + step] = torch.randn(min(step, rows - a), dim, generator=gen, device="cuda") * std
    return mem, view


# rows, dim, vocab, stride of the weight and of its gradient: more than 2^32 elements by vocabulary (few rows in registers, past LDS and through it; tiles) or by rows far apart; rows longer than 65536; more rows
# than 65536; few rows over several pieces
LARGE = [
    (5, 4096, 1100007, 0, "bf16"), (40, 4096, 1100007, 0, "bf16"), (200, 4096, 1100007, 0, "bf16"), (9, 2050, 2100003, 0, "f16"),
    (7, 100, 5003, (1 << 20) - 8, "bf16"), (200, 128, 5003, (1 << 20) - 8, "bf16"), (200, 128, 5003, (1 << 20) - 1, "f16"), (70, 128, 4099, (1 << 20) - 1, "f32"),
    (3, 70001, 50, 0, "bf16"), (200, 70001, 300, 0, "f16"), (20, 70000, 300, 0, "f32"),
    (70000, 64, 300, 0, "bf16"), (131073, 24, 1000, 0, "f16"), (66000, 33, 200, 0, "f32"),
    (10, 64, 1100000, 0, "f32"), (100, 64, 530000, 0, "bf16"), (33, 65, 700001, 0, "f16"),
]


@pytest.mark.parametrize("rows,dim,vocab,stride,dt", LARGE)
def test_vocab_loss(rows, dim, vocab, stride, dt):
    _room(60)
    torch, td = _t()
    dfx, kinds = _dfx()
    gen = torch.Generator("cuda").manual_seed(1)
    stride = stride or dim
    wm, w = _fill(vocab, dim, stride, dt, 2.5 / math.sqrt(dim), gen)
    x = torch.randn(rows, dim, generator=gen, device="cuda").to(td[dt])
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    t[0] = vocab - 1
    if rows > 3:
        t[1], t[2] = 0, -1
    gm, g = _fill(vocab, dim, stride, dt, 0.0, gen)
    between = torch.as_strided(gm, (vocab - 1, min(stride - dim, 1000)), (stride, 1), dim) if stride > dim else None
    if between is not None:
        between.fill_(7.0)
    gx = torch.empty_like(x)
    logp = torch.empty(rows, device="cuda")
    nbytes = dfx.vocab_loss_workspace(rows, dim, vocab, kinds[dt], True)
    mem, ws, end = _work(nbytes)
    dfx.vocab_loss(rows, dim, vocab, kinds[dt], x.data_ptr(), wm.data_ptr(), t.data_ptr(), logp=logp.data_ptr(), grad_hidden=gx.data_ptr(), grad_weight=gm.data_ptr(), weight_stride=stride,
                   grad_weight_stride=stride, workspace=ws, workspace_bytes=nbytes)
    assert bool((mem[end:] == 0xA5).all())
    if between is not None:
        assert bool((between == 7.0).all())
    on = t >= 0
    X = torch.where(on[:, None], x, torch.zeros((), dtype=x.dtype, device="cuda")).double()
    part = max(1, min((1 << 26) // max(dim, rows), vocab))
    lse, zt, most = torch.full((rows,), -math.inf, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda"), 0.0
    for a in range(0, vocab, part):
        W = w[a:a + part].double()
        z = X @ W.t()
        lse = torch.logaddexp(lse, torch.logsumexp(z, 1))
        here = on & (t >= a) & (t < a + len(W))
        zt[here] = z[here, t[here] - a]
        most = max(most, float((X.abs() @ W.t().abs()).max()))
    products = 6 if dt == "f32" else 1
    ez = (2 * (dim * products + 4) * U + (2.0 ** -22 if dt == "f32" else 0)) * most
    want = torch.where(on, zt - lse, torch.zeros((), dtype=torch.float64, device="cuda"))
    assert float((logp.double() - want).abs().max()) <= 2 * ez + (48 + vocab / 256 + 3 * math.log(vocab) + 8) * U
    GX, GM, WM = torch.zeros(rows, dim, dtype=torch.float64, device="cuda"), torch.zeros(rows, dim, dtype=torch.float64, device="cuda"), torch.zeros(dim, dtype=torch.float64, device="cuda")
    bound, step = 2 * HALF[dt] + 2.0 ** -10, 2.0 ** -40 if dt == "f16" else 0.0
    least = TINY[dt] * math.sqrt(dim)
    for a in range(0, vocab, part):
        W = w[a:a + part].double()
        dz = (X @ W.t() - lse[:, None]).exp()
        here = on & (t >= a) & (t < a + len(W))
        dz[here, t[here] - a] -= 1.0
        dz[~on] = 0.0
        GX += dz @ W
        GM += dz.abs() @ W.abs()
        WM += W.abs().sum(0)
        GW, GWM = dz.t() @ X, dz.t().abs() @ X.abs()
        got = g[a:a + part].double()
        assert bool(((got - GW).norm(dim=1) <= bound * GWM.norm(dim=1) + least + step * X.abs().sum(0).norm()).all()), a
    assert bool(((gx.double() - GX).norm(dim=1) <= bound * GM.norm(dim=1) + least + step * WM.norm()).all())
    assert not gx[~on].any()


@pytest.mark.parametrize("vocab,dim,stride,dt", [(1100007, 4096, 0, "bf16"), (5003, 200, (1 << 20) - 1, "f16"), (4200, 100, (1 << 20) - 1, "f32")])
@pytest.mark.parametrize("rows", [300, 3000, 20000])
def test_embed_and_its_gradient(rows, vocab, dim, stride, dt):
    """Rows of the table beyond 2^32 elements are read, summed onto, and cleared; what lies between rows stays."""
    _room(60)
    torch, td = _t()
    dfx, kinds = _dfx()
    gen = torch.Generator("cuda").manual_seed(2)
    stride = stride or dim
    tm, table = _fill(vocab, dim, stride, dt, 1.0, gen)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    t[:3] = torch.tensor([vocab - 1, 0, vocab], device="cuda")
    out = torch.full((rows, dim), 7.0, dtype=td[dt], device="cuda")
    dfx.embed(rows, dim, vocab, kinds[dt], t.data_ptr(), tm.data_ptr(), out.data_ptr(), table_stride=stride, scale=2.0)
    on = t < vocab
    assert torch.equal(out[on], table[t[on]] * 2.0) and not out[~on].any()
    between = torch.as_strided(tm, (vocab - 1, min(stride - dim, 1000)), (stride, 1), dim) if stride > dim else None
    if between is not None:
        between.fill_(7.0)
    grad = torch.randint(-3, 4, (rows, dim), generator=gen, device="cuda").to(td[dt])      # (whole numbers: sums are exact)
    nbytes = dfx.embed_grad_workspace(rows, dim, vocab, kinds[dt])
    mem, ws, end = _work(nbytes, 16)
    distinct, at = torch.unique(t[on], return_inverse=True)
    sums = torch.zeros(len(distinct), dim, device="cuda").index_add_(0, at, grad[on].float())
    old = table[distinct].float()
    dfx.embed_grad(rows, dim, vocab, kinds[dt], t.data_ptr(), grad.data_ptr(), tm.data_ptr(), table_grad_stride=stride, accumulate=True, workspace=ws, workspace_bytes=nbytes)
    assert torch.equal(table[distinct], (old + sums).to(td[dt]))
    dfx.embed_grad(rows, dim, vocab, kinds[dt], t.data_ptr(), grad.data_ptr(), tm.data_ptr(), table_grad_stride=stride, workspace=ws, workspace_bytes=nbytes)
    assert torch.equal(table[distinct], sums.to(td[dt]))
    step = max(1, (1 << 28) // dim)
    named = sum(int((table[a:a + step] != 0).any(1).sum()) for a in range(0, vocab, step))
    assert named == int((sums != 0).any(1).sum())
    assert bool((mem[end:] == 0xA5).all()) and (between is None or bool((between == 7.0).all()))


@pytest.mark.parametrize("rows,dim,stride,dt", [(1 << 21, 2100, 0, "bf16"), (4300, 200, (1 << 20) - 1, "f16"), (4300, 9000, (1 << 20) - 1, "f32")])
def test_layer_norm_and_its_gradient(rows, dim, stride, dt):
    """Rows beyond 2^32 elements: the same bits as the same rows by themselves; the sums over rows add up."""
    _room(60)
    torch, td = _t()
    dfx, kinds = _dfx()
    gen = torch.Generator("cuda").manual_seed(3)
    stride = stride or dim
    xm, x = _fill(rows, dim, stride, dt, 1.0, gen)
    dm, dy = _fill(rows, dim, stride, dt, 1.0, gen)
    w, b = torch.randn(dim, generator=gen, device="cuda"), torch.randn(dim, generator=gen, device="cuda")
    at = torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device="cuda")
    xs, ds = x[at].contiguous(), dy[at].contiguous()
    ys, dxs = torch.empty_like(xs), torch.empty_like(xs)
    nbytes = dfx.layer_norm_grad_workspace(rows, dim, kinds[dt])
    mem, ws, end = _work(nbytes, 16)
    gb, gs = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    kw = dict(weight=w.data_ptr(), param_dtype=dfx.F32)
    dfx.layer_norm(5, dim, kinds[dt], xs.data_ptr(), ys.data_ptr(), bias=b.data_ptr(), **kw)
    dfx.layer_norm_grad(5, dim, kinds[dt], xs.data_ptr(), ds.data_ptr(), dxs.data_ptr(), **kw)
    whole = torch.zeros(dim, dtype=torch.float64, device="cuda")
    size = torch.zeros(dim, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // dim)
    for a in range(0, rows, step):
        p = dy[a:a + step].double()
        whole += p.sum(0)
        size += p.abs().sum(0)
    dfx.layer_norm_grad(rows, dim, kinds[dt], xm.data_ptr(), dm.data_ptr(), dm.data_ptr(), grad_weight=gs.data_ptr(), grad_bias=gb.data_ptr(), x_stride=stride, dy_stride=stride, dx_stride=stride,
                        workspace=ws, workspace_bytes=nbytes, **kw)
    dfx.layer_norm(rows, dim, kinds[dt], xm.data_ptr(), xm.data_ptr(), x_stride=stride, y_stride=stride, bias=b.data_ptr(), **kw)
    assert torch.equal(dy[at], dxs) and torch.equal(x[at], ys)
    assert bool(((gb.double() - whole).abs() <= (rows + 20) * U * size).all())
    assert bool((mem[end:] == 0xA5).all())
