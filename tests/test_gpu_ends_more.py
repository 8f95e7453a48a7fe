"""More of the operators at the two ends of a language model against their definitions in 64 bits: calls that went wrong once.  Tolerances as in test_gpu_ends.py."""
import numpy as np
import pytest

from tests.test_gpu_ends import Vocab, _dfx, _np, _rows, _t
from tests.test_gpu_step import HALF, TINY, U, Guarded, _near
from tests.test_vocab_plan import WIDE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,dim,vocab", [(128, 64, 78700), (100, 67, 131072), (65, 64, 200003)])
def test_few_32_bit_rows_of_a_long_vocabulary(rows, dim, vocab):
    """The planes of dz lie apart from the logits that it is made of (which rows from the 65th on found overwritten)."""
    v = Vocab(rows, dim, vocab, "f32", seed=100)
    v.run()
    v.check()


def test_more_long_rows_than_a_launch_has():
    """2^22 rows by workgroups of 1024 are one thread more than a launch counts: in place, 64 GiB."""
    torch, _ = _t()
    dfx, kinds = _dfx()
    rows, dim = (1 << 22) + 1, 8200
    if torch.cuda.mem_get_info()[0] < rows * dim * 2 + (8 << 30):
        pytest.skip("the rows do not fit")
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22], device="cuda")
    some = torch.randn(5, dim, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    x[at] = some
    want = torch.empty_like(some)
    dfx.layer_norm(5, dim, kinds["bf16"], some.data_ptr(), want.data_ptr())
    dfx.layer_norm(rows, dim, kinds["bf16"], x.data_ptr(), x.data_ptr())
    assert torch.equal(x[at], want) and bool(want.any())
    assert not x[1:2000].any() and not x[-2000:-2].any()      # (the last two are of the five)
    del x
    torch.cuda.empty_cache()


# Rows that are few and many, dim and vocab, and a piece (0: the library's): hidden states in registers, through LDS and past it; tiles of one piece, whose logits are kept, and of several
INFINITE = [(9, 1024, 520, 0), (20, 128, 700, 0), (70, 100, 700, 256), (300, 128, 700, 0), (300, 128, 700, 256), (130, 70, 700, 512)]


def _hide(v, rows):
    """The call's own arrays without some of its rows, as Vocab.check takes them: no target."""
    v.t = v.t.copy()
    v.t[rows] = -1


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,dim,vocab,piece", INFINITE)
def test_a_logit_of_plus_infinity(rows, dim, vocab, piece, dt):
    """Its row is NaN, and with it the weight's gradient; the other rows' numbers are the same bits as without it."""
    torch, _ = _t()
    v = Vocab(rows, dim, vocab, dt, seed=110, weights=None)
    v.t[5] = 1
    keep = np.delete(np.arange(rows), 5)
    v.w[:, 7] = v.w[:, 7].abs() + 0.5
    v.x[:, 7] = 0.0
    v.run(piece=piece)
    before = [v.lg.t.clone(), v.og.t.clone(), v.gh.clone()]
    v.x[5, 7] = float("inf")
    v.run(piece=piece)
    for a, b in zip(before, (v.lg.t, v.og.t, v.gh)):
        assert torch.equal(a[keep], b[keep])
    assert bool(v.lg.t[5].isnan()) and bool(v.og.t[5].isnan()) and bool(v.gh[5].isnan().all()) and bool(v.gw.isnan().any()) and bool(v.sg.t[0].isnan())


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows,dim,vocab,piece", INFINITE)
def test_a_row_without_a_logit_above_minus_infinity(rows, dim, vocab, piece, dt):
    """It has nothing to learn from: zeros, no weight in the sums, and no part in the weight's gradient, infinite as its hidden state is."""
    v = Vocab(rows, dim, vocab, dt, seed=120, weights=None)
    v.t[5], v.t[6] = 1, 2
    v.w[:, 7] = -v.w[:, 7].abs() - 0.5
    v.x[:, 7] = 0.0
    v.x[5:7, 7] = float("inf")
    v.run(piece=piece)
    assert float(v.lg.t[5]) == 0.0 and float(v.og.t[6]) == 0.0 and not v.gh[5:7].any()
    v.x[5:7, 7] = 0.0
    _hide(v, [5, 6])
    v.check()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows,dim,vocab,piece", INFINITE)
def test_a_token_of_minus_infinity(rows, dim, vocab, piece, dt):
    """A row of the weight whose logits are all -infinity has probability 0, and its gradient is 0 (that of the hidden states, 0 times an infinity, is NaN by its definition)."""
    v = Vocab(rows, dim, vocab, dt, seed=130, weights=None)
    v.x[:, 7] = v.x[:, 7].abs() + 0.5
    off = vocab - 300                          # (not in the last of several pieces)
    v.t[v.t == off] = off - 1
    v.w[off] = 0.0
    v.w[off, 7] = -float("inf")
    v.run(piece=piece, hidden=False)
    got = _np(v.gw)
    assert not np.isnan(v.lg.host()).any() and not np.isnan(got).any() and not got[off].any()
    # the other tokens: as if that one were not there
    v.w[off] = 0.0
    v.w[off, 7] = -1000.0                      # (far below all others: probability 0 as well)
    v.run(piece=piece, hidden=False)
    assert np.array_equal(np.delete(_np(v.gw), off, 0), np.delete(got, off, 0))


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", WIDE, ids=lambda c: "x".join(map(str, c[0])))
def test_wide_tiles(case, dt):
    """The weight read in place where its rows are whole steps, by a stride and without one; and at odd places, the gradient in 32 bits and onto what is there."""
    rows, dim, vocab, piece = case[0]
    for more, off, onto, gt in ((8 if dim % 64 == 0 else 0, 0, False, dt), (3, 1, True, "f32")):
        v = Vocab(rows, dim, vocab, dt, gt, more=more, off=off, seed=140)
        v.run(onto=onto, piece=piece)
        v.check(onto=onto)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,dim", [(1, 4000), (40, 4000), (40, 4096), (100, 3001)])
def test_logits_of_few_long_rows(rows, dim, dt):
    """The error of logp over many rows, by their root mean square: additions on the matrix cores cost up to 2 u of the sum that they meet, evenly spread (2 / sqrt 3 u), and one takes 32
    products.  Where blocks are added up, of B steps of 64 elements and with P products of each (1, or 6 of 32 bits), the sum grows to Z sqrt(f) over a fraction f of the row: 2 P dim / 64 additions inside
    of blocks of B / (dim / 64) of the row, and dim / (64 B) of blocks, rounded.  The sum of exponentials costs as much again, its logarithm and the rest 8 u.  (As one sum, the 32-bit rows were beyond.)"""
    torch, _ = _t()
    dfx, kinds = _dfx()
    vocab, errors, sizes = 1000, [], []
    for seed in range(max(1, 40 // rows)):
        gen = torch.Generator("cuda").manual_seed(seed)
        T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dt]
        w = (torch.randn(vocab, dim, generator=gen, device="cuda") * (2.5 / dim ** 0.5)).to(T)
        t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        x = (torch.randn(rows, dim, generator=gen, device="cuda") + torch.rand(rows, 1, generator=gen, device="cuda") * 2 * w[t].float()).to(T)
        logp = torch.empty(rows, device="cuda")
        nbytes = dfx.vocab_loss_workspace(rows, dim, vocab, kinds[dt])
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        dfx.vocab_loss(rows, dim, vocab, kinds[dt], x.data_ptr(), w.data_ptr(), t.data_ptr(), logp=logp.data_ptr(), workspace=work.data_ptr(), workspace_bytes=nbytes)
        z = x.double().cpu() @ w.double().cpu().t()
        zt = z.gather(1, t.cpu()[:, None])[:, 0]
        errors.append((logp.double().cpu() - (zt - torch.logsumexp(z, 1))).numpy())
        sizes.append(zt.numpy())
    rms = lambda a: float(np.sqrt(np.mean(np.concatenate(a) ** 2)))
    steps, block, products = dim / 64, 3 if dt == "f32" else 8, 6 if dt == "f32" else 1
    inside = 2 * products * steps * 0.5 * (block / steps) * 4 / 3
    between = steps / (2 if dt == "f32" else 8) * 0.5 / 3
    assert rms(errors) <= (2 ** 0.5 * (inside + between) ** 0.5 * rms(sizes) + 8) * U, (rms(errors) / U, rms(sizes))


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,dim,vocab,piece", [(1, 64, 300, 0), (20, 1024, 300, 0), (70, 100, 700, 256), (300, 64, 700, 0), (300, 64, 700, 256)])
def test_expected_tokens(rows, dim, vocab, piece, dt):
    """A target that is all but certain (1 - p mostly of 1e-9 to 1e-2): logp, and the gradients that are made of 1 - p, keep their digits.  The other tokens' sum R is off by the errors of their logits and of the
    target's, 8 u for each exponential and its place in the sums, and (48 + V / 256) u as in test_gpu_ends.py, all relative to R; dz by that, and rounded to the inputs' type (f16: to half a step of 2^-39
    of the weight at least)."""
    torch, td = _t()
    dfx, kinds = _dfx()
    gen = torch.Generator("cuda").manual_seed(150)
    w = (torch.randn(vocab, dim, generator=gen, device="cuda") * (2.5 / dim ** 0.5)).to(td[dt])
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    x = (w[t].float() * (2.0 + 2.0 * torch.rand(rows, 1, generator=gen, device="cuda"))).to(td[dt])
    lg, hg, vg = Guarded(rows, "f32"), Guarded(rows * dim, dt), Guarded(vocab * dim, "f32")
    nbytes = dfx.vocab_loss_workspace(rows, dim, vocab, kinds[dt], True, piece)
    work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    dfx.vocab_loss(rows, dim, vocab, kinds[dt], x.data_ptr(), w.data_ptr(), t.data_ptr(), logp=lg.ptr(), grad_hidden=hg.ptr(), grad_weight=vg.ptr(), grad_dtype=dfx.F32, piece=piece,
                   workspace=work.data_ptr(), workspace_bytes=nbytes)
    X, W, at = _np(x), _np(w), np.arange(rows)
    z = X @ W.T
    far = z[at, t.cpu().numpy()][:, None] - z
    others = np.exp(-far)
    others[at, t.cpu().numpy()] = 0.0
    R = others.sum(1, keepdims=True)
    assert float(R.max()) < 1.0 and float(np.median(R)) < 1e-2      # (what the inputs are meant to be)
    logp = -np.log1p(R[:, 0])
    left = 2.0 ** -22 if dt == "f32" else 0.0
    ez = (2 * (dim * (6 if dt == "f32" else 1) + 4) * U + left) * (np.abs(X) @ np.abs(W).T)
    rel = (ez + ez[at, t.cpu().numpy()][:, None] + (8 + 3 * far) * U)      # of each other token's exponential
    eR = (others * rel).sum(1, keepdims=True) + (48 + vocab / 256 + 8) * U * R
    _near(lg.host(), logp, eR[:, 0] + 2 * U * np.abs(logp), "logp")
    p = others / (1 + R)
    dz = p.copy()
    dz[at, t.cpu().numpy()] = -(R / (1 + R))[:, 0]
    edz = p * (rel + eR + 8 * U)
    edz[at, t.cpu().numpy()] = (eR * (1 + 2 * R) + 8 * U * R)[:, 0]
    edz = edz + HALF[dt] * np.abs(dz) + (2.0 ** -40 if dt == "f16" else 0.0)
    product = 2 * (max(rows, vocab) * (6 if dt == "f32" else 1) + 300) * U + left
    want = dz @ W
    _near(hg.host().reshape(rows, dim), want, edz @ np.abs(W) + product * (np.abs(dz) @ np.abs(W)) + (HALF[dt] + 4 * U) * np.abs(want) + TINY[dt], "grad_hidden")
    want = dz.T @ X
    _near(vg.host().reshape(vocab, dim), want, edz.T @ np.abs(X) + product * (np.abs(dz).T @ np.abs(X)) + 4 * U * np.abs(want), "grad_weight")


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("rows,dim,vocab,piece", INFINITE)
def test_a_target_of_nan_among_minus_infinities(rows, dim, vocab, piece, dt):
    """The target's logit is not in the sum of the others: its NaN makes the row NaN all the same, and the rest of that token's column."""
    v = Vocab(rows, dim, vocab, dt, seed=160, weights=None)
    v.t[5] = 1
    v.w[:, 7] = -v.w[:, 7].abs() - 0.5
    v.x[:, 7] = 0.0
    v.x[5, 7] = float("inf")
    v.w[1, 7] = float("nan")
    v.run(piece=piece)
    on = (v.t >= 0) & (v.t < vocab)
    assert np.isnan(v.lg.host()[on]).all() and np.isnan(v.og.host()[on]).all() and bool(v.gh[5].isnan().all()) and not v.lg.host()[~on].any()
