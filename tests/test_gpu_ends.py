"""The operators at the two ends of a language model (embedding, layer norm, the vocabulary's cross entropy, and their gradients) against
their definitions in 64 bits, at the sizes, alignments, masks and values where they can go wrong.  Guard zones lie around what is written.

Tolerances, from the arithmetic and before the first run (u = 2^-24; H half a step of a result's type, which its one rounding costs):
  embed        a product in 32 bits: u, and H
  embed_grad   n places of a token added up in some grouping: n u of the sum of their magnitudes, the scale's product and the addition onto the gradient
               that is there 2 u more, and H
  layer norm   sums of a row are chains of 64 at most in a thread and 22 steps over threads: 90 u of the mean magnitude, for mean and variance; 1/sqrt(variance)
               is off by half of that and 4 u: with the product 60 u of h, and the mean's error times 1/deviation
  its gradient the same sums over g and g h, whose terms carry h's error; each product and difference u.  Sums over rows: rows + 20 additions
  vocab        z: products of 16-bit numbers are exact in 32 bits, a sum of K terms on the matrix cores is off by K 2 u of the sum of magnitudes (an addition there may
               cut off instead of rounding); 32-bit inputs leave out 2^-22 of each product.  log S by S's chain (32 + 8 + tiles) u, each exponential's 4 u and its
               exponent's rounding 3 u |c (z - m)| (mean at most log V), and z's error.
               dz: p's error (z's errors of the element and of the sum, and as above), and H of the inputs' type where it is rounded on the way, or 2^-41 of the largest weight
               (f16: half the smallest step times 2^-15); the products as above, and H
"""
import math

import numpy as np
import pytest

from oracle import ends as en
from tests.test_gpu_step import HALF, TINY, U, Guarded, _dfx, _near, _t

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16", "f16"]


def _rows(rows, dim, dtype, stride=0, off=0, fill=None, seed=0, std=1.0):
    """A matrix in guarded memory: (Guarded, view of rows)."""
    torch, td = _t()
    stride = stride or dim
    g = Guarded(max(0, (rows - 1) * stride + dim) if rows else 0, dtype, off)
    if fill is None:
        gen = torch.Generator("cuda").manual_seed(seed)
        g.t.copy_(torch.randn(g.t.numel(), generator=gen, device="cuda") * std)
    else:
        g.t.fill_(fill)
    return g, torch.as_strided(g.t, (rows, dim), (stride, 1))


def _np(t):
    return t.double().cpu().numpy()


def _work(nbytes, align=256):
    torch, _ = _t()
    w = torch.full((nbytes + align + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    at = -w.data_ptr() % align
    return w, w.data_ptr() + at, at + nbytes


def _tokens(rows, vocab, seed, none=0.1):
    rng = np.random.RandomState(seed)
    t = np.minimum((np.exp(rng.rand(rows) * math.log(vocab + 1.0))).astype(np.int64) - 1, vocab - 1)      # a few often, many seldom
    t[rng.rand(rows) < none] = -1
    return t


def _dev(a, dtype=None):
    torch, _ = _t()
    return torch.as_tensor(a, device="cuda") if dtype is None else torch.as_tensor(a, device="cuda").to(dtype)


# ------------------------------------------------------------------------------------------------------------ embedding
EMBED = [(1, 1, 1), (1, 2048, 50), (3, 7, 11), (64, 64, 100), (65, 129, 40), (300, 1001, 503), (9, 5000, 33), (2, 33000, 5)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,dim,vocab", EMBED)
def test_embed(rows, dim, vocab, dt):
    dfx, kinds = _dfx()
    for off, more, scale in ((0, 0, 1.0), (1, 3, math.sqrt(dim)), (3, 8, -0.3)):
        tg, table = _rows(vocab, dim, dt, dim + more, off, seed=1)
        og, out = _rows(rows, dim, dt, dim + 2 * more, off, fill=7.0)
        t = _tokens(rows, vocab, 5)
        if rows > 2:
            t[1] = vocab                     # one beyond the table
            t[2] = -(1 << 40)
        tok = _dev(t)
        dfx.embed(rows, dim, vocab, kinds[dt], tok.data_ptr(), tg.ptr(), og.ptr(), table_stride=dim + more, out_stride=dim + 2 * more, scale=scale)
        want = en.embed(t, _np(table), float(np.float32(scale)))
        _near(_np(out), want, (HALF[dt] + 2 * U) * np.abs(want) + TINY[dt])
        og.check()
        if more and rows > 1:                # between the rows nothing is written
            assert bool((og.t[dim:dim + 2 * more] == 7.0).all())


GRAD = [(0, 5, 3), (1, 1, 1), (1, 64, 7), (5, 7, 3), (64, 64, 100), (300, 1001, 503), (2047, 40, 9), (2049, 72, 3000), (4097, 24, 5), (9000, 16, 1 << 11), (70000, 8, 300)]


@pytest.mark.parametrize("dt,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("rows,dim,vocab", GRAD)
def test_embed_grad(rows, dim, vocab, dt, out):
    dfx, kinds = _dfx()
    for onto, more, off in ((False, 0, 0), (True, 3, 1)):
        gg, grad = _rows(rows, dim, dt, dim + more, off, seed=2)
        og, G = _rows(vocab, dim, out, dim + more, off, seed=3)
        before = _np(G)
        raw = og.t.clone()
        t = _tokens(rows, vocab, 9)
        tok = _dev(t)
        nbytes = dfx.embed_grad_workspace(rows, dim, vocab, kinds[dt])
        w, ws, end = _work(nbytes, 16)
        dfx.embed_grad(rows, dim, vocab, kinds[dt], tok.data_ptr(), gg.ptr(), og.ptr(), out_dtype=kinds[out], grad_stride=dim + more, table_grad_stride=dim + more,
                       scale=1.7, accumulate=onto, workspace=ws, workspace_bytes=nbytes)
        want, mag, many = en.embed_grad(t, _np(grad), vocab, float(np.float32(1.7)), before if onto else None)
        _near(_np(G), want, (many[:, None] + 3) * U * mag + HALF[out] * np.abs(want) + TINY[out])
        og.check()
        assert bool((w[end:] == 0xA5).all())
        if onto:                             # rows without a token, and what lies between rows, stay as they were
            torch, _ = _t()
            same = torch.as_strided(og.t, (vocab, dim), (dim + more, 1))
            for v in np.nonzero(many == 0)[0][:50]:
                assert torch.equal(same[v], torch.as_strided(raw, (vocab, dim), (dim + more, 1))[v])
            if vocab > 1:
                assert torch.equal(og.t[dim:dim + more], raw[dim:dim + more])


@pytest.mark.parametrize("rows", [100, 3000, 20000])
def test_embed_grad_of_one_token(rows):
    """Every place the same token, and none at all; twice the same bits."""
    torch, _ = _t()
    dfx, kinds = _dfx()
    dim, vocab = 130, 1 << 17
    gg, grad = _rows(rows, dim, "bf16", seed=4)
    for value in (77777, vocab - 1, -1, vocab):
        tok = torch.full((rows,), value, dtype=torch.int64, device="cuda")
        outs = []
        nbytes = dfx.embed_grad_workspace(rows, dim, vocab, kinds["bf16"])
        for _ in range(2):
            G = torch.full((vocab, dim), 3.0, dtype=torch.float32, device="cuda")
            w, ws, end = _work(nbytes, 16)
            dfx.embed_grad(rows, dim, vocab, kinds["bf16"], tok.data_ptr(), gg.ptr(), G.data_ptr(), out_dtype=dfx.F32, workspace=ws, workspace_bytes=nbytes)
            outs.append(G)
        assert torch.equal(outs[0], outs[1])
        want = _np(grad).sum(0) if 0 <= value < vocab else np.zeros(dim)
        _near(_np(outs[0][min(max(value, 0), vocab - 1)]), want, (rows + 3) * U * np.abs(_np(grad)).sum(0))
        assert int((outs[0] != 0).any(1).sum()) == (1 if 0 <= value < vocab else 0)


# ------------------------------------------------------------------------------------------------------------ layer norm
NORM = [(1, 1), (1, 64), (3, 5), (2, 511), (5, 513), (1, 4096), (33, 1001), (700, 72), (4, 2049), (3, 8192), (2, 8200), (2, 16385), (1, 32768), (1100, 2048)]
EPS = 1e-5


def _norm_tol(x, w, eps):
    """(h, r, error of h) in 64 bits."""
    h, r = en.layer_norm(x, eps)
    return h, r, r * 90 * U * np.abs(x).mean(1, keepdims=True) + 60 * U * np.abs(h)


@pytest.mark.parametrize("dt,pt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("rows,dim", NORM)
def test_layer_norm(rows, dim, dt, pt):
    dfx, kinds = _dfx()
    for off, more, shift, params in ((0, 0, 0.0, 3), (1, 3, 5.0, 2), (3, 8, -0.5, 0)):
        xg, x = _rows(rows, dim, dt, dim + more, off, seed=5)
        x += shift
        wg, w = _rows(1, dim, pt, off=off, seed=6)
        bg, b = _rows(1, dim, pt, off=off, seed=7)
        yg, y = _rows(rows, dim, dt, dim + 2 * more, off, fill=7.0)
        dfx.layer_norm(rows, dim, kinds[dt], xg.ptr(), yg.ptr(), weight=wg.ptr() if params & 1 else 0, bias=bg.ptr() if params & 2 else 0, param_dtype=kinds[pt],
                       x_stride=dim + more, y_stride=dim + 2 * more, eps=EPS)
        X, W, B = _np(x), _np(w) if params & 1 else np.ones((1, dim)), _np(b) if params & 2 else np.zeros((1, dim))
        h, r, eh = _norm_tol(X, W, EPS)
        want = h * W + B
        _near(_np(y), want, np.abs(W) * eh + 3 * U * (np.abs(h * W) + np.abs(B)) + HALF[dt] * np.abs(want) + TINY[dt])
        yg.check()
        if more and rows > 1:
            assert bool((yg.t[dim:dim + 2 * more] == 7.0).all())
        got = y.clone()                      # in place: the same bits
        yg2, y2 = _rows(rows, dim, dt, dim + more, off, fill=0.0)
        y2.copy_(x)
        dfx.layer_norm(rows, dim, kinds[dt], yg2.ptr(), yg2.ptr(), weight=wg.ptr() if params & 1 else 0, bias=bg.ptr() if params & 2 else 0, param_dtype=kinds[pt],
                       x_stride=dim + more, y_stride=dim + more, eps=EPS)
        assert bool((y2 == got).all())


@pytest.mark.parametrize("dt,pt,gt", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "bf16", "f32"), ("bf16", "f32", "bf16"), ("f16", "f16", "f32"), ("f16", "f32", "f16")])
@pytest.mark.parametrize("rows,dim", NORM + [(0, 12), (1500, 8)])
def test_layer_norm_grad(rows, dim, dt, pt, gt):
    dfx, kinds = _dfx()
    for off, more, onto in ((0, 0, False), (1, 3, True)):
        xg, x = _rows(rows, dim, dt, dim + more, off, seed=8)
        yg, dy = _rows(rows, dim, dt, dim + more, off, seed=9)
        wg, w = _rows(1, dim, pt, off=off, seed=10)
        dg, dx = _rows(rows, dim, dt, dim + more, off, fill=7.0)
        gw, GW = _rows(1, dim, gt, off=off, seed=11)
        gb, GB = _rows(1, dim, gt, off=off, seed=12)
        old_w, old_b = _np(GW)[0], _np(GB)[0]
        nbytes = dfx.layer_norm_grad_workspace(rows, dim, kinds[dt])
        mem, ws, end = _work(nbytes, 16)
        dfx.layer_norm_grad(rows, dim, kinds[dt], xg.ptr(), yg.ptr(), dg.ptr(), weight=wg.ptr(), grad_weight=gw.ptr(), grad_bias=gb.ptr(), param_dtype=kinds[pt],
                            grad_dtype=kinds[gt], x_stride=dim + more, dy_stride=dim + more, dx_stride=dim + more, eps=EPS, accumulate=onto, workspace=ws, workspace_bytes=nbytes)
        for g in (dg, gw, gb):
            g.check()
        assert bool((mem[end:] == 0xA5).all())
        X, DY, W = _np(x), _np(dy), _np(w)
        base_w, base_b = (old_w, old_b) if onto else (0 * old_w, 0 * old_b)
        if rows == 0:
            _near(_np(GW)[0], base_w, 0 * base_w)
            _near(_np(GB)[0], base_b, 0 * base_b)
            continue
        h, r, eh = _norm_tol(X, W, EPS)
        want, ww, wb = en.layer_norm_grad(X, DY, W, EPS)
        g = DY * W
        c1 = np.abs((g * h).mean(1, keepdims=True))
        tol = r * (6 * U * np.abs(g) + 92 * U * np.abs(g).mean(1, keepdims=True) + np.abs(h) * (94 * U * np.abs(g * h).mean(1, keepdims=True) + (np.abs(g) * eh).mean(1, keepdims=True))
                   + c1 * (eh + 4 * U * np.abs(h))) + 60 * U * np.abs(want)
        _near(_np(dx), want, tol + HALF[dt] * np.abs(want) + TINY[dt])
        chain = (rows + 20) * U
        tw = (np.abs(DY) * eh).sum(0) + chain * np.abs(DY * h).sum(0)
        _near(_np(GW)[0], base_w + ww, tw + 2 * U * np.abs(base_w) + HALF[gt] * np.abs(base_w + ww) + TINY[gt])
        _near(_np(GB)[0], base_b + wb, chain * np.abs(DY).sum(0) + 2 * U * np.abs(base_b) + HALF[gt] * np.abs(base_b + wb) + TINY[gt])
        # dx in the place of dy: the same bits; without the sums, and the sums alone
        keep, kw, kb = dx.clone(), GW.clone(), GB.clone()
        dfx.layer_norm_grad(rows, dim, kinds[dt], xg.ptr(), yg.ptr(), yg.ptr(), weight=wg.ptr(), param_dtype=kinds[pt], x_stride=dim + more, dy_stride=dim + more,
                            dx_stride=dim + more, eps=EPS)
        assert bool((dy == keep).all())
        if not onto:
            dy.copy_(_dev(DY))
            GW.fill_(9.0)
            dfx.layer_norm_grad(rows, dim, kinds[dt], xg.ptr(), yg.ptr(), 0, weight=wg.ptr(), grad_weight=gw.ptr(), param_dtype=kinds[pt], grad_dtype=kinds[gt], x_stride=dim + more,
                                dy_stride=dim + more, eps=EPS, workspace=ws, workspace_bytes=nbytes)
            assert bool((GW == kw).all()) and bool((GB == kb).all())


@pytest.mark.parametrize("dt", TYPES)
def test_layer_norm_values(dt):
    """Constant rows are the bias; a row with an infinity or NaN is NaN and no other is; a mean far from 0 costs no more than its size says."""
    torch, _ = _t()
    dfx, kinds = _dfx()
    rows, dim = 6, 300
    xg, x = _rows(rows, dim, dt, seed=13)
    x[0] = 2.5
    x[1, 7] = math.inf
    x[2, 299] = math.nan
    x[3] = 0.0
    x[4] += 1000.0
    yg, y = _rows(rows, dim, dt, fill=7.0)
    dfx.layer_norm(rows, dim, kinds[dt], xg.ptr(), yg.ptr(), eps=EPS)
    assert bool((y[0] == 0).all()) and bool((y[3] == 0).all()) and bool(y[1].isnan().all()) and bool(y[2].isnan().all())
    X = _np(x)[4:]
    h, r, eh = _norm_tol(X, None, EPS)
    _near(_np(y)[4:], h, eh + 3 * U * np.abs(h) + HALF[dt] * np.abs(h) + TINY[dt])


def test_more_rows_than_a_launch_has():
    """Short rows, so many that they take several launches; and a table of as many, cleared."""
    torch, _ = _t()
    dfx, kinds = _dfx()
    rows, dim, vocab = (1 << 22) + 5, 8, 1000
    gen = torch.Generator("cuda").manual_seed(17)
    tokens = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda")
    table = torch.randn(vocab, dim, generator=gen, device="cuda").bfloat16()
    og, out = _rows(rows, dim, "bf16", fill=7.0)
    dfx.embed(rows, dim, vocab, kinds["bf16"], tokens.data_ptr(), table.data_ptr(), og.ptr(), scale=0.5)
    og.check()
    assert torch.equal(out, torch.where(tokens[:, None] >= 0, (table * 0.5)[tokens.clamp(min=0)], torch.zeros((), dtype=torch.bfloat16, device="cuda")))
    yg, y = _rows(rows, dim, "bf16", fill=7.0)
    dfx.layer_norm(rows, dim, kinds["bf16"], og.ptr(), yg.ptr(), eps=EPS)
    yg.check()
    one, two = _rows(6, dim, "bf16", fill=7.0)
    last = out[-6:].contiguous()
    dfx.layer_norm(6, dim, kinds["bf16"], last.data_ptr(), one.ptr(), eps=EPS)
    assert torch.equal(y[-6:], two)
    for n, vocab in ((600, (1 << 24) + 3), (600, 1 << 18), (20, (1 << 22) + 9)):
        t = torch.arange(n, device="cuda") * 7 + vocab - 7 * n
        g = torch.ones(n, 1, dtype=torch.float16, device="cuda")
        Gg, G = _rows(vocab, 1, "f16", fill=7.0)
        nbytes = dfx.embed_grad_workspace(n, 1, vocab, kinds["f16"])
        work = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        dfx.embed_grad(n, 1, vocab, kinds["f16"], t.data_ptr(), g.data_ptr(), Gg.ptr(), workspace=work.data_ptr(), workspace_bytes=nbytes)
        Gg.check()
        assert bool((G[t, 0] == 1).all()) and int((G != 0).sum()) == n


# ------------------------------------------------------------------------------------------------------------ the vocabulary's loss
class Vocab:
    """A call's memory, and the check of everything that it gives."""

    def __init__(self, rows, dim, vocab, dt, gt=None, more=0, off=0, seed=0, weights="some", c=1.0, scale=True):
        torch, td = _t()
        self.dfx, self.kinds = _dfx()
        self.rows, self.dim, self.vocab, self.dt, self.gt, self.c = rows, dim, vocab, dt, gt or dt, c
        self.stride = dim + more
        self.xg, self.x = _rows(rows, dim, dt, self.stride, off, seed=seed + 1)
        self.wg, self.w = _rows(vocab, dim, dt, self.stride, off, seed=seed + 2, std=2.5 / math.sqrt(dim))
        self.t = _tokens(rows, vocab, seed + 3, 0.15) if vocab else np.full(rows, 0, np.int64)
        if rows > 4:
            self.t[3] = vocab
        rng = np.random.RandomState(seed + 4)
        self.rw = None if weights is None else np.where(rng.rand(rows) < 0.2, 0.0, rng.choice([1.0, 0.25, -0.5, 3.0], rows)).astype(np.float32)
        if weights is not None and rows:     # what is masked is not looked at
            self.x[_dev(np.nonzero(self.rw == 0)[0])] = math.nan
        self.scale = np.float32(0.37) if scale else None
        self.lg, self.og = Guarded(rows, "f32"), Guarded(rows, "f32")
        self.sg = Guarded(2, "f32")
        self.hg, self.gh = _rows(rows, dim, dt, self.stride, off, fill=7.0)
        self.vg, self.gw = _rows(vocab, dim, self.gt, self.stride, off, seed=seed + 5)
        self.old = _np(self.gw)

    def run(self, grad=True, onto=False, piece=0, hidden=True, weight=True, keep=None):
        dfx = self.dfx
        nbytes = dfx.vocab_loss_workspace(self.rows, self.dim, self.vocab, self.kinds[self.dt], grad, piece)
        mem, ws, end = keep or _work(nbytes)
        tok = self.tok = _dev(self.t)
        rw = self.rwd = None if self.rw is None else _dev(self.rw)
        sc = self.scd = None if self.scale is None else _dev(np.array([self.scale]))
        dfx.vocab_loss(self.rows, self.dim, self.vocab, self.kinds[self.dt], self.xg.ptr(), self.wg.ptr(), tok.data_ptr(), row_weight=0 if rw is None else rw.data_ptr(),
                       scale=0 if sc is None else sc.data_ptr(), logp=self.lg.ptr(), loss=self.og.ptr(), sums=self.sg.ptr(), grad_hidden=self.hg.ptr() if grad and hidden else 0,
                       grad_weight=self.vg.ptr() if grad and weight else 0, grad_dtype=self.kinds[self.gt], accumulate=onto, hidden_stride=self.stride, weight_stride=self.stride,
                       grad_hidden_stride=self.stride, grad_weight_stride=self.stride, inv_temperature=self.c, piece=piece, workspace=ws, workspace_bytes=nbytes)
        for g in (self.lg, self.og, self.sg, self.hg, self.vg):
            g.check()
        assert bool((mem[end:] == 0xA5).all())

    def check(self, grad=True, onto=False, hidden=True, weight=True):
        x, w, c, dt = _np(self.x), _np(self.w), self.c, self.dt
        scale = 1.0 if self.scale is None else float(self.scale)
        on = np.array([0 <= t < self.vocab and (self.rw is None or self.rw[i] != 0) for i, t in enumerate(self.t)], bool)
        x = np.where(on[:, None], x, 0.0)
        r = en.vocab_loss(x, w, self.t, self.rw, scale, c)
        rw = np.ones(self.rows) if self.rw is None else np.abs(self.rw.astype(np.float64))
        out = 2.0 ** -22 if dt == "f32" else 0.0
        ez = (2 * (self.dim * (6 if dt == "f32" else 1) + 4) * U + out) * (np.abs(x) @ np.abs(w).T)       # errors of the logits
        z = c * (x @ w.T)
        far = np.abs(z - z.max(1, keepdims=True)) if self.vocab else z
        es = c * (r["p"] * ez).sum(1) + (48 + self.vocab / 256 + 3 * math.log(max(2, self.vocab)) + 8) * U      # of the sum and its logarithm
        at = np.where(on, self.t, 0)
        tol = np.where(on, c * ez[np.arange(self.rows), at] + es, 0.0) if self.vocab else np.zeros(self.rows)
        tol = tol + 2 * U * np.abs(r["logp"])
        _near(self.lg.host(), r["logp"], tol, "logp")
        _near(self.og.host(), r["loss"], rw * tol + 2 * U * np.abs(r["loss"]), "loss")
        _near(self.sg.host(), r["sums"], np.array([(rw * on * tol).sum() + 2 * U * np.abs(r["loss"]).sum(), 2 * U * (rw * on).sum()]), "sums")
        if not grad:
            return
        k = scale * c
        half = HALF[dt]
        ep = r["p"] * (c * ez + es[:, None] + (8 + 3 * far) * U)                # of p
        edz = np.abs(k) * rw[:, None] * ep + half * np.abs(r["dz"]) + 6 * U * np.abs(k) * rw[:, None] * (r["p"] + (r["dz"] != 0))
        edz = (edz + np.abs(k) * rw.max(initial=0) * 2.0 ** -41) * on[:, None]
        adz = np.abs(r["dz"]) + edz
        if hidden:
            want = r["grad_hidden"]
            tol = edz @ np.abs(w) + (2 * (self.vocab * (6 if dt == "f32" else 1) + 300) * U + out) * (adz @ np.abs(w))
            _near(_np(self.gh), want, tol + (half + 4 * U) * np.abs(want) + TINY[dt], "grad_hidden")
        if weight:
            want = r["grad_weight"] + (self.old if onto else 0.0)
            tol = edz.T @ np.abs(x) + (2 * (self.rows * (6 if dt == "f32" else 1) + 300) * U + out) * (adz.T @ np.abs(x)) + 2 * U * np.abs(self.old) * onto
            _near(_np(self.gw), want, tol + (HALF[self.gt] + 4 * U) * np.abs(want) + TINY[self.gt], "grad_weight")


VOCAB = [(1, 1, 1), (1, 64, 257), (2, 7, 5), (48, 128, 1000), (64, 64, 256), (65, 192, 513), (130, 100, 777), (200, 256, 1025), (257, 65, 300), (300, 320, 3000), (600, 64, 512),
         (1, 77, 300), (20, 1001, 700), (33, 66, 1000), (100, 130, 515), (128, 200, 900), (129, 64, 400), (5, 63, 300), (3, 64, 65600), (70, 71, 66001),
         (16, 1024, 300), (17, 1025, 300), (9, 2048, 520), (31, 2040, 260), (3, 2047, 300), (12, 4095, 270), (16, 4096, 260), (33, 4096, 260), (1000, 96, 600), (1025, 70, 300),
         (2, 1100, 9000), (20, 1100, 9000), (7, 2050, 9000), (1030, 66, 16500), (650, 200, 2400), (4000, 98, 700)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,dim,vocab", VOCAB)
def test_vocab_loss(rows, dim, vocab, dt):
    for more, off, c in ((0, 0, 1.0), (3, 1, 0.7)):
        v = Vocab(rows, dim, vocab, dt, more=more, off=off, c=c)
        v.run()
        v.check()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,dim,vocab", [(1, 64, 1000), (40, 96, 700), (200, 128, 1500)])
def test_vocab_loss_forward_alone(rows, dim, vocab, dt):
    v = Vocab(rows, dim, vocab, dt, seed=20, weights=None, scale=False)
    v.run(grad=False)
    v.check(grad=False)
    torch, _ = _t()
    assert bool((v.gh == 7.0).all())


@pytest.mark.parametrize("dt,gt", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("piece", [256, 512, 1 << 20])
def test_vocab_loss_in_pieces_and_onto(dt, gt, piece):
    """Pieces of any length, onto what the gradient holds; either gradient alone."""
    for rows, dim, vocab in ((70, 128, 1300), (300, 72, 1024)):
        v = Vocab(rows, dim, vocab, dt, gt, seed=30)
        v.run(onto=True, piece=piece)
        v.check(onto=True)
        for hidden, weight in ((True, False), (False, True)):
            v = Vocab(rows, dim, vocab, dt, gt, seed=31)
            v.run(piece=piece, hidden=hidden, weight=weight)
            v.check(hidden=hidden, weight=weight)


@pytest.mark.parametrize("dt", TYPES)
def test_vocab_loss_with_nothing_to_learn(dt):
    """No row counts, or there are no rows, or no vocabulary: zeros, or the gradient as it was."""
    torch, _ = _t()
    for rows, vocab, t in ((50, 300, -1), (0, 300, 0), (50, 0, 3), (300, 300, 300)):
        for onto in (False, True):
            v = Vocab(rows, 64, vocab, dt, seed=40, weights=None)
            v.t = np.full(rows, t, np.int64)
            v.x.fill_(math.nan)
            v.run(onto=onto)
            assert not v.lg.host().any() and not v.og.host().any() and not v.sg.host().any() and not _np(v.gh).any()
            assert np.array_equal(_np(v.gw), v.old if onto else 0 * v.old)


@pytest.mark.parametrize("dt", TYPES)
def test_vocab_loss_of_extreme_logits(dt):
    """Logits far apart, a NaN in one row, an infinite one in another: the other rows' losses stay right."""
    v = Vocab(40, 64, 600, dt, seed=50, weights=None)
    v.x[5] *= 40.0
    v.x[6] = 0.0
    v.run(grad=False)
    v.check(grad=False)
    v.x[7, 3] = math.nan
    v.t[7] = 1
    v.t[8] = 2
    before = v.lg.host()
    v.run()
    after = v.lg.host()
    assert math.isnan(after[7]) and np.array_equal(np.delete(before, [7, 8]), np.delete(after, [7, 8]))
    got = _np(v.gh)
    assert np.isnan(got[7]).all() and np.isfinite(np.delete(got, 7, 0)).all() and np.isnan(_np(v.gw)).any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_vocab_loss_gives_the_same_bits(dt):
    """Twice on the same memory, in a workspace of other contents, and for a workspace of more rows."""
    torch, _ = _t()
    v = Vocab(300, 128, 2000, dt, seed=60)
    v.run()
    first = [t.clone() for t in (v.lg.t, v.og.t, v.sg.t, v.gh, v.gw)]
    nbytes = v.dfx.vocab_loss_workspace(300, 128, 2000, v.kinds[dt], True)
    mem, ws, end = _work(nbytes)
    mem[:end].copy_(torch.randint(0, 256, (end,), dtype=torch.uint8, device="cuda"))
    v.run(keep=(mem, ws, end))
    for a, b in zip(first, (v.lg.t, v.og.t, v.sg.t, v.gh, v.gw)):
        assert torch.equal(a, b)


def test_vocab_loss_against_differences():
    """The gradient in a direction is the loss's difference along it (32-bit inputs; a step of 2^-5 leaves 2^-10 of its third derivative's share)."""
    torch, _ = _t()
    v = Vocab(20, 64, 400, "f32", seed=70, weights="some", scale=False)
    on = np.nonzero((v.rw != 0) & (v.t >= 0) & (v.t < 400))[0]
    v.run()
    gh, gw = _np(v.gh), _np(v.gw)
    gen = torch.Generator("cuda").manual_seed(3)
    dx = torch.zeros_like(v.x)
    dx[_dev(on)] = torch.randn(len(on), 64, generator=gen, device="cuda") * 0.1
    dw = torch.randn(400, 64, generator=gen, device="cuda") * 0.01
    x0, w0, h = v.x.clone(), v.w.clone(), 2.0 ** -5
    sums = []
    for s in (h, -h):
        v.x.copy_(x0 + s * dx)
        v.w.copy_(w0 + s * dw)
        v.run(grad=False)
        sums.append(v.og.host().sum())
    want = (gh * _np(dx)).sum() + (gw * _np(dw)).sum()
    assert abs((sums[0] - sums[1]) / (2 * h) - want) < 3e-3 * (abs(want) + 0.1)


@pytest.mark.parametrize("rows,dim,vocab,piece", [(1, 64, 1000, 0), (20, 2048, 9000, 0), (40, 96, 20000, 0), (300, 128, 2000, 0), (1030, 66, 16500, 0), (300, 1600, 700, 0),
                                                  (40, 96, 20000, 512), (3, 1024, 3000, 768), (300, 128, 2000, 256), (300, 77, 2000, 768)])
@pytest.mark.parametrize("dt", TYPES)
def test_vocab_loss_is_the_same_with_gradients(rows, dim, vocab, piece, dt):
    """Scoring and training see the same numbers: logp, loss and sums with gradients, with either and without; each gradient with the other and alone."""
    torch, _ = _t()
    v = Vocab(rows, dim, vocab, dt, seed=80)
    v.run(piece=piece)
    first = [t.clone() for t in (v.lg.t, v.og.t, v.sg.t, v.gh, v.gw)]
    for grad, hidden, weight in ((False, False, False), (True, True, False), (True, False, True)):
        v.run(grad=grad, hidden=hidden, weight=weight, piece=piece)
        for a, b in zip(first, (v.lg.t, v.og.t, v.sg.t, v.gh, v.gw)):
            assert torch.equal(a, b)
