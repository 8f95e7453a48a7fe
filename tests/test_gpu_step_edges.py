"""Values and layouts at the edge of what the training step's operators are asked for: log-probabilities of -infinity, penalties far from 0,
small rates, numbers beyond 32 bits, memory that is named twice, calls that overlap, rows where they begin to be split, a context in front.
Helpers and tolerances are those of test_gpu_step.py, whose docstring derives them."""
import math

import numpy as np
import pytest

from oracle import step as st
from tests import test_gpu_step as ts

pytestmark = pytest.mark.gpu

U = ts.U


def _banned(rows, vocab, dt, big):
    """Rows whose penalty is beyond 32 bits: the policy bans the token, the reference does, d is 1000, the token's logit is the type's lowest, that and the
    reference bans it too, d is `big`; the others are ordinary."""
    import torch
    z, _, t, cols = ts._loss_case(rows, vocab, dt, 17)
    x = z.t.view(rows, vocab)
    lowest = float(torch.finfo(x.dtype).min)
    x[0, int(t[0])] = -math.inf
    x[3, int(t[3])] = lowest
    x[4, int(t[4])] = lowest
    zh = z.host().reshape(rows, vocab)
    lp = st.policy_loss(zh, t.numpy())["logp"]
    old, ref = lp - 0.1, lp + 0.1
    for k in (0, 3, 4):
        old[k] = ref[k] = -3.0
    ref[1] = ref[4] = -math.inf
    ref[2], ref[5] = lp[2] + 1000.0, lp[5] + big
    cols.update(old=old.astype(np.float32), ref=ref.astype(np.float32), weight=np.ones(rows, np.float32))
    return z, zh, t, cols


WAYS = [(12, 100), (12, 30011), (70, 30011)]        # a row to a workgroup; split; too many rows to split


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", WAYS)
def test_a_penalty_that_is_only_watched(rows, vocab, dt):
    """kl_coef = 0 with reference log-probabilities: whatever the penalty comes to, loss and gradient are those without a reference."""
    z, zh, t, cols = _banned(rows, vocab, dt, 90.0)
    out = ts._run_loss(z, t, cols, rows, vocab, dt, kl_coef=0.0)
    assert float(out["sums"].t[2]) == math.inf
    out["sums"].t[2] = 0.0
    del cols["ref"]
    want = ts._check_loss(out, zh, t, cols, rows, vocab, dt, kl_coef=0.0)
    assert np.isfinite(want["loss"]).all() and np.isfinite(want["grad"]).all() and want["logp"][0] == -math.inf
    fwd = ts._run_loss(z, t, dict(cols, ref=np.full(rows, -np.inf, np.float32)), rows, vocab, dt, grad=False, kl_coef=0.0)
    fwd["sums"].t[2] = 0.0
    ts._check_loss(fwd, zh, t, cols, rows, vocab, dt, grad=False, kl_coef=0.0)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", WAYS)
def test_a_penalty_that_is_infinite(rows, vocab, dt):
    """The loss is infinite; the gradient of a row whose token the reference bans is finite, exp(d) - 1 being -1 there, and no other row is touched."""
    kl = 0.1
    z, zh, t, cols = _banned(rows, vocab, dt, 0.1)
    out = ts._run_loss(z, t, cols, rows, vocab, dt, kl_coef=kl)
    want = st.policy_loss(zh, t.numpy(), cols["old"], cols["ref"], cols["adv"], cols["weight"], float(np.float32(0.37)), kl_coef=kl)
    loss = out["loss"].host()
    assert np.all(loss[:5] == math.inf) and float(out["sums"].t[0]) == math.inf and float(out["sums"].t[2]) == math.inf
    assert float(out["logp"].t[0]) == -math.inf
    got, logv = out["grad"].host().reshape(rows, vocab), math.log(vocab)
    e_s = (vocab / 256 + 68 + 3 * logv) * U
    dl = e_s + 4 * U
    for k in [1, 4] + list(range(5, rows)):
        lp = want["logp"][k]
        per = abs(float(cols["adv"][k])) * math.exp(lp - float(cols["old"][k])) + kl * math.exp(float(cols["ref"][k]) - lp)
        if k >= 5:
            ts._near(loss[k], want["loss"][k], 2 * (per + kl) * dl + 4 * U * abs(want["loss"][k]), "loss")
        far = zh[k].max() - zh[k]
        p = np.exp(-far)
        p /= p.sum()
        coef, g = 0.37 * (per + kl), want["grad"][k]
        assert np.isfinite(g).all()
        tol = coef * p * (3 * U * far + 8 * U + 2 * e_s + dl) + np.abs(g) * (2 * dl + 4 * U + ts.HALF[dt]) + ts.TINY[dt]
        tol[int(t[k])] += 3 * coef * dl
        ts._near(got[k], g, tol, "grad of row %d" % k)


@pytest.mark.parametrize("vocab", [64, 32768])
def test_the_penalty_and_its_slope_far_from_zero(vocab):
    """Rows of equal logits (probability, sum and log-probability are exact), an advantage of 0: loss and gradient are the penalty and its slope times
    powers of two.  exp(d) is off by the rounding of d / log 2, |d| u, and its own 2 u; the slope exp(d) - 1 is rounded once, the penalty twice (and
    its series' 4 u below 1/2), the gradient of an element beside the target once more."""
    d = np.array([-80.2, -33.3, -16.7, -8.1, -4.3, -1.7, -0.6, -0.4, -0.01, 0.01, 0.3, 0.7, 1.9, 5.2, 21.7, 60.3])
    rows = len(d)
    z = ts.Guarded(rows * vocab, "f32")
    z.t.fill_(1.5)
    lp = -math.log(vocab)
    ref = (lp + d).astype(np.float32)
    d = ref.astype(np.float64) - lp
    import torch
    t = torch.arange(rows) % vocab
    cols = {"ref": ref, "adv": np.zeros(rows, np.float32), "weight": np.full(rows, 0.5, np.float32)}
    out = ts._run_loss(z, t, cols, rows, vocab, "f32", kl_coef=0.25)
    e, kl, grows = np.exp(d), np.expm1(d) - d, np.expm1(d)
    ts._near(out["loss"].host(), 0.125 * kl, 0.125 * (e * (np.abs(d) + 3) * (np.abs(d) > 0.4) + 8 * kl) * U, "loss")
    scale = float(np.float32(0.37))
    got = out["grad"].host().reshape(rows, vocab)[np.arange(rows), (np.arange(rows) + 1) % vocab]
    # -g p, g = -0.125 scale grows
    want = 0.125 * scale * grows / vocab
    ts._near(got, want, np.abs(want) * 3 * U + 0.125 * scale / vocab * e * (np.abs(d) + 3) * U * (np.abs(d) > 0.4) + ts.TINY["f32"], "grad")


@pytest.mark.parametrize("on_device", [False, True])
@pytest.mark.parametrize("lr,decay", [(1e-6, 0.01), (1e-6, 0.1), (1e-5, 0.01)])
def test_adamw_decays_at_small_rates(lr, decay, on_device):
    """1000 steps of noise at rates of fine-tuning.  A parameter's rounding is 2^-25 a step at most, as likely up as down: the mean over 16384 parameters is off by
    2^-25 sqrt(1000 / 16384) < 1e-8, where the decay moves it by 7.5e-6 at least.  2 % of that are allowed."""
    import torch
    dfx, _ = ts._dfx()
    n, steps = 16384, 1000
    gen = torch.Generator("cuda").manual_seed(7)
    p = ts.Guarded(n, "f32")
    p.t.uniform_(0.5, 1.0, generator=gen)
    g, m, v = (ts.Guarded(n, "f32", fill=np.zeros(n)) for _ in range(3))
    lists = [dfx.TensorList([(b.ptr(), n, dfx.F32)]) for b in (p, g, m, v)]
    rate = torch.full((), lr, device="cuda")
    want = [p.host(), m.host(), v.host()]
    for step in range(1, steps + 1):
        g.t.normal_(generator=gen)
        cfg = dfx.AdamWConfig(lr=7.0, step=step, weight_decay=decay, lr_dev=rate.data_ptr()) if on_device else dfx.AdamWConfig(lr=lr, step=step, weight_decay=decay)
        dfx.adamw(*lists, cfg, stream=torch.cuda.current_stream().cuda_stream)
        want = st.adamw(want[0], g.host(), want[1], want[2], step, lr, 0.9, 0.999, 1e-8, decay)
    asked = lr * decay * steps * 0.75
    assert asked > 7e-6
    assert abs(float((p.host() - want[0]).mean())) < 0.02 * asked


def test_adamw_of_no_step_on_the_device():
    """A counter that has not been counted up yet: there is no update 0, and nothing is written."""
    import torch
    dfx, _ = ts._dfx()
    lists, bufs = ts._adam_state(ts.LISTS["odd"], 51, "bf16", "bf16")
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = [b.raw.clone() for bb in bufs for b in bb]
    cfg = dfx.AdamWConfig(step_dev=step.data_ptr())
    dfx.adamw(*lists[:4], cfg, copies=lists[4])
    assert all(bool((a == b.raw).all()) for a, b in zip(before, [b for bb in bufs for b in bb]))
    step.add_(1)
    host = [[b.host() for b in bb] for bb in bufs[:4]]
    dfx.adamw(*lists[:4], cfg, copies=lists[4])
    ts._check_adam(host, bufs, "bf16", 1, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0)


def test_results_in_the_space_between_rows():
    """What is written may lie between rows of logits, where nothing is read."""
    import torch
    dfx, _ = ts._dfx()
    rows, vocab, stride = 5, 100, 120
    z, zh, t, cols = ts._loss_case(rows, vocab, "f32", 9, stride=stride)
    want = st.policy_loss(zh, t.numpy(), cols["old"], None, cols["adv"], cols["weight"])
    dev = {k: torch.from_numpy(v).cuda() for k, v in cols.items()}
    tt, ws = t.cuda(), torch.empty(dfx.policy_loss_workspace(rows, vocab, dfx.F32), dtype=torch.uint8, device="cuda")
    x = z.t.view(rows, stride)
    x[:, vocab:] = 7.0
    at = [x[k, vocab:].data_ptr() for k in range(rows)]
    dfx.policy_loss(rows, vocab, dfx.F32, z.ptr(), tt.data_ptr(), old_logp=dev["old"].data_ptr(), advantage=dev["adv"].data_ptr(), weight=dev["weight"].data_ptr(), logp=at[0],
                    loss=at[0] + 4 * rows, sums=at[3], logits_stride=stride, workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    e = (vocab / 256 + 68 + 3 * math.log(vocab)) * U + 4 * U
    size = 4 * np.abs(cols["adv"])
    ts._near(x[0, vocab:vocab + rows].double().cpu().numpy(), want["logp"], e + 4 * U * np.abs(want["logp"]))
    ts._near(x[0, vocab + rows:vocab + 2 * rows].double().cpu().numpy(), want["loss"], size * e + 4 * U * np.abs(want["loss"]))
    ts._near(x[3, vocab:vocab + 5].double().cpu().numpy(), want["sums"], size.sum() * e + 2 * U * np.abs(want["sums"]))
    assert bool((x[1, vocab:] == 7.0).all()) and bool((x[3, vocab + 5:] == 7.0).all()) and bool((x[0, vocab + 2 * rows:] == 7.0).all())
    for k in (x[0, vocab - 1:].data_ptr(), x[1].data_ptr() - 4 * rows + 4):
        with pytest.raises(dfx.DfxError):
            dfx.policy_loss(rows, vocab, dfx.F32, z.ptr(), tt.data_ptr(), logp=k, logits_stride=stride)
    z.check()


@pytest.mark.parametrize("max_norm", [1e300, math.inf])
def test_a_bound_beyond_32_bits(max_norm):
    """The largest norm that there may be is one: finite norms are below it, and a norm of infinity still makes finite gradients 0."""
    dfx, _ = ts._dfx()
    lst, bufs = ts._list(ts.LISTS["odd"], 5)
    src = [b.host() for b in bufs]
    norm = ts._scalar(3e38)
    dfx.grad_clip(lst, norm.ptr(), max_norm, scale=0.5)
    assert all(np.array_equal(b.host(), b.t.new_tensor(0.5 * x).double().cpu().numpy()) for x, b in zip(src, bufs))
    norm.t.fill_(math.inf)
    dfx.grad_clip(lst, norm.ptr(), max_norm)
    assert not any(b.host().any() for b in bufs)


def test_a_clip_beyond_32_bits():
    """A ratio that overflows is clipped by any bound, so that an advantage of 0 gives 0 there too."""
    rows, vocab = 4, 50
    z, zh, t, cols = ts._loss_case(rows, vocab, "f32", 3)
    cols.update(old=np.full(rows, -800.0, np.float32), adv=np.zeros(rows, np.float32), weight=np.ones(rows, np.float32))
    out = ts._run_loss(z, t, cols, rows, vocab, "f32", clip_high=1e300)
    assert out["loss"].t.tolist() == [0.0] * rows and not bool(out["grad"].t.any()) and float(out["sums"].t[3]) == rows


def test_numbers_that_32_bits_do_not_hold_are_refused():
    dfx, _ = ts._dfx()
    a, b, c, d = (ts._list([(5, "f32"), (6, "f32")], k)[0] for k in range(4))
    n = ts._scalar(2.0)
    for scale in (1e39, -1e300, 1e-39, 1e-60, math.nan):
        for call in (dfx.grad_clip, dfx.clip_grad_norm):
            with pytest.raises(dfx.DfxError) as e:
                call(a, n.ptr(), 1.0, scale=scale)
            assert e.value.status == dfx.ERR_INVALID_ARG
    for kw in (dict(grad_scale=1e39), dict(grad_scale=1e-40), dict(lr=1e39), dict(lr=-1e200), dict(weight_decay=1e39), dict(eps=1e39), dict(eps=1e-40)):
        with pytest.raises(dfx.DfxError) as e:
            dfx.adamw(a, b, c, d, dfx.AdamWConfig(**kw))
        assert e.value.status == dfx.ERR_INVALID_ARG
    dfx.grad_norm(a, n.ptr(), scale=1e-60)              # (a norm's scale is taken in 64 bits)
    assert float(n.t) == 0.0
    dfx.grad_clip(a, n.ptr(), 1.0, scale=0.0)
    dfx.adamw(a, b, c, d, dfx.AdamWConfig(lr=1e-60, eps=1e-37))


def test_lists_that_would_be_written_over_are_refused():
    """A tensor that is written lies on no other tensor of its list and on none of the source but itself; what is only read may lie anywhere."""
    import torch
    dfx, _ = ts._dfx()
    x, y, m, v = (ts.Guarded(40, "f32") for _ in range(4))
    for k, b in enumerate((x, y, m, v)):
        b.t.copy_(torch.arange(40) + k)
    n = ts._scalar(2.0)

    def lst(*at, kind=dfx.F32, of=x, eb=4):
        return dfx.TensorList([(of.ptr() + eb * a, c, kind) for a, c in at])

    def refused(f, *args, **kw):
        with pytest.raises(dfx.DfxError) as e:
            f(*args, **kw)
        assert e.value.status == dfx.ERR_INVALID_ARG

    src = lst((0, 8), (8, 8), (20, 8))
    bad = [lst((28, 8), (0, 8), (8, 8)), lst((8, 8), (0, 8), (20, 8)), lst((0, 8), (8, 8), (13, 8)), lst((0, 8), (27, 8), (28, 8)), lst((0, 8), (1, 8), (20, 8)),
           lst((28, 8), (28, 8), (20, 8)), lst((30, 8), (16, 8), (12, 8))]
    # widened in the bucket itself: the second result lies on the third source
    half = dfx.TensorList([(x.ptr() + 2 * a, 8, dfx.BF16) for a in (0, 8, 40)])
    wide = dfx.TensorList([(y.ptr(), 8, dfx.F32), (x.ptr() + 68, 8, dfx.F32), (y.ptr() + 40, 8, dfx.F32)])
    twice = lst((0, 8), (30, 8), (0, 8))
    for call in (dfx.grad_clip, dfx.clip_grad_norm):
        for out in bad:
            refused(call, src, n.ptr(), 1.0, out=out)
        refused(call, half, n.ptr(), 1.0, out=wide)
        refused(call, twice, n.ptr(), 1.0)
    one, g = lst((0, 8), (8, 8), (16, 8), of=y), lst((0, 8), (8, 8), (16, 8))
    good = [lst((0, 8), (8, 8), (16, 8), of=b) for b in (y, m, v)]
    over = lst((0, 8), (7, 8), (16, 8), of=y)
    refused(dfx.adamw, over, g, good[1], good[2], dfx.AdamWConfig())
    refused(dfx.adamw, good[0], g, lst((0, 8), (0, 8), (16, 8), of=m), good[2], dfx.AdamWConfig())
    refused(dfx.adamw, good[0], g, good[1], lst((0, 8), (9, 8), (16, 8), of=v), dfx.AdamWConfig())
    refused(dfx.adamw, good[0], g, good[1], good[2], dfx.AdamWConfig(), copies=lst((20, 8), (28, 8), (35, 8)))
    assert all(bool((b.t == torch.arange(40, device="cuda") + k).all()) for k, b in enumerate((x, y, m, v)))
    # taken: read twice, written once; the same tensors under another list, in part and between the others; with an empty tensor on them
    want = x.t.clone()
    dfx.grad_clip(twice, n.ptr(), 1.0, out=lst((0, 8), (8, 8), (16, 8), of=y), scale=2.0)
    for a, b in ((0, 0), (30, 8), (0, 16)):
        assert torch.allclose(y.t[b:b + 8], want[a:a + 8], rtol=1e-6)
    dfx.grad_clip(lst((0, 8), (8, 0), (20, 8)), n.ptr(), 1.0, out=lst((0, 8), (4, 0), (30, 8)), scale=0.5)
    assert torch.allclose(x.t[:8], 0.25 * want[:8], rtol=1e-6) and torch.allclose(x.t[30:38], 0.25 * want[20:28], rtol=1e-6)
    assert bool((x.t[8:30] == want[8:30]).all()) and bool((x.t[38:] == want[38:]).all())
    for b in (x, y, m, v):
        b.check()


@pytest.mark.parametrize("chunks", [2, 31, 33, 100, 544])
def test_norms_behind_calls_that_overlapped(chunks):
    """Calls on one list from two streams at once leave norms that mean nothing, and the list as good as new."""
    import torch
    dfx, _ = ts._dfx()
    n = chunks * 8192 - 3
    g = ts.Guarded(n, "f32")
    g.t.fill_(0.25)
    lst = dfx.TensorList([(g.ptr(), n, dfx.F32)])
    outs = [ts._scalar() for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = 0.25 * math.sqrt(n)
    torch.cuda.synchronize()
    for _ in range(4):
        for _ in range(50):
            for s, o in zip(streams, outs):
                dfx.grad_norm(lst, o.ptr(), stream=s.cuda_stream)
        torch.cuda.synchronize()
        for _ in range(2):
            outs[0].t.fill_(-1.0)
            dfx.grad_norm(lst, outs[0].ptr())
            torch.cuda.synchronize()
            assert abs(float(outs[0].t) - want) <= 2 * U * want
    for o in outs:
        o.check()


KW = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [1, 64, 65])
@pytest.mark.parametrize("vocab", [19999, 20000])
def test_loss_where_rows_with_gradient_begin_to_be_split(rows, vocab, dt):
    z, zh, t, cols = ts._loss_case(rows, vocab, dt, vocab + rows)
    cols["old"][0] = st.policy_loss(zh[:1], t[:1].numpy())["logp"][0] + 0.05
    out = ts._run_loss(z, t, cols, rows, vocab, dt, goff=1, **KW)
    ts._check_loss(out, zh, t, cols, rows, vocab, dt, **KW)
    out = ts._run_loss(z, t, cols, rows, vocab, dt, in_place=True, **KW)
    ts._check_loss(out, zh, t, cols, rows, vocab, dt, **KW)


@pytest.mark.parametrize("dt,vocab", [("f32", 60001), ("bf16", 131071), ("f16", 106500)])
def test_gradient_in_the_place_of_logits_that_are_read_again(dt, vocab):
    """Rows that neither are split nor fit registers and LDS: what is left of a row is read a second time, with gradients already written around it."""
    rows, stride = 66, vocab + 3
    z, zh, t, cols = ts._loss_case(rows, vocab, dt, 23, stride=stride, off=1)
    z.t.view(rows, stride)[:, vocab:] = 7.0
    out = ts._run_loss(z, t, cols, rows, vocab, dt, in_place=True, stride=stride, gstride=stride, **KW)
    ts._check_loss(out, zh, t, cols, rows, vocab, dt, gstride=stride, **KW)
    assert bool((z.t.view(rows, stride)[:, vocab:] == 7.0).all())


def test_the_update_behind_a_contexts_all_reduce():
    """Three buckets all-reduced over eight virtual ranks by a context, then norm and update on what they have become, with the daemon still there; three
    steps, the next gradients written behind it each time."""
    import torch
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import harness as gh
    R, sizes, lr = 8, (70001, 8, 300000), 0.01
    gen = torch.Generator("cuda").manual_seed(5)
    send = [[torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in sizes] for _ in range(R)]
    recv = [[torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in sizes] for _ in range(R)]
    state = [[torch.zeros(n, device="cuda") for n in sizes] for _ in range(3)]
    for p in state[0]:
        p.normal_(generator=gen)
    copy = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in sizes]
    kind = {torch.float32: dfx.F32, torch.bfloat16: dfx.BF16}
    p, m, v, c = (dfx.TensorList([(t.data_ptr(), t.numel(), kind[t.dtype]) for t in tt]) for tt in (*state, copy))
    grads = [dfx.TensorList([(t.data_ptr(), t.numel(), dfx.BF16) for t in recv[r]]) for r in range(R)]
    norms = torch.zeros(R, device="cuda")
    want = [[t.double().cpu().numpy() for t in tt] for tt in state]
    torch.cuda.synchronize()
    ctx = dfx.Context(R, gh.make_config())
    try:
        for k, n in enumerate(sizes):
            ctx.prepare(k, dfx.ALLREDUCE, n, dfx.BF16)
        for step in range(1, 4):
            for r in range(R):
                for t in send[r]:
                    t.normal_(generator=gen)
            ready = torch.cuda.Event()
            ready.record()
            ready.synchronize()
            for r in range(R):
                for k in np.random.default_rng(r + step).permutation(len(sizes)):       # any order
                    assert ctx.submit(r, int(k), send[r][k].data_ptr(), recv[r][k].data_ptr()) == dfx.OK
            assert ctx.wait_all(20.0) == dfx.OK
            stream = torch.cuda.current_stream().cuda_stream
            for r in range(R):
                dfx.grad_norm(grads[r], norms[r].data_ptr(), scale=1.0 / R, stream=stream)
            dfx.adamw(p, grads[3], m, v, dfx.AdamWConfig(lr=lr, step=step, grad_scale=1.0 / R, max_norm=1.0), copies=c, norm=norms[3].data_ptr(), stream=stream)
            torch.cuda.synchronize()
            g = [t.double().cpu().numpy() for t in recv[0]]
            assert all(torch.equal(recv[r][k], recv[0][k]) for r in range(R) for k in range(len(sizes)))
            total = sum(send[r][0].double() for r in range(R)).cpu().numpy()
            assert np.abs(g[0] - total).max() <= R * 2.0 ** -8 * 16         # (a sum of eight normal numbers, rounded at each)
            n = st.grad_norm(g, "2", 1.0 / R)
            ts._near(norms.double().cpu().numpy(), np.full(R, n), 2 * U * n)
            f = st.clip_factor(n, 1.0, 1.0 / R)
            for k in range(len(sizes)):
                wp, wm, wv = st.adamw(want[0][k], g[k], want[1][k], want[2][k], step, lr, 0.9, 0.999, 1e-8, 0.01, f)
                got = state[0][k].double().cpu().numpy()
                dm = 8 * U * (0.9 * np.abs(want[1][k]) + 0.1 * np.abs(g[k] * f))
                move = lr / (1 - 0.9 ** step) * (np.abs(wm) * 24 * U + dm) / (np.sqrt(wv / (1 - 0.999 ** step)) + 1e-8)
                ts._near(got, wp, move + 3 * U * (np.abs(want[0][k]) + np.abs(wp)), "p")
                assert torch.equal(copy[k], state[0][k].to(torch.bfloat16))
                for q in range(3):
                    want[q][k] = state[q][k].double().cpu().numpy()
    finally:
        assert ctx.finalize() == dfx.OK
