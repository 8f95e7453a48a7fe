"""The ways that the training step's operators take by size, on both sides of where they change: workgroups' tickets of the norm, AdamW's
staged loads, rows split over workgroups, several rows to a workgroup with masked ones in between, logits read past the caches, rows that
begin at every place of 16 bytes.  Helpers and tolerances are those of test_gpu_step.py."""
import math

import numpy as np
import pytest

from oracle import step as st
from tests import test_gpu_step as ts

pytestmark = pytest.mark.gpu

CHUNK = 8192


@pytest.mark.parametrize("chunks", [1, 2, 31, 32, 33, 63, 64, 65, 511, 512, 513, 544, 1025])
def test_norm_at_every_count_of_tickets(chunks):
    """A list of so many chunks, short but for the last element of each, three times in a row with the largest magnitude in between."""
    import torch
    dfx, _ = ts._dfx()
    n = (chunks - 1) * CHUNK + 5
    g = ts.Guarded(n, "bf16", off=1)
    g.t.zero_()
    g.t[::CHUNK] = 3.0
    g.t[-1] = -4.0
    lst = dfx.TensorList([(g.ptr(), n, dfx.BF16)])
    out = ts._scalar()
    for _ in range(3):
        dfx.grad_norm(lst, out.ptr())
        want = math.sqrt(9.0 * chunks + 16.0)
        assert abs(float(out.t) - want) <= 2 * ts.U * want
        out.t.fill_(-1.0)
        dfx.grad_norm(lst, out.ptr(), dfx.NORM_INF, 0.5)
        assert float(out.t) == 2.0
    torch.cuda.synchronize()
    out.check()
    g.check()


@pytest.mark.parametrize("chunks", [639, 640, 641])
@pytest.mark.parametrize("grad_type,copy_type", [("bf16", "bf16"), ("f32", None), ("f16", "f16")])
def test_adamw_where_loads_are_staged(chunks, grad_type, copy_type):
    dfx, _ = ts._dfx()
    sizes = [((chunks - 2) * CHUNK, "f32"), (CHUNK - 3, "f32"), (7, "f32")]
    lists, bufs = ts._adam_state(sizes, chunks, grad_type, copy_type)
    before = [[b.host() for b in bb] for bb in bufs[:4]]
    n = ts._scalar(2.0)
    dfx.adamw(*lists[:4], dfx.AdamWConfig(lr=0.01, step=5, weight_decay=0.1), copies=lists[4], norm=n.ptr())
    ts._check_adam(before, bufs, copy_type, 5, 0.01, 0.9, 0.999, 1e-8, 0.1, st.clip_factor(2.0, 1.0))


KW = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", [(1, 39999), (1, 40000), (7, 40003), (64, 40001), (65, 40001), (9, 65535), (9, 65536), (5, 65541), (6, 131071)])
@pytest.mark.parametrize("grad", [True, False])
def test_loss_where_rows_are_split(rows, vocab, dt, grad):
    stride = vocab + rows % 5
    z, zh, t, cols = ts._loss_case(rows, vocab, dt, vocab, stride=stride, off=rows % 7)
    t[0] = (0, vocab - 1, vocab // 2)[vocab % 3]
    cols["old"][0] = st.policy_loss(zh[:1], t[:1].numpy())["logp"][0] + 0.05
    out = ts._run_loss(z, t, cols, rows, vocab, dt, grad=grad, stride=stride, goff=3, **KW)
    ts._check_loss(out, zh, t, cols, rows, vocab, dt, grad=grad, **KW)
    if grad:
        before = z.t.clone()
        out = ts._run_loss(z, t, cols, rows, vocab, dt, in_place=True, stride=stride, gstride=stride, **KW)
        ts._check_loss(out, zh, t, cols, rows, vocab, dt, gstride=stride, **KW)
        assert bool((z.t.view(rows, stride)[:, vocab:] == before.view(rows, stride)[:, vocab:]).all())


@pytest.mark.parametrize("vocab", [40, 1300, 70003])
def test_loss_without_a_workspace(vocab):
    import torch
    dfx, kinds = ts._dfx()
    rows = 5
    z, zh, t, cols = ts._loss_case(rows, vocab, "bf16", 2)
    want = st.policy_loss(zh, t.numpy(), weight=cols["weight"])["logp"]
    w, tt = torch.from_numpy(cols["weight"]).cuda(), t.cuda()
    lp = ts.Guarded(rows, "f32")
    for nbytes in (0, 8):
        lp.t.fill_(7.0)
        ws = torch.full((8,), 0xA5, dtype=torch.uint8, device="cuda")
        dfx.policy_loss(rows, vocab, dfx.BF16, z.ptr(), tt.data_ptr(), weight=w.data_ptr(), logp=lp.ptr(), workspace=ws.data_ptr() if nbytes else 0, workspace_bytes=nbytes)
        ts._near(lp.host(), want, (vocab / 256 + 68 + 3 * math.log(vocab)) * ts.U + 4 * ts.U * np.abs(want))
        assert bool((ws == 0xA5).all())
    lp.check()


def _by_torch(z, t, cols, scale, kl_coef=0.05, lo=0.8, hi=1.28):
    """The definition in 64 bits, by torch on the GPU (long cases): loss, gradient and sums of rows that all have a distribution."""
    import torch
    z = z.double()
    c = {k: torch.from_numpy(v).cuda().double() for k, v in cols.items()}
    on = (c["weight"] != 0) & (t >= 0) & (t < z.shape[1])
    tt = t.clamp(0, z.shape[1] - 1)
    lp = (z.gather(1, tt[:, None])[:, 0] - torch.logsumexp(z, 1)) * on
    r, d = torch.exp(lp - c["old"]), c["ref"] - lp
    a = c["adv"]
    cut = torch.where(a >= 0, r > hi, r < lo)
    pg = -a * torch.where(cut, torch.where(a >= 0, hi, lo), r)
    w = c["weight"] * on
    loss = w * (pg + kl_coef * (torch.expm1(d) - d))
    g = scale * w * (torch.where(cut, 0.0, -a * r) - kl_coef * torch.expm1(d))
    p = torch.softmax(z, 1)
    grad = -g[:, None] * p
    grad[torch.arange(len(tt), device=z.device), tt] += g
    return lp, loss, grad, torch.stack([loss.sum(), (w * pg).sum(), (w * (torch.expm1(d) - d)).sum(), (w * cut).sum(), w.sum()])


@pytest.mark.parametrize("rows,vocab,dt", [(4097, 300, "bf16"), (12301, 129, "f32"), (20000, 77, "f16"), (9000, 5003, "bf16")])
def test_loss_of_several_rows_to_a_workgroup(rows, vocab, dt):
    """More rows than workgroups, every second to fifth masked in turn, so that a workgroup's rows come with and without barriers."""
    import torch
    z, _, t, cols = ts._loss_case(1, 1, dt, 1)
    gen = torch.Generator("cuda").manual_seed(rows)
    z = ts.Guarded(rows * vocab, dt, off=1)
    z.t.normal_(0.0, 2.0, generator=gen)
    zz = z.t.view(rows, vocab)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    lp = torch.log_softmax(zz.double(), 1).gather(1, t[:, None])[:, 0]
    i = torch.arange(rows, device="cuda")
    cols = {"old": lp - 0.1 * (i % 7 - 3).double() - 0.05, "ref": lp + 0.1, "adv": torch.randn(rows, generator=gen, device="cuda").double(),
            "weight": ((i * i) % (2 + i // 1000 % 4) != 0).double()}
    t[::97] = -1
    cols = {k: v.float().cpu().numpy() for k, v in cols.items()}
    scale = float(np.float32(0.37))
    for _ in range(3):
        out = ts._run_loss(z, t.cpu(), cols, rows, vocab, dt, **KW)
        wl, wloss, wgrad, wsums = _by_torch(zz, t, cols, scale)
        e = (vocab / 256 + 68 + 3 * math.log(vocab)) * ts.U
        a = np.abs(cols["adv"]).astype(np.float64)
        size = np.abs(cols["weight"]) * (a * math.exp(0.4) + 0.15) * 2
        ts._near(out["logp"].host(), wl.cpu().numpy(), e + 4 * ts.U * np.abs(wl.cpu().numpy()), "logp")
        ts._near(out["loss"].host(), wloss.cpu().numpy(), 2 * size * (e + 4 * ts.U) + 4 * ts.U * np.abs(wloss.cpu().numpy()), "loss")
        got, want = out["grad"].host().reshape(rows, vocab), wgrad.cpu().numpy()
        ts._near(got, want, np.abs(want) * (ts.HALF[dt] + 8 * e + 40 * ts.U) + (scale * size * 4 * (e + 30 * ts.U))[:, None] * torch.softmax(zz.double(), 1).cpu().numpy() + ts.TINY[dt] + (np.arange(vocab)[None] == t.cpu().numpy()[:, None]) * (scale * size * 4 * (e + 8 * ts.U))[:, None], "grad")
        s = wsums.cpu().numpy()
        ts._near(out["sums"].host(), s, 2 * size.sum() * (e + 4 * ts.U) * np.array([1, 1, 1, 0, 0]) + 2 * ts.U * np.abs(s), "sums")


def test_loss_of_logits_that_are_read_past_the_caches():
    """175 MiB of bf16 logits; every 20th row against the definition, all others by their sum (a gradient's row adds up to 0)."""
    import torch
    dfx, _ = ts._dfx()
    rows, vocab = 701, 131071
    gen = torch.Generator("cuda").manual_seed(3)
    z = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda").normal_(0.0, 2.0, generator=gen)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    lp = torch.cat([torch.log_softmax(z[k:k + 100].double(), 1).gather(1, t[k:k + 100, None])[:, 0] for k in range(0, rows, 100)])
    cols = {"old": lp + 0.07, "ref": lp - 0.1, "adv": torch.randn(rows, generator=gen, device="cuda").double(), "weight": (torch.arange(rows, device="cuda") % 6 != 0).double()}
    dev = {k: v.float() for k, v in cols.items()}
    grad = torch.full_like(z, 7.0)
    out = {k: torch.empty(rows, device="cuda") for k in ("logp", "loss")}
    sums = torch.empty(5, device="cuda")
    nb = dfx.policy_loss_workspace(rows, vocab, dfx.BF16)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    dfx.policy_loss(rows, vocab, dfx.BF16, z.data_ptr(), t.data_ptr(), old_logp=dev["old"].data_ptr(), ref_logp=dev["ref"].data_ptr(), advantage=dev["adv"].data_ptr(),
                    weight=dev["weight"].data_ptr(), logp=out["logp"].data_ptr(), loss=out["loss"].data_ptr(), sums=sums.data_ptr(), grad=grad.data_ptr(),
                    workspace=ws.data_ptr(), workspace_bytes=nb, stream=torch.cuda.current_stream().cuda_stream, **KW)
    some = torch.arange(0, rows, 20, device="cuda")
    part = {k: v[some].cpu().numpy() for k, v in dev.items()}
    wl, wloss, wgrad, _ = _by_torch(z[some], t[some], part, 1.0)
    e = (vocab / 256 + 68 + 3 * math.log(vocab)) * ts.U
    size = (np.abs(part["adv"]).astype(np.float64) * 1.2 + 0.1) * np.abs(part["weight"]) * 2
    ts._near(out["logp"][some].double().cpu().numpy(), wl.cpu().numpy(), e + 4 * ts.U * np.abs(wl.cpu().numpy()))
    ts._near(out["loss"][some].double().cpu().numpy(), wloss.cpu().numpy(), 2 * size * (e + 4 * ts.U) + 4 * ts.U * np.abs(wloss.cpu().numpy()))
    w = wgrad.cpu().numpy()
    ts._near(grad[some].double().cpu().numpy(), w, np.abs(w) * (ts.HALF["bf16"] + 8 * e + 80 * ts.U) + ts.TINY["bf16"] + (np.arange(vocab)[None] == t[some].cpu().numpy()[:, None]) * (size * 4 * (e + 8 * ts.U))[:, None])
    total = grad.double().sum(1).abs()
    assert bool((total <= 2.0 ** -8 * 2 * grad.double().abs().sum(1)).all()) and not bool(grad[::6].any())
    assert float(sums[4]) == float(dev["weight"].sum())


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [16500, 33001])
def test_loss_of_rows_that_begin_anywhere(vocab, dt):
    """Every offset of a row within 16 bytes, and of its gradient another one."""
    n = 4 if dt == "f32" else 8
    for off in range(n):
        z, zh, t, cols = ts._loss_case(2, vocab, dt, off, stride=vocab + 1, off=off)
        t[0], t[1] = off, vocab - 1 - off
        lp = st.policy_loss(zh, t.numpy())["logp"]
        cols["old"], cols["ref"] = (lp + 0.05).astype(np.float32), (lp - 0.1).astype(np.float32)
        out = ts._run_loss(z, t, cols, 2, vocab, dt, stride=vocab + 1, goff=(off * 3 + 1) % n, **KW)
        ts._check_loss(out, zh, t, cols, 2, vocab, dt, **KW)
        z.check()


def test_an_error_that_another_call_left_behind_is_not_this_ones():
    """A call of the program's own that failed (a device that there is not) leaves its error with the runtime; the calls here report their own."""
    import ctypes
    import glob
    import os
    import torch
    dfx, _ = ts._dfx()
    libs = glob.glob(os.path.join(torch.__path__[0], "lib", "libamdhip64.so*"))
    if not libs:
        pytest.skip("the runtime's library is not beside torch")
    hip = ctypes.CDLL(libs[0])
    lists, bufs = ts._adam_state([(300, "f32")], 1, "bf16", "bf16")
    n = ts._scalar()
    z, zh, t, cols = ts._loss_case(4, 30000, "bf16", 3)
    lp, tt = ts.Guarded(4, "f32"), t.cuda()
    torch.cuda.synchronize()
    assert hip.hipSetDevice(999) != 0
    try:
        dfx.grad_norm(lists[1], n.ptr())
        dfx.clip_grad_norm(lists[1], n.ptr(), 1.0)
        dfx.adamw(*lists[:4], dfx.AdamWConfig(), copies=lists[4], norm=n.ptr())
        dfx.policy_loss(4, 30000, dfx.BF16, z.ptr(), tt.data_ptr(), logp=lp.ptr())
    finally:
        hip.hipGetLastError()
    torch.cuda.synchronize()
    assert float(n.t) > 0 and bool((lp.t < 0).all())


def test_lists_of_more_chunks_than_a_launch_has_workgroups():
    """2^20 + 3 tensors of one or two elements, so that a list begins a second launch: norm, clipping in place, AdamW with a copy."""
    dfx, _ = ts._dfx()
    n = (1 << 20) + 3
    _, bufs = ts._adam_state([(n + 1, "f32")], 41, "bf16", "f16")
    lists = []
    for bb in bufs:
        at, eb, dt = bb[0].ptr(), bb[0].t.element_size(), {"torch.float32": dfx.F32, "torch.bfloat16": dfx.BF16, "torch.float16": dfx.F16}[str(bb[0].t.dtype)]
        lists.append(dfx.TensorList([(at + k * eb, 1 if k < n - 1 else 2, dt) for k in range(n)]))
    norm = ts._scalar()
    g = bufs[1][0].host()
    dfx.grad_norm(lists[1], norm.ptr())
    want = math.sqrt(float((g * g).sum()))
    assert abs(float(norm.t) - want) <= 2 * ts.U * want
    f = st.clip_factor(float(norm.t), want / 4)
    dfx.grad_clip(lists[1], norm.ptr(), want / 4)
    ts._near(bufs[1][0].host(), g * f, np.abs(g * f) * (2.0 ** -9 + 8 * ts.U) + ts.TINY["bf16"], "clipped")
    before = [[b.host() for b in bb] for bb in bufs[:4]]
    dfx.adamw(*lists[:4], dfx.AdamWConfig(lr=0.01, step=3, weight_decay=0.1), copies=lists[4])
    ts._check_adam(before, bufs, "f16", 3, 0.01, 0.9, 0.999, 1e-8, 0.1, 1.0)
    norm.check()
