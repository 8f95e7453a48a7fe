"""What the operators of the training step refuse before they touch a GPU."""
import ctypes

import pytest


def _args(dfx, **kw):
    a = dfx.PolicyLossArgs()
    a.struct_bytes, a.dtype, a.rows, a.vocab = ctypes.sizeof(a), dfx.BF16, 4, 100
    a.logits, a.targets, a.advantage, a.inv_temperature = 0x10000, 0x20000, 0x30000, 1.0
    a.clip_low = a.clip_high = 0.2
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD = [dict(struct_bytes=4), dict(dtype=3), dict(dtype=-1), dict(logits=0x10001), dict(targets=0x20004), dict(targets=None), dict(logits=None),
       dict(logits_stride=99), dict(grad=0x90000, grad_stride=99), dict(grad=0x90001), dict(grad=0x10000, grad_stride=101), dict(grad=0x10010),
       dict(grad=0x10000 - 798), dict(advantage=None, grad=0x90000), dict(advantage=None, loss=0x90000), dict(loss=0x90002),
       dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-0.1), dict(clip_high=float("nan")), dict(kl_coef=0.1), dict(kl_coef=float("inf")),
       dict(inv_temperature=0.0), dict(inv_temperature=-1.0), dict(inv_temperature=float("inf")),
       dict(sums=0x90000), dict(sums=0x90000, workspace=0x80000, workspace_bytes=8), dict(sums=0x90000, workspace=0x80004, workspace_bytes=1 << 20)]


@pytest.mark.parametrize("kw", BAD, ids=[",".join(k) for k in BAD])
def test_loss_refuses(kw):
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding
    assert binding._lib.dfx_policy_loss(_args(dfx, **kw), None) == dfx.ERR_INVALID_ARG


def test_loss_refuses_what_is_too_large():
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding
    lib = binding._lib
    assert lib.dfx_policy_loss(None, None) == dfx.ERR_INVALID_ARG
    for kw in (dict(rows=1 << 31), dict(vocab=(1 << 30) + 1), dict(rows=1 << 30, logits_stride=1 << 40), dict(grad=0x90000, grad_stride=1 << 62)):
        assert lib.dfx_policy_loss(_args(dfx, **kw), None) == dfx.ERR_TOO_LARGE, kw


def test_workspace_grows_no_further_than_its_workgroups():
    import paper_2303_06324_amd as dfx
    sizes = [dfx.policy_loss_workspace(r, 1000, dfx.BF16) for r in (0, 1, 100, 10000, 1 << 30)]
    assert 0 < sizes[0] and sizes == sorted(sizes) and sizes[-1] < 1 << 20


def test_lists_refuse():
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding
    lib = binding._lib
    h = ctypes.c_void_p(5)
    one = (dfx.Tensor * 1)

    def create(*t):
        return lib.dfx_list_create(ctypes.byref(h), one(dfx.Tensor(*t)), 1)

    assert lib.dfx_list_create(None, one(dfx.Tensor(0x1000, 4, dfx.F32, 0)), 1) == dfx.ERR_INVALID_ARG
    assert lib.dfx_list_create(ctypes.byref(h), None, 1) == dfx.ERR_INVALID_ARG and h.value is None
    assert lib.dfx_list_create(ctypes.byref(h), None, -1) == dfx.ERR_INVALID_ARG
    for t in ((0x1000, 4, dfx.I32, 0), (0x1000, 4, 9, 0), (0x1002, 4, dfx.F32, 0), (0x1001, 4, dfx.BF16, 0), (None, 4, dfx.F32, 0), (0x1000, 4, dfx.F32, 1)):
        assert create(*t) == dfx.ERR_INVALID_ARG, t
    assert create(0x1000, 1 << 62, dfx.BF16, 0) == dfx.ERR_TOO_LARGE
    assert create(0x1000, 1 << 50, dfx.BF16, 0) == dfx.ERR_TOO_LARGE
    assert lib.dfx_list_destroy(None) == dfx.ERR_INVALID_ARG
    for call in (lambda: lib.dfx_grad_norm(None, 0, 1.0, 0x1000, None), lambda: lib.dfx_grad_clip(None, None, 0x1000, 1.0, 1.0, None),
                 lambda: lib.dfx_clip_grad_norm(None, None, 0, 1.0, 1.0, 0x1000, None), lambda: lib.dfx_adamw(None, None, None, None, None, None, None, None),
                 lambda: lib.dfx_adamw_default(None)):
        assert call() == dfx.ERR_INVALID_ARG


def test_defaults():
    import paper_2303_06324_amd as dfx
    c = dfx.AdamWConfig(lr=0.5)
    assert c.struct_bytes == ctypes.sizeof(c) and c.lr == 0.5 and c.beta1 == 0.9 and c.grad_scale == 1.0 and not c.step_dev
    with pytest.raises(KeyError):
        dfx.AdamWConfig(momentum=0.9)


@pytest.mark.parametrize("kw", [dict(logp=0x30000), dict(loss=0x30000), dict(logp=0x3000c, loss=0x90000), dict(logp=0x90000, loss=0x90008), dict(logp=0x20010),
                                dict(loss=0x20000 - 12), dict(old_logp=0x90000, logp=0x90000), dict(ref_logp=0x90000, loss=0x90004), dict(weight=0x90000, logp=0x8fff4), dict(scale=0x90000, loss=0x8fff4)])
def test_loss_refuses_results_that_lie_on_what_is_read(kw):
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding
    assert binding._lib.dfx_policy_loss(_args(dfx, **kw), None) == dfx.ERR_INVALID_ARG


def test_lists_of_what_is_no_tensor():
    import paper_2303_06324_amd as dfx
    for bad in ([(0x1000, 4)], [(0x1000, 4, dfx.F32), (0x1000, 4)], [(0x1000, 4, dfx.F32, 0)]):
        with pytest.raises(ValueError):
            dfx.TensorList(bad)
    with pytest.raises(OverflowError):
        dfx.TensorList([(0x1000, -1, dfx.F32)])
    for bad in ([(0x1000, 4, 1 << 32)], [(0x1000, 4, 3)], [(0x1001, 4, dfx.F32)]):
        with pytest.raises(dfx.DfxError):
            dfx.TensorList(bad)


def test_the_longest_vocabulary_is_below_its_bound():
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding
    assert binding._lib.dfx_policy_loss(_args(dfx, vocab=1 << 30), None) == dfx.ERR_TOO_LARGE
