"""What the operators at the two ends of a language model refuse before they touch a GPU, and the bytes that their workspaces take."""
import ctypes

import pytest

NAN, INF = float("nan"), float("inf")


def _lib():
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding
    return dfx, binding._lib


def _fill(a, base, kw):
    a.struct_bytes = ctypes.sizeof(a)
    for k, v in {**base, **kw}.items():
        assert hasattr(a, k), k
        setattr(a, k, v)
    return a


# 4 rows of 100 bf16, a table of 50 rows (0x2710 bytes)
EMBED = dict(dtype=1, rows=4, dim=100, vocab=50, tokens=0x10000, table=0x20000, out=0x30000, scale=1.0)
EMBED_BAD = [dict(struct_bytes=8), dict(dtype=3), dict(dtype=-1), dict(tokens=None), dict(tokens=0x10004), dict(table=None), dict(table=0x20001), dict(out=None), dict(out=0x30001),
             dict(table_stride=99), dict(out_stride=99), dict(scale=NAN), dict(scale=INF), dict(scale=1e39), dict(out=0x10000), dict(out=0x1001e), dict(out=0x10000 - 0x31e),
             dict(out=0x20000 + 0x270e), dict(out=0x20000 - 0x31e), dict(out=0x20000 - 0x400, out_stride=200)]

GRAD = dict(dtype=1, out_dtype=1, rows=4, dim=100, vocab=50, tokens=0x10000, grad=0x20000, table_grad=0x30000, scale=1.0, workspace=0x40000, workspace_bytes=1 << 24)
GRAD_BAD = [dict(struct_bytes=8), dict(dtype=3), dict(out_dtype=2), dict(dtype=0, out_dtype=1), dict(tokens=None), dict(tokens=0x10004), dict(grad=None), dict(grad=0x20001),
            dict(table_grad=None), dict(table_grad=0x30001), dict(out_dtype=0, table_grad=0x30002), dict(grad_stride=99), dict(table_grad_stride=99), dict(scale=NAN),
            dict(workspace=None), dict(workspace=0x40008), dict(workspace_bytes=16), dict(table_grad=0x10000), dict(table_grad=0x20000), dict(table_grad=0x40000),
            dict(workspace=0x10000), dict(workspace=0x20000), dict(table_grad=0x20000 - 0x2700)]

NORM = dict(dtype=1, param_dtype=0, rows=4, dim=100, x=0x10000, weight=0x20000, bias=0x30000, y=0x40000, eps=1e-5)
NORM_BAD = [dict(struct_bytes=8), dict(dtype=3), dict(param_dtype=2), dict(dtype=0, param_dtype=1), dict(reserved0=1), dict(dim=0), dict(x=None), dict(y=None), dict(x=0x10001), dict(y=0x40001),
            dict(weight=0x20002), dict(bias=0x30002), dict(x_stride=99), dict(y_stride=99), dict(eps=-1e-5), dict(eps=NAN), dict(eps=INF), dict(eps=1e-39),
            dict(y=0x10002), dict(y=0x10000, y_stride=101), dict(y=0x20000), dict(y=0x3018e), dict(y=0x20000 - 0x31e)]

NORM_GRAD = dict(dtype=1, param_dtype=0, grad_dtype=0, rows=4, dim=100, x=0x10000, dy=0x20000, weight=0x30000, dx=0x40000, grad_weight=0x50000, grad_bias=0x60000, eps=1e-5,
                 workspace=0x70000, workspace_bytes=1 << 20)
NORM_GRAD_BAD = [dict(struct_bytes=8), dict(dtype=3), dict(param_dtype=2), dict(grad_dtype=2), dict(dtype=0, param_dtype=0, grad_dtype=1), dict(reserved0=1), dict(dim=0), dict(x=None),
                 dict(dy=None), dict(x=0x10001), dict(dy=0x20001), dict(dx=0x40001), dict(weight=0x30002), dict(grad_weight=0x50002), dict(grad_bias=0x60002), dict(x_stride=99), dict(dy_stride=99),
                 dict(dx_stride=99), dict(eps=-1.0), dict(eps=1e-40), dict(workspace=None), dict(workspace=0x70008), dict(workspace_bytes=100), dict(dx=0x10002), dict(dx=0x20000, dx_stride=101),
                 dict(dx=0x30000), dict(grad_weight=0x10000), dict(grad_bias=0x20000), dict(grad_weight=0x60000), dict(grad_bias=0x40000), dict(grad_weight=0x30000), dict(workspace=0x10000),
                 dict(workspace=0x20000), dict(workspace=0x30000), dict(workspace=0x40000), dict(grad_weight=0x70000)]

# 4 rows and 50 of 64 bf16 (0x200 and 0x1900 bytes)
VOCAB = dict(dtype=1, grad_dtype=1, rows=4, dim=64, vocab=50, hidden=0x10000, weight=0x20000, targets=0x30000, row_weight=0x40000, scale=0x50000, logp=0x60000, loss=0x70000, sums=0x80000,
             grad_hidden=0x90000, grad_weight=0xa0000, inv_temperature=1.0, workspace=0x1000000, workspace_bytes=1 << 30)
READS = {"hidden": 0x10000, "weight": 0x20000, "targets": 0x30000, "row_weight": 0x40000, "scale": 0x50000}
VOCAB_BAD = [dict(struct_bytes=8), dict(dtype=3), dict(grad_dtype=2), dict(dtype=0, grad_dtype=1), dict(dim=0), dict(hidden=None), dict(weight=None), dict(targets=None), dict(targets=0x30004),
             dict(hidden=0x10001), dict(weight=0x20001), dict(grad_hidden=0x90001), dict(grad_weight=0xa0001), dict(grad_dtype=0, grad_weight=0xa0002), dict(row_weight=0x40002), dict(scale=0x50002),
             dict(logp=0x60002), dict(loss=0x70002), dict(sums=0x80002), dict(hidden_stride=63), dict(weight_stride=63), dict(grad_hidden_stride=63), dict(grad_weight_stride=63),
             dict(inv_temperature=0.0), dict(inv_temperature=-1.0), dict(inv_temperature=INF), dict(inv_temperature=NAN), dict(inv_temperature=1e-39), dict(piece=100), dict(workspace=None),
             dict(workspace=0x1000080), dict(workspace_bytes=1000), dict(grad_hidden=0x101fe), dict(grad_hidden=0x10000), dict(grad_weight=0x20000), dict(grad_weight=0x90000), dict(loss=0x60008),
             dict(sums=0x60008), dict(logp=0xa1800), dict(workspace=0x10000), dict(workspace=0x0)] + [
    dict([(w, at)]) for w in ("logp", "loss", "sums", "grad_hidden") for at in READS.values()]

CALLS = {"embed": ("EmbedArgs", EMBED, EMBED_BAD), "embed_grad": ("EmbedGradArgs", GRAD, GRAD_BAD), "layer_norm": ("LayerNormArgs", NORM, NORM_BAD),
         "layer_norm_grad": ("LayerNormGradArgs", NORM_GRAD, NORM_GRAD_BAD), "vocab_loss": ("VocabLossArgs", VOCAB, VOCAB_BAD)}


def _call(what, kw):
    dfx, lib = _lib()
    name, base, _ = CALLS[what]
    return getattr(lib, "dfx_" + what)(_fill(getattr(dfx, name)(), base, kw), None)


@pytest.mark.parametrize("what,kw", [(w, k) for w, c in CALLS.items() for k in c[2]], ids=lambda v: v if isinstance(v, str) else ",".join("%s=%s" % i for i in v.items()))
def test_refused(what, kw):
    dfx, _ = _lib()
    assert _call(what, kw) == dfx.ERR_INVALID_ARG


@pytest.mark.parametrize("what", list(CALLS))
def test_too_large(what):
    dfx, lib = _lib()
    name, base, _ = CALLS[what]
    assert getattr(lib, "dfx_" + what)(None, None) == dfx.ERR_INVALID_ARG
    sizes = [dict(rows=1 << 31), dict(rows=(1 << 31) - 1024), dict(dim=1 << 20)] + [{k: 1 << 20} for k in base if k.endswith("_stride")]
    if "vocab" in base:
        sizes.append(dict(vocab=(1 << 31) - 1024))
    else:
        sizes.append(dict(dim=32769))
    for kw in sizes:
        assert _call(what, kw) == dfx.ERR_TOO_LARGE, kw


def test_too_many_tiles_of_a_vocabulary():
    """A launch's threads are counted in 32 bits."""
    dfx, _ = _lib()
    for kw in (dict(rows=(1 << 24) - 1024), dict(vocab=1 << 28), dict(rows=1 << 22, vocab=1 << 16), dict(rows=1 << 23, vocab=50257)):
        assert _call("vocab_loss", kw) == dfx.ERR_TOO_LARGE, kw
        size = dict(dict(rows=4, vocab=50), **kw)
        assert dfx.vocab_loss_workspace(size["rows"], 100, size["vocab"], dfx.BF16) == 0, kw
    for rows, vocab in ((1 << 20, 1 << 16), (256, (1 << 28) - 1), (1, (1 << 28) - 1)):
        assert dfx.vocab_loss_workspace(rows, 100, vocab, dfx.BF16) > 0


def test_workspaces_have_room_for_fewer_rows():
    dfx, _ = _lib()
    rows = [0, 1, 2, 3, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 1023, 1024, 1025, 4095, 4097, 8191, 8192, 16384, 65535, 65536, 65537, 100000, 300001]
    for dim, vocab in ((64, 1000), (1001, 50257), (4096, 131072), (8192, 300)):
        for sizes in ([dfx.embed_grad_workspace(r, dim, vocab, dfx.BF16) for r in rows], [dfx.layer_norm_grad_workspace(r, dim, dfx.BF16) for r in rows],
                      *[[dfx.vocab_loss_workspace(r, dim, vocab, t, g, p) for r in rows] for t in (dfx.F32, dfx.BF16) for g in (False, True) for p in (0, 512, 1 << 20)]):
            assert sizes == sorted(sizes) and sizes[0] > 0, (dim, vocab)


def test_workspaces_of_what_is_refused():
    dfx, _ = _lib()
    assert dfx.vocab_loss_workspace(10, 64, 100, dfx.BF16, True, 100) == 0 and dfx.vocab_loss_workspace(1 << 31, 64, 100, dfx.BF16) == 0
    assert dfx.embed_grad_workspace(1 << 31, 64, 100, dfx.BF16) == 0 and dfx.layer_norm_grad_workspace(10, 1 << 15 | 1, dfx.BF16) == 0


def test_nothing_to_do_is_no_error():
    dfx, _ = _lib()
    assert _call("embed", dict(rows=0, tokens=None, out=None)) == dfx.OK
    assert _call("embed", dict(dim=0)) == dfx.OK
    assert _call("embed_grad", dict(vocab=0, table_grad=None)) == dfx.OK
    assert _call("layer_norm", dict(rows=0, x=None, y=None)) == dfx.OK
    assert _call("layer_norm_grad", dict(rows=0, x=None, dy=None, dx=None, grad_weight=None, grad_bias=None, workspace=None)) == dfx.OK
