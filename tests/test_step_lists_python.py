"""Lists as the Python side hands them on, without a GPU: triples that only add up, and lists that are gone."""
import ctypes

import pytest


def test_triples_that_only_add_up_are_refused():
    """Two and four numbers are two tensors' worth, but not two tensors: read as words they would name memory that nobody meant."""
    import paper_2303_06324_amd as dfx
    for bad in ([(0x1000, 4), (dfx.F32, 0x2000, 4, dfx.F32)], [(0x1000, 4, dfx.F32, 0x2000), (4, dfx.F32)], [(), (0x1000, 4, dfx.F32, 0x2000, 4, dfx.F32)]):
        with pytest.raises(ValueError):
            dfx.TensorList(bad)


def _list(handle):
    """A list of this handle, which no call below follows and nothing frees."""
    import paper_2303_06324_amd as dfx
    t = dfx.TensorList.__new__(dfx.TensorList)
    t._h = ctypes.c_void_p(handle)
    t.destroy = lambda: 0
    return t


def test_a_list_that_is_gone_is_not_an_absent_one(monkeypatch):
    """out = a destroyed list is not "in place", copies = a destroyed list is not "no copies"."""
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding

    class Lib:
        dfx_strerror = staticmethod(binding._lib.dfx_strerror)

        def __getattr__(self, name):
            def call(*args):
                raise AssertionError(name + " was called")
            return call

    held, gone = _list(0x1000), _list(None)
    config = dfx.AdamWConfig()
    monkeypatch.setattr(binding, "_lib", Lib())
    for call in (lambda: dfx.grad_clip(held, 0x2000, 1.0, out=gone), lambda: dfx.clip_grad_norm(held, 0x2000, 1.0, out=gone),
                 lambda: dfx.adamw(held, held, held, held, config, copies=gone)):
        with pytest.raises(dfx.DfxError) as e:
            call()
        assert e.value.status == dfx.ERR_INVALID_ARG
