"""More of what the operators at the two ends of a language model refuse before they touch a GPU."""
import subprocess
import sys

import pytest

from tests.test_ends_refusals import _call, _lib

TYPES = (0, 1, 2)


@pytest.mark.parametrize("dtype", [-1, *TYPES, 3, 99])
@pytest.mark.parametrize("grad", [False, True])
def test_workspace_of_rows_without_elements(dtype, grad):
    """The call refuses dim = 0; so does the question for its workspace (which divided by the number of tiles: in a process of its own, as that ends one)."""
    code = "import paper_2303_06324_amd as dfx; print([dfx.vocab_loss_workspace(r, 0, v, %d, %r, p) for r in (0, 5, 300) for v in (0, 100) for p in (0, 256)])" % (dtype, grad)
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == str([0] * 12), out


@pytest.mark.parametrize("dtype", [-1, 3, 99])
def test_workspace_of_an_unknown_type(dtype):
    dfx, _ = _lib()
    assert _call("vocab_loss", dict(dtype=dtype, grad_dtype=dtype)) == dfx.ERR_INVALID_ARG
    for grad in (False, True):
        assert dfx.vocab_loss_workspace(10, 64, 100, dtype, grad) == 0


# 4 rows of 100 bf16, 400 elements (0x320 bytes) from one to the next: behind a row's 0xc8 bytes there are 0x258 that are the matrix's as well
@pytest.mark.parametrize("kw", [dict(x_stride=101, y_stride=400, weight=0x40000 + 0xc8), dict(y_stride=400, bias=0x40000 + 0x320 + 0xc8)])
def test_layer_norm_with_parameters_between_the_rows(kw):
    """All space from a written matrix's first to its last row is that matrix's: its type's parameters (0xc8 bytes) would fit in between."""
    dfx, _ = _lib()
    assert _call("layer_norm", dict(kw, param_dtype=1)) == dfx.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(dx_stride=400, weight=0x40000 + 0xc8), dict(x_stride=400, grad_weight=0x10000 + 0xc8), dict(dy_stride=400, grad_bias=0x20000 + 0x320 + 0xc8),
                                dict(dx_stride=400, grad_bias=0x40000 + 0xc8)])
def test_layer_norm_grad_with_parameters_between_the_rows(kw):
    dfx, _ = _lib()
    assert _call("layer_norm_grad", dict(kw, param_dtype=1, grad_dtype=1)) == dfx.ERR_INVALID_ARG
