"""More of the operators at the two ends of a language model against their definitions in 64 bits: calls that went wrong once.  Tolerances as in test_gpu_ends.py."""
import numpy as np
import pytest

from tests.test_gpu_ends import Vocab, _dfx, _np, _rows, _t
from tests.test_gpu_step import HALF, TINY, U, Guarded, _near

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
