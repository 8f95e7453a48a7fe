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
