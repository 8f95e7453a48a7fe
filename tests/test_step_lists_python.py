"""Lists as the Python side hands them on, without a GPU: triples that only add up."""
import pytest


def test_triples_that_only_add_up_are_refused():
    """Two and four numbers are two tensors' worth, but not two tensors: read as words they would name memory that nobody meant."""
    import paper_2303_06324_amd as dfx
    for bad in ([(0x1000, 4), (dfx.F32, 0x2000, 4, dfx.F32)], [(0x1000, 4, dfx.F32, 0x2000), (4, dfx.F32)], [(), (0x1000, 4, dfx.F32, 0x2000, 4, dfx.F32)]):
        with pytest.raises(ValueError):
            dfx.TensorList(bad)
