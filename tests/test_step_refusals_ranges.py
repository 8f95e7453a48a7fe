"""What the operators of the training step refuse because memory that is written lies on other memory of the call, before they touch a GPU."""
import pytest

from tests.test_step_refusals import _args

# 4 rows of 100 bf16 at 0x10000 (0x320 bytes), targets at 0x20000 (0x20), advantage at 0x30000 (0x10)
WORK = dict(workspace=0x80000, workspace_bytes=1 << 16)
INPUTS = {"old_logp": 0x40000, "ref_logp": 0x50000, "weight": 0x60000, "scale": 0x70000}
ON = [dict(sums=0x30000 - 16), dict(sums=0x3000c), dict(sums=0x2001c), dict(sums=0x20000 - 16), dict(sums=0x10000), dict(sums=0x1031c), dict(sums=0x40000), dict(sums=0x5000c),
      dict(sums=0x60000 - 16), dict(sums=0x70000), dict(sums=0x70000 - 16), dict(sums=0x90000, logp=0x90010), dict(sums=0x90000, loss=0x90000 - 12), dict(sums=0x80000),
      dict(logp=0x10000), dict(loss=0x10320 - 4), dict(logp=0x10000 - 12), dict(grad=0x90000, logp=0x90000), dict(grad=0x90000, loss=0x9031c), dict(grad=0x90000, sums=0x90100),
      dict(grad=0x20000 - 0x310), dict(grad=0x30004), dict(grad=0x40000), dict(grad=0x50000 - 0x31e), dict(grad=0x6000e), dict(grad=0x70002), dict(grad=0x80000), dict(logp=0x80000),
      dict(sums=0x90000, workspace=0x10008), dict(sums=0x90000, workspace=0x20000), dict(sums=0x90000, workspace=0x60008),
      # rows apart: in the second and in the last row's logits
      dict(logits_stride=200, logp=0x10000 + 400 - 4), dict(logits_stride=200, sums=0x10000 + 1200 + 196), dict(logits_stride=200, sums=0x10000 + 200 + 184)]


@pytest.mark.parametrize("kw", ON, ids=[",".join("%s=%x" % i for i in k.items()) for k in ON])
def test_loss_refuses_to_write_on_what_it_reads_or_writes(kw):
    import paper_2303_06324_amd as dfx
    from paper_2303_06324_amd import binding
    assert binding._lib.dfx_policy_loss(_args(dfx, **{**INPUTS, **WORK, **kw}), None) == dfx.ERR_INVALID_ARG
