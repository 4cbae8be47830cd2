"""Paths of the operators for adapters over 8-bit frozen weights that take particular sizes or values to be reached.  Tolerances as in
test_gpu_i8."""
import pytest
import torch

import test_gpu_i8 as I
from paper_2407_00952_b200 import binding as B

pytestmark = pytest.mark.gpu

U, HALF, CHAIN, DTYPES = I.U, I.HALF, I.CHAIN, I.DTYPES
BF16, F32 = torch.bfloat16, torch.float32


# ---- loss --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,V", [(BF16, 500), (BF16, 20000), (BF16, 120001), (BF16, 120000), (F32, 500), (F32, 20000), (F32, 60000)])
def test_loss_without_the_teachers_weight_does_not_see_its_logits(V, dtype):
    """kd_weight 0: the cross-entropy, whatever the buffers of the teacher hold."""
    z, idx, t, y = I.distill_case(9, V, 12, dtype, V)
    idx = torch.where(torch.rand(9, 12, device="cuda", generator=I.gen(1), dtype=F32) < 0.3, y.clamp(0, V - 1)[:, None], idx).contiguous()
    kw = dict(labels=y, temperature=2.0, ce_weight=1.0, kd_weight=0.0)
    want = B.distill_loss(z, idx, t, **kw)
    I.check_distill(z, idx, t, y, 2.0, 1.0, 0.0, want)
    for bad in (float("nan"), float("inf"), 3e38):
        u = t.clone()
        u[:, 3::2] = bad
        for a, b in zip(B.distill_loss(z, idx, u, **kw), want):
            assert torch.equal(a, b), bad
