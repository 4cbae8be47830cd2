"""Paths of the operators for adapters over 8-bit frozen weights that take particular sizes or values to be reached.  Tolerances as in
test_gpu_i8."""
import pytest
import torch

import test_gpu_i8 as I
from paper_2407_00952_b200 import binding as B

pytestmark = pytest.mark.gpu

U, HALF, CHAIN, DTYPES = I.U, I.HALF, I.CHAIN, I.DTYPES
BF16, F32 = torch.bfloat16, torch.float32


# ---- norm and its gradient ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,d", [(50, 136), (37, 1001), (9, 8192), (6, 16383)])
def test_norm_and_gradient_in_place_wherever_arrays_start(M, d, residual, dtype):
    """The sum over x or the residual, dx over dy or the residual: bit for bit what separate outputs get, at every pair of places."""
    g = I.gen(M + 5 * d)
    x, r, dy = (I.randn(g, M, d, dtype=dtype) for _ in range(3))
    gain = (1 + 0.2 * I.randn(g, d)).to(dtype)
    for ox, orr in [(0, 0), (1, 1), (0, 3), (2, 1)]:
        def fresh():
            return I.offset(x, ox), I.offset(r, orr) if residual else None
        a, b = fresh()
        want = B.rmsnorm_quantize(a, gain, residual=b, want_y=True, h=I.offset(x, ox))
        for into in (0, 1) if residual else (0,):
            a, b = fresh()
            got = B.rmsnorm_quantize(a, gain, residual=b, want_y=True, h=(a, b)[into])
            for i in range(4):
                assert torch.equal(got[i], want[i]), (ox, orr, into, i)
        up, res = I.offset(dy, ox), I.offset(r, orr) if residual else None
        dx = B.rmsnorm_bwd(up, x, gain, resid=res)[0]
        assert torch.equal(B.rmsnorm_bwd(up, x, gain, resid=res, dx=up)[0], dx)
        if residual:
            assert torch.equal(B.rmsnorm_bwd(I.offset(dy, ox), x, gain, resid=res, dx=res)[0], dx)


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


# ---- streams -----------------------------------------------------------------------------------
def test_the_current_stream_by_either_name(monkeypatch):
    x = I.randn(I.gen(2), 40, 136, dtype=BF16)
    want = B.quantize_rows(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        dev = torch.cuda.current_device()
        assert B._raw_stream(dev) == B._public_raw_stream(dev) == s.cuda_stream
        monkeypatch.setattr(B, "_raw_stream", B._public_raw_stream)
        got = B.quantize_rows(x)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
