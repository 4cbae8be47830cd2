"""Paths of the operators for adapters over 8-bit frozen weights that take particular sizes or values to be reached: several rows per group in the
gain's gradient, few tokens onto many channels, losses over rows wider than shared memory, and outputs in place of inputs.  Tolerances as in test_gpu_i8."""
import math

import pytest
import torch

import test_gpu_i8 as I
from paper_2407_00952_b200 import binding as B

pytestmark = pytest.mark.gpu

U, HALF, CHAIN, DTYPES = I.U, I.HALF, I.CHAIN, I.DTYPES
BF16, F32 = torch.bfloat16, torch.float32


# ---- gain's gradient, several rows per group ---------------------------------------------------
def dg_chain(M, d, dtype, frame):
    """(longest chain of additions in a column of dg, rows per group): a group's rows one after the other, the groups of a block, then
    eight threads adding the blocks' sums and their eight sums."""
    w = 8 if dtype is BF16 else 4
    need = math.ceil(math.ceil(d / w) / 4)
    if need > 32:
        threads = math.ceil(need / 32) * 32
    else:
        threads = 2 * w if frame else 1
        while threads < need:
            threads *= 2
    per = 1 if threads > 512 else 512 // threads
    most = math.ceil(M / per)
    blocks = min(torch.cuda.get_device_properties(0).multi_processor_count, 592, most)
    if blocks < most:
        blocks = blocks // 8 * 8
    rows = math.ceil(M / (blocks * per))
    return rows + per + math.ceil(blocks / 8) + 8, rows


def check_bwd(h, dy, gain, res, dx, dg, frame, what):
    M, d = h.shape
    chain, rows = dg_chain(M, d, h.dtype, frame)
    assert rows > 1, "one row per group: not what this test is about"
    ref, size, rg, sg = I.norm_grad64(dy, h, gain, res, 1e-5)
    I.check(dx, ref, HALF[h.dtype] * ref.abs() + 2 * CHAIN * U * size + 1e-40, ("dx", what))
    # a term dy h rstd: rstd (its sum's chain halved by the root, rsqrt and the mean), a product, a fused product and sum
    I.check(dg, rg, (chain + CHAIN / 2 + 10) * U * sg + 1e-40, ("dg", what))


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,d,dtype", [
    (700, 4096, BF16), (2000, 4096, F32), (700, 4095, BF16), (2000, 4095, F32), (60000, 64, BF16), (20000, 64, F32), (60001, 24, F32), (3000, 1001, BF16),
    (3000, 1001, F32), (400, 16384, BF16), (400, 16383, BF16), (400, 16384, F32), (400, 16383, F32), (301, 8200, F32)])
def test_gain_gradient_over_several_rows_per_group(M, d, dtype, residual):
    g = I.gen(M + d)
    h, dy = I.randn(g, M, d, dtype=dtype), I.randn(g, M, d, dtype=dtype)
    h[1], dy[2] = 0, 0
    h[M - 1] *= 50                                 # the last row, which few groups have, weighs as much as any
    gain = (1 + 0.2 * I.randn(g, d)).to(dtype)
    res = I.randn(g, M, d, dtype=dtype) if residual else None
    frame = d % (8 if dtype is BF16 else 4) != 0
    dx, dg = B.rmsnorm_bwd(dy, h, gain, resid=res, want_dg=True)
    check_bwd(h, dy, gain, res, dx, dg, frame, "plain")
    assert torch.equal(B.rmsnorm_bwd(dy, h, gain, resid=res)[0], dx)             # dx does not depend on whether dg is asked for
    a = dy.clone()
    over, dg2 = B.rmsnorm_bwd(a, h, gain, resid=res, want_dg=True, dx=a)
    assert torch.equal(over, dx) and torch.equal(dg2, dg)
    if residual:
        a = res.clone()
        over, dg2 = B.rmsnorm_bwd(dy, h, gain, resid=a, want_dg=True, dx=a)
        assert torch.equal(over, dx) and torch.equal(dg2, dg)
    # a workspace whose contents on entry do not matter
    n = 4 * min(M, 592) * d
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")                 # NaN as fp32
    assert torch.equal(B.rmsnorm_bwd(dy, h, gain, resid=res, want_dg=True, workspace=ws)[1], dg)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,d", [(5000, 1000), (3000, 1001), (400, 16384)])
def test_gain_gradient_over_several_rows_of_arrays_at_different_places(M, d, dtype):
    g = I.gen(M * 3 + d)
    h, dy, res = (I.randn(g, M, d, dtype=dtype) for _ in range(3))
    gain = I.randn(g, d, dtype=dtype)
    places = [(1, 1, 1), (0, 1, 2), (3, 0, 1), (2, 3, 3)]
    for oy, oh, orr in places:
        a, b = I.offset(dy, oy), I.offset(res, orr)
        hh = I.offset(h, oh)
        dx, dg = B.rmsnorm_bwd(a, hh, gain, resid=b, want_dg=True)
        check_bwd(h, dy, gain, res, dx, dg, True, (oy, oh, orr))
        for into in (a, b):
            keep = into.clone()
            over, dg2 = B.rmsnorm_bwd(a, hh, gain, resid=b, want_dg=True, dx=into)
            assert torch.equal(over, dx) and torch.equal(dg2, dg)
            into.copy_(keep)


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


def test_gain_gradient_beyond_32_bit_offsets():
    """Hundreds of rows per group, more than 2^31 elements; rows of zeros but for the first and last, which alone count."""
    M, d = 131300, 16383
    g = I.gen(8)
    h = torch.zeros(M, d, dtype=BF16, device="cuda")
    ends = torch.cat([torch.arange(40), torch.arange(M - 40, M)]).cuda()
    part = I.randn(g, 80, d, dtype=BF16)
    h[ends] = part
    gain = (1 + 0.2 * I.randn(g, d)).to(BF16)
    dx, dg = B.rmsnorm_bwd(h, h, gain, want_dg=True)
    ref, size, rg, sg = I.norm_grad64(part, part, gain, None, 1e-5)
    I.check(dx[ends], ref, HALF[BF16] * ref.abs() + 2 * CHAIN * U * size, "dx")
    chain, rows = dg_chain(M, d, BF16, True)
    assert rows > 500
    I.check(dg, rg, (chain + CHAIN / 2 + 10) * U * sg, "dg")


# ---- products: few tokens onto many channels ---------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 2, 3, 4])
@pytest.mark.parametrize("K,N", [(100, 8192), (100, 11009), (4096, 8192), (4096, 11009), (520, 8191), (15, 9000)])
def test_few_tokens_onto_many_channels(M, K, N, dtype):
    """Channels per warp go by their number; 11009 and 8191 leave the last warp a part of its own."""
    I.run_product(M, K, N, dtype)
    I.run_product(M, K, N, dtype, sw=False, bias=False, res=False)
    assert B.library_status() == 0


def test_few_tokens_are_rows_of_many():
    x, sx, w, sw, b, r, y = I.run_product(64, 1000, 8200, BF16)
    for m in (1, 2, 3, 4):
        assert torch.equal(B.linear_i8(x[:m], sx[:m], w, sw, bias=b, residual=r[:m].contiguous()), y[:m])


# ---- loss --------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 3, 8, 9, 15, 255, 256, 1023, 1024, 1025, 1031, 2047, 2048, 2056, 2063, 4103, 32001, 113001])
def test_loss_in_place_bit_for_bit_wherever_rows_start(V, dtype):
    if dtype is F32 and V > 100000:
        V = 57003
    z, idx, t, y = I.distill_case(13, V, min(V, 9), dtype, V + 3)
    for T in (1.0, 2.0, 1.3):
        for by in (0, 1, 2, 3):
            kw = dict(labels=y, temperature=T, ce_weight=0.4, kd_weight=0.6)
            loss, rows, dz = B.distill_loss(I.offset(z, by), idx, t, **kw)
            same = I.offset(z, by)
            loss1, rows1, _ = B.distill_loss(same, idx, t, dlogits=same, **kw)
            assert torch.equal(same, dz) and torch.equal(rows1, rows) and torch.equal(loss1, loss), (T, by)


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


@pytest.mark.parametrize("dtype,V", [(BF16, 120000), (BF16, 120001), (F32, 60000), (F32, 60001)])
@pytest.mark.parametrize("T", [1.0, 2.0, 1.3])
def test_loss_of_masked_and_broken_logits_in_rows_wider_than_shared_memory(V, T, dtype):
    z, idx, t, y = I.distill_case(12, V, 6, dtype, V + 1)
    z, idx, t = z.clamp(min=-20), idx.clamp(0, V - 1), torch.zeros_like(t)
    y[:] = 5
    dead = torch.zeros(12, V, dtype=torch.bool, device="cuda")
    for m in range(6):
        dead[m, m % 3::3] = True
    dead[4, :V // 2] = True
    dead[5, V // 3:] = True
    keep = torch.zeros_like(dead).scatter_(1, idx.long(), True)
    keep[:, 5] = True
    dead &= ~keep
    z[dead] = -float("inf")
    z[6, 17], z[7, V - 1], z[8, 0], z[9, V // 2] = float("nan"), float("nan"), float("inf"), float("inf")
    loss, rows, dz = B.distill_loss(z, idx, t, labels=y, temperature=T, ce_weight=0.5, kd_weight=0.5)
    assert (dz[dead] == 0).all() and torch.isnan(loss)
    broken = torch.zeros(12, dtype=torch.bool, device="cuda")
    broken[6:10] = True
    assert torch.isnan(rows[broken]).all() and torch.isnan(dz[broken]).all()
    ok = ~broken
    rr, _, rg, size = I.distill64(z[ok].double().clamp(min=-1e30), idx[ok], t[ok], y[ok], T, 0.5, 0.5, 12)
    rel = (2 * 40 / min(T, 1.0) + V / 128 + 64) * U
    I.check(dz[ok], rg, HALF[dtype] * rg.abs() + rel * size + 1e-40, "dlogits")
    I.check(rows[ok], rr, rel * (rr.abs() + 0.5 + 0.5 * T * T * 50), "rows")


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
