"""Operators for adapters over 8-bit frozen weights against their definitions in 64 bits (decisions of the quantiser: the fp32
operations that the definition prescribes, done by numpy).

Tolerances, per element, from the arithmetic: a rounding to the output type is off by at most eps/2 of the value; every fp32
operation by 2^-24 of its result; a sum in fp32 by its longest chain of additions times 2^-24 times the sum of magnitudes; rsqrtf and
ex2.approx by 2 units in the last place (2^-22)."""
import numpy as np
import pytest
import torch

from paper_2407_00952_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.bfloat16, torch.float32]
CHAIN = 64          # additions in the longest chain of a row's sum: 16 accesses of one element or 4 of 8 per thread, 2 x 5 in the trees


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32).to(dtype)


def offset(t, by):
    """The same values in memory that starts `by` elements past a 16-byte boundary."""
    buf = torch.zeros(t.numel() + by + 64, dtype=t.dtype, device="cuda")
    v = buf[by:by + t.numel()].view(t.shape)
    v.copy_(t)
    return v


def check(got, ref, tol, what=""):
    """|got - ref| <= tol per element, ref and tol in 64 bits."""
    got = got.double()
    assert got.shape == ref.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what
    bad = ((got - ref).abs() > tol) & torch.isfinite(ref)
    assert not bad.any(), (what, float(((got - ref).abs() / tol.clamp(min=1e-300))[torch.isfinite(ref)].max()))


def np_codes(v):
    """Codes and largest magnitudes of rows (numpy fp32), as the definition has them."""
    with np.errstate(all="ignore"):
        a = np.abs(v).max(axis=1)
        fine = np.isfinite(v).all(axis=1)
        live = fine & (a >= np.float32(1e-36))
        inv = np.where(live, np.float32(127) / np.where(live, a, np.float32(1)), np.float32(0)).astype(np.float32)
        q = np.where(live[:, None], np.rint((np.where(live[:, None], v, np.float32(0)) * inv[:, None]).astype(np.float32)), 0)
    return q.astype(np.int8), a, live, fine


def hard_rows(x):
    """Rows on which a quantiser goes wrong: zeros, ties, tiny and huge values, infinities, NaN."""
    M = x.shape[0]
    if M > 3:
        x[1] = 0
        x[2] *= 1e-38
        x[3] *= 1e30
    if M > 8:
        x[4, 0] = float("inf")
        x[5, -1] = float("nan")
        x[6] = 0
        x[6, 0] = 254.0                 # inv = 0.5: odd values are ties
        x[6, 1:] = torch.arange(x.shape[1] - 1, device=x.device) % 250 - 125
        x[7] = -x[7].abs()
        x[8] = 1e-37
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,d", [(1, 1), (1, 128), (3, 7), (9, 8), (17, 100), (64, 1024), (65, 1000), (33, 1001), (5, 4096), (12, 11008), (10, 16385),
                                 (9, 20000), (9, 65536), (9, 40001), (9, 32771),
                                 (9, 49001), (9, 60001)])
def test_quantize_rows(M, d, dtype):
    x = hard_rows(randn(gen(M + d), M, d)).to(dtype)
    f = 0.5 + torch.rand(d, device="cuda", generator=gen(3), dtype=torch.float32)
    for col in (None, f):
        codes, scales = B.quantize_rows(x, col_scale=col)
        v = x.float().cpu().numpy()
        if col is not None:
            with np.errstate(all="ignore"):
                v = v * f.cpu().numpy()
        q, a, live, fine = np_codes(v)
        assert np.array_equal(codes.cpu().numpy(), q)
        want = np.where(live, a / np.float32(127), np.where(fine, np.float32(0), np.float32("nan"))).astype(np.float32)
        assert np.array_equal(scales.cpu().numpy(), want, equal_nan=True)
        for out in DTYPES:
            back = B.dequantize_rows(codes, scales, out)
            ref = torch.from_numpy(q.astype(np.float32) * want[:, None]).cuda()         # one fp32 product, then one rounding
            assert torch.equal(torch.nan_to_num(back), torch.nan_to_num(ref.to(out))) and torch.equal(torch.isnan(back), torch.isnan(ref))


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_rows_layouts(dtype):
    """Rows that start anywhere, codes whose rows lie apart; what lies between the rows stays as it was."""
    x = randn(gen(5), 37, 200, dtype=dtype)
    want, ws = B.quantize_rows(x)
    for by in (1, 2, 3):
        got, gs = B.quantize_rows(offset(x, by))
        assert torch.equal(got, want) and torch.equal(gs, ws)
    for lead, wide in ((0, 208), (0, 201), (3, 217), (8, 240)):
        buf = torch.full((38, wide), 77, dtype=torch.int8, device="cuda")
        view = buf[:37, lead:lead + 200]
        got, gs = B.quantize_rows(x, codes=view)
        assert torch.equal(got, want) and torch.equal(gs, ws)
        rest = buf.clone()
        rest[:37, lead:lead + 200] = 77
        assert (rest == 77).all()
        assert torch.equal(B.dequantize_rows(view, gs, dtype), B.dequantize_rows(want, ws, dtype))


def norm_case(M, d, dtype, seed, residual):
    g = gen(seed)
    x = hard_rows(randn(g, M, d) * (1 + 15 * (torch.rand(d, device="cuda", generator=g, dtype=torch.float32) < 0.02))).to(dtype)
    r = randn(g, M, d, dtype=dtype) if residual else None
    if residual and M > 3:
        r[1] = 0
        r[2] *= 0
    gain = (1 + 0.2 * randn(g, d)).to(dtype)
    return x, r, gain


SHAPES = [(1, 1), (1, 128), (2, 8), (9, 7), (17, 96), (64, 768), (65, 1000), (33, 1001), (70, 1024), (5, 4096), (12, 11008), (9, 16384), (9, 16383)]


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,d", SHAPES)
def test_rmsnorm_quantize(M, d, dtype, residual):
    x, r, gain = norm_case(M, d, dtype, 11 * M + d, residual)
    eps = 1e-5
    codes, scales, h, y = B.rmsnorm_quantize(x, gain, residual=r, eps=eps, want_y=True)
    with np.errstate(all="ignore"):
        s = x.float().cpu().numpy()
        if residual:
            s = s + r.float().cpu().numpy()
        q, a, live, fine = np_codes(s * gain.float().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), q)
    assert (h is None) == (r is None)
    if residual:
        want = torch.from_numpy(s).cuda().to(dtype)
        assert torch.equal(torch.nan_to_num(h), torch.nan_to_num(want))
    # the sum of squares of the row of 1e30 passes the range of fp32: rstd is 0 there
    over = torch.from_numpy((s.astype(np.float64) ** 2).sum(axis=1) > 3.4e38).cuda()
    s64 = torch.from_numpy(s.astype(np.float64)).cuda()
    rstd = (s64.pow(2).mean(dim=1, keepdim=True) + eps).rsqrt()
    rstd[over] = 0
    ref = torch.from_numpy(np.where(live, a.astype(np.float64), np.where(fine, 0.0, np.nan))).cuda() * rstd[:, 0] / 127
    rel = (CHAIN / 2 + 8) * U            # rsqrt halves the sum's error
    check(scales, ref, ref.abs() * rel + 1e-44, "scales")
    yr = s64 * gain.double() * rstd
    ok = torch.from_numpy(fine).cuda() & ~over
    # below fp32's normal range s g and y are multiples of 2^-149: s g is off by up to 2^-150, which rstd multiplies, y by 2^-150 more
    check(y[ok], yr[ok], yr[ok].abs() * (HALF[dtype] + rel) + ((1e-40 if dtype == torch.bfloat16 else 2.0 ** -150) + 2.0 ** -150 * rstd[ok]), "y")
    again = B.rmsnorm_quantize(x, gain, residual=r, eps=eps)
    assert torch.equal(again[0], codes) and torch.equal(torch.nan_to_num(again[1]), torch.nan_to_num(scales)) and again[3] is None


@pytest.mark.parametrize("dtype", DTYPES)
def test_rmsnorm_quantize_layouts_and_in_place(dtype):
    x, r, gain = norm_case(40, 264, dtype, 3, True)
    want = B.rmsnorm_quantize(x, gain, residual=r, want_y=True)
    got = B.rmsnorm_quantize(offset(x, 1), offset(gain, 3), residual=offset(r, 2), want_y=True)
    assert torch.equal(got[0], want[0]) and torch.equal(torch.nan_to_num(got[2]), torch.nan_to_num(want[2]))
    for into in (0, 1):
        a, b = x.clone(), r.clone()
        got = B.rmsnorm_quantize(a, gain, residual=b, h=(a, b)[into])
        assert torch.equal(got[0], want[0]) and torch.equal(torch.nan_to_num((a, b)[into]), torch.nan_to_num(want[2]))
        assert torch.equal(torch.nan_to_num(got[1]), torch.nan_to_num(want[1]))


def norm_grad64(dy, h, g, res, eps):
    dy, h, g = dy.double(), h.double(), g.double()
    rstd = (h.pow(2).mean(dim=1, keepdim=True) + eps).rsqrt()
    w = dy * g
    c = (w * h).mean(dim=1, keepdim=True)
    dx = rstd * (w - h * rstd ** 2 * c)
    size = rstd * (w.abs() + h.abs() * rstd ** 2 * (w * h).abs().mean(dim=1, keepdim=True))
    if res is not None:
        dx = dx + res.double()
        size = size + res.double().abs()
    t = dy * h * rstd
    return dx, size, t.sum(dim=0), t.abs().sum(dim=0)


@pytest.mark.parametrize("want_dg", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,d", SHAPES + [(593, 64), (2500, 24), (1184, 1001)])
def test_rmsnorm_bwd(M, d, dtype, residual, want_dg):
    g = gen(M * 7 + d)
    h, dy = randn(g, M, d, dtype=dtype), randn(g, M, d, dtype=dtype)
    if M > 3:
        h[1] = 0
        dy[2] = 0
    gain = (1 + 0.2 * randn(g, d)).to(dtype)
    res = randn(g, M, d, dtype=dtype) if residual else None
    dx, dg = B.rmsnorm_bwd(dy, h, gain, resid=res, want_dg=want_dg)
    ref, size, rg, sg = norm_grad64(dy, h, gain, res, 1e-5)
    check(dx, ref, HALF[dtype] * ref.abs() + 2 * CHAIN * U * size + 1e-40, "dx")
    assert (dg is None) == (not want_dg)
    if want_dg:
        # a column's chain: rows of one block, then 8 threads adding the blocks' partial sums
        chain = -(-M // min(M, 592)) + 592 // 8 + 8 + CHAIN
        check(dg, rg, chain * U * sg + 1e-40, "dg")
        again = B.rmsnorm_bwd(dy, h, gain, resid=res, want_dg=True)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dg)
    # in place of an input, and without the other gradient: the same values
    a = dy.clone()
    assert torch.equal(B.rmsnorm_bwd(a, h, gain, resid=res, want_dg=want_dg, dx=a)[0], dx)
    if residual:
        a = res.clone()
        assert torch.equal(B.rmsnorm_bwd(dy, h, gain, resid=a, dx=a)[0], dx)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rmsnorm_bwd_layouts(dtype):
    g = gen(9)
    h, dy, res = (randn(g, 50, 136, dtype=dtype) for _ in range(3))
    gain = randn(g, 136, dtype=dtype)
    ref, size, rg, sg = norm_grad64(dy, h, gain, res, 1e-5)
    dx, dg = B.rmsnorm_bwd(offset(dy, 1), offset(h, 2), offset(gain, 1), resid=offset(res, 3), want_dg=True)
    check(dx, ref, HALF[dtype] * ref.abs() + 2 * CHAIN * U * size)
    check(dg, rg, (CHAIN + 100) * U * sg)


def test_rmsnorm_gradient_against_differences():
    """dx and dg against central differences of sum(y * up) in 64 bits, y the normalised row: step e of a smooth function is off by e^2
    times a third derivative (below 10 here), fp32 results by CHAIN units."""
    g = gen(21)
    M, d, e = 3, 40, 1e-4
    x, r, up = (randn(g, M, d) for _ in range(3))
    gain = 1 + 0.2 * randn(g, d)
    h = B.rmsnorm_quantize(x, gain, residual=r)[2]
    dx, dg = B.rmsnorm_bwd(up, h, gain, want_dg=True)

    def f(hh, gg):
        return (hh * (hh.pow(2).mean(dim=1, keepdim=True) + 1e-5).rsqrt() * gg * up.double()).sum()

    for (m, c) in [(0, 0), (1, 17), (2, 39)]:
        hp, hm = h.double().clone(), h.double().clone()
        hp[m, c] += e
        hm[m, c] -= e
        num = float((f(hp, gain.double()) - f(hm, gain.double())) / (2 * e))
        assert abs(num - float(dx[m, c])) <= 10 * e * e + 2 * CHAIN * U * 10
        gp, gm = gain.double().clone(), gain.double().clone()
        gp[c] += e
        gm[c] -= e
        num = float((f(h.double(), gp) - f(h.double(), gm)) / (2 * e))
        assert abs(num - float(dg[c])) <= 10 * e * e + 2 * CHAIN * U * 10


# ---- products ------------------------------------------------------------------------------
def codes_case(rows, cols, seed, pad=None, extreme=False):
    g = gen(seed)
    q = torch.randint(-127, 128, (rows, cols), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
    if extreme:
        q.fill_(127)
        q[::2] = -128
    if pad is None:
        t = B.empty_codes(rows, cols)
    else:
        t = torch.full((rows, pad), 99, dtype=torch.int8, device="cuda")[:, :cols]      # what lies behind a row must not count
    t.copy_(q)
    return t


def product64(x, sx, w, sw, bias, res):
    acc = x.double() @ w.double().t()
    scale = sx.double()[:, None] * (1 if sw is None else sw.double()[None, :])
    y = acc * scale
    size = y.abs()
    for t in (bias, res):
        if t is not None:
            y = y + t.double()
            size = size + t.double().abs()
    return y, size


def run_product(M, K, N, dtype, sw=True, bias=True, res=True, padx=None, padw=None, extreme=False, off=0):
    g = gen(M + 3 * K + 7 * N)
    x, w = codes_case(M, K, M + K, padx, extreme), codes_case(N, K, N + K, padw, extreme)
    sx = 0.01 + 0.02 * torch.rand(M, device="cuda", generator=g, dtype=torch.float32)
    if M > 2:
        sx[M // 2] = 0
    sw = 1e-3 * (0.5 + torch.rand(N, device="cuda", generator=g, dtype=torch.float32)) if sw else None
    b = randn(g, N, dtype=dtype) if bias else None
    r = randn(g, M, N, dtype=dtype) if res else None
    if off:
        b, r = (None if t is None else offset(t, off) for t in (b, r))
    y = torch.full((M * N + 64 + off,), 7.0, dtype=dtype, device="cuda")
    out = y[off:off + M * N].view(M, N)
    B.linear_i8(x, sx, w, sw, bias=b, residual=r, y=out)
    ref, size = product64(x, sx, w, sw, b, r)
    check(out, ref, HALF[dtype] * ref.abs() + 5 * U * size + 1e-40, (M, K, N))       # integer to float, two products, two additions
    assert (y[:off] == 7).all() and (y[off + M * N:] == 7).all()
    return x, sx, w, sw, b, r, out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", [
    (1, 1, 1), (1, 16, 8), (1, 4096, 4096), (2, 100, 30), (7, 128, 64), (16, 768, 2304), (33, 130, 72), (64, 4096, 1024), (100, 1000, 1000),
    (128, 128, 64), (129, 256, 65), (130, 2048, 264), (300, 384, 1000), (512, 1024, 1024), (777, 768, 2304), (1000, 11008, 256), (1665, 768, 2307),
    (2048, 1024, 4096), (4100, 1000, 1032), (5000, 64, 999)])
def test_linear_i8(M, K, N, dtype):
    run_product(M, K, N, dtype)
    run_product(M, K, N, dtype, sw=False, bias=False, res=False)
    assert B.library_status() == 0


@pytest.mark.parametrize("M,K,N", [(1, 65536, 16), (200, 65536, 128), (300, 65536, 256)])
def test_linear_i8_largest_sums(M, K, N):
    """Sums of 65536 products of the largest codes: 2^30, the range the 32-bit accumulator has to hold."""
    run_product(M, K, N, torch.float32, extreme=True, bias=False, res=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kw", [dict(padx=112, padw=112), dict(padx=101, padw=112), dict(padx=112, padw=105), dict(off=1), dict(off=2), dict(off=8),
                                dict(bias=False), dict(res=False), dict(sw=False)])
def test_linear_i8_layouts(kw, dtype):
    for M in (5, 150, 600):
        run_product(M, 100, 136, dtype, **kw)


def test_linear_i8_rows_are_independent_of_the_kernel():
    """The sums are exact, so a row's result does not depend on how many others there are."""
    x, sx, w, sw, b, _, y = run_product(1500, 768, 520, torch.bfloat16, res=False)
    for m in (1, 3, 130, 400, 1499):
        assert torch.equal(B.linear_i8(x[:m], sx[:m], w, sw, bias=b), y[:m])


def test_linear_i8_values_that_are_not_finite_stay_in_their_rows():
    x, sx, w, sw, b, r, y = run_product(300, 256, 264, torch.bfloat16)
    sx[7] = float("nan")
    r[200, 5] = float("inf")
    got = B.linear_i8(x, sx, w, sw, bias=b, residual=r)
    assert torch.isnan(got[7]).all() and torch.isinf(got[200, 5])
    keep = torch.ones(300, 264, dtype=torch.bool, device="cuda")
    keep[7] = False
    keep[200, 5] = False
    assert torch.equal(got[keep], y[keep])


def test_linear_i8_in_place_of_the_residual():
    for M, N in ((40, 136), (700, 264), (700, 263)):
        x, sx, w, sw, b, r, y = run_product(M, 512, N, torch.bfloat16)
        assert torch.equal(B.linear_i8(x, sx, w, sw, bias=b, residual=r, y=r), y)


# ---- loss ----------------------------------------------------------------------------------
def distill64(z, idx, t, labels, T, wc, wk, n=0):
    """Row losses, loss, gradient and the gradient's magnitude before cancellation."""
    z, t, idx = z.double(), t.double(), idx.long()
    M, V = z.shape
    take = torch.ones(M, dtype=torch.bool, device=z.device) if labels is None else (labels >= 0) & (labels < V)
    n = n or max(1, int(take.sum()))
    rows, grad, size = torch.zeros(M, dtype=torch.float64, device=z.device), torch.zeros_like(z), torch.zeros_like(z)
    for m in range(M):
        if not take[m]:
            continue
        ok = (idx[m] >= 0) & (idx[m] < V)
        j, e = idx[m][ok], t[m][ok] / T
        if len(j) and not bool((e == -float("inf")).all()) and wk != 0:
            q = torch.softmax(e, 0)
            lp = torch.log_softmax(z[m] / T, 0)
            live = q != 0
            rows[m] += wk * T * T * (q[live] * (q[live].log() - lp[j[live]])).sum()
            Q = torch.zeros(V, dtype=torch.float64, device=z.device).index_add_(0, j, q)
            grad[m] += wk * T * (lp.exp() - Q)
            size[m] += abs(wk) * T * (lp.exp() + Q)
        if wc != 0:
            lp = torch.log_softmax(z[m], 0)
            one = torch.zeros(V, dtype=torch.float64, device=z.device)
            one[int(labels[m])] = 1
            rows[m] -= wc * lp[int(labels[m])]
            grad[m] += wc * (lp.exp() - one)
            size[m] += abs(wc) * (lp.exp() + one)
    return rows, rows.sum() / n, grad / n, size / n


def distill_case(M, V, k, dtype, seed, labels=True):
    g = gen(seed)
    z = (2.5 * randn(g, M, V)).to(dtype)
    idx = torch.argsort(torch.rand(M, V, device="cuda", generator=g, dtype=torch.float32), dim=1)[:, :k].to(torch.int32).contiguous() if k <= V else \
        torch.randint(0, V, (M, k), device="cuda", generator=g, dtype=torch.int32)
    t = (4 + 2 * randn(g, M, k)).contiguous()
    y = torch.randint(0, V, (M,), device="cuda", generator=g, dtype=torch.int32) if labels else None
    if labels and M > 2:
        y[M // 2] = -100
        y[2] = V
    if k > 2:
        idx[::3, k // 2:] = -1
        idx[1 % M, 0] = V + 3
        idx[0, 1] = idx[0, 0]                       # one index twice
        if labels:
            idx[0, 0] = y[0]                        # the label among the entries
        t[0, 2] = -float("inf")
    if M > 5:
        idx[5] = -1                                 # no entry at all
        t[4] = -float("inf")                        # entries without weight
        z[3, :: 2] = torch.finfo(dtype).min         # a masked vocabulary
        z[3, int(idx[3, 0].clamp(min=0))] = 1.0
    return z, idx, t, y


def check_distill(z, idx, t, y, T, wc, wk, got, n=0):
    dtype = z.dtype
    loss, rows, dz = got
    V = z.shape[1]
    rr, rl, rg, size = distill64(z, idx, t, y, T, wc, wk, n)
    # exponents: two roundings of up to |z - max| / min(T, 1); sums: elements per thread plus trees; ex2 and the factors
    spread = float((z.double().clamp(min=-100).amax(dim=1) - z.double().clamp(min=-100).amin(dim=1)).max()) / min(T, 1.0)
    rel = (2 * spread + V / 128 + 64) * U
    check(dz, rg, HALF[dtype] * rg.abs() + rel * size + 1e-40, "dlogits")
    # a loss beyond the largest fp32 value (a student that gives finfo.min to what the teacher says) is rounded to infinity
    top = torch.finfo(torch.float32).max
    over = rr.abs() > top * (1 + U)
    assert torch.isinf(rows[over]).all()
    tol = rel * (rr.abs() + abs(wc) + abs(wk) * T * T * (10 + spread))
    check(rows[~over], rr[~over], tol[~over], "rows")
    if over.any():
        assert torch.isinf(loss)
    else:
        assert abs(float(loss) - float(rl)) <= float(tol.sum()) / (n or 1) + 1e-30


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,wc,wk", [(1.0, 0.5, 0.5), (2.0, 0.3, 0.7), (1.5, 0.0, 1.0), (4.0, 1.0, 1.0), (3.0, 0.5, 0.5), (0.7, 0.2, 1.0), (2.0, 1.0, 0.0)])
@pytest.mark.parametrize("M,V,k", [(1, 1, 1), (1, 50, 5), (7, 64, 64), (9, 1000, 8), (12, 1001, 33), (64, 1024, 256), (10, 32000, 20), (8, 50257, 64), (3, 30, 100)])
def test_distill_loss(M, V, k, dtype, T, wc, wk):
    z, idx, t, y = distill_case(M, V, k, dtype, M + V + k)
    check_distill(z, idx, t, y, T, wc, wk, B.distill_loss(z, idx, t, labels=y, temperature=T, ce_weight=wc, kd_weight=wk))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1.0, 2.0])
def test_distill_loss_without_labels(dtype, T):
    z, idx, t, _ = distill_case(11, 777, 16, dtype, 4, labels=False)
    check_distill(z, idx, t, None, T, 0.0, 1.0, B.distill_loss(z, idx, t, temperature=T))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,ld,by", [(1000, 1024, 0), (1001, 1008, 0), (50257, 50304, 0), (999, 1003, 0), (1000, 1000, 3), (64, 64, 1)])
def test_distill_loss_layouts_and_in_place(V, ld, by, dtype):
    z, idx, t, y = distill_case(9, V, 12, dtype, V)
    wide = torch.full((9, ld), 50.0, dtype=dtype, device="cuda")
    wide[:, :V] = z
    wide = offset(wide, by)
    got = B.distill_loss(wide, idx, t, labels=y, temperature=2.0, ce_weight=0.5, kd_weight=0.5, vocab=V)
    assert (got[2][:, V:] == 0).all()
    check_distill(z, idx, t, y, 2.0, 0.5, 0.5, (got[0], got[1], got[2][:, :V]))
    same = B.distill_loss(wide, idx, t, labels=y, temperature=2.0, ce_weight=0.5, kd_weight=0.5, vocab=V, dlogits=wide)
    assert same[2].data_ptr() == wide.data_ptr() and torch.equal(wide, got[2]) and torch.equal(same[0], got[0]) and torch.equal(same[1], got[1])


@pytest.mark.parametrize("dtype,V,ld", [(torch.bfloat16, 131072, 131072), (torch.bfloat16, 128001, 128001), (torch.float32, 60000, 60008), (torch.float32, 65537, 65537),
                                        (torch.bfloat16, 113001, 113001), (torch.float32, 56001, 56001)])
def test_distill_loss_of_large_vocabularies(dtype, V, ld):
    """Rows about as wide as shared memory, and wider."""
    z, idx, t, y = distill_case(7, V, 40, dtype, V)
    wide = torch.full((7, ld), 50.0, dtype=dtype, device="cuda")
    wide[:, :V] = z
    for T in (1.0, 2.0, 1.5):
        got = B.distill_loss(wide, idx, t, labels=y, temperature=T, ce_weight=0.5, kd_weight=0.5, vocab=V)
        assert (got[2][:, V:] == 0).all()
        check_distill(z, idx, t, y, T, 0.5, 0.5, (got[0], got[1], got[2][:, :V]))
        same = wide.clone()
        again = B.distill_loss(same, idx, t, labels=y, temperature=T, ce_weight=0.5, kd_weight=0.5, vocab=V, dlogits=same)
        assert torch.equal(same, got[2]) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1.0, 1.3, 2.0, 3.0, 4.0])
@pytest.mark.parametrize("V", [64, 1003, 20000])
def test_distill_loss_of_masked_and_broken_logits_at_every_column(V, T, dtype):
    """-inf logits have probability 0 exactly, wherever in a vector they stand; NaN and inf reach their own row and no other."""
    z, idx, t, y = distill_case(40, V, 6, dtype, V + 1)
    z, idx, t = z.clamp(min=-20), idx.clamp(0, V - 1), torch.zeros_like(t)
    y[:] = 5
    dead = torch.zeros(40, V, dtype=torch.bool, device="cuda")
    for m in range(16):
        dead[m, m::16] = True
    for m in range(16, 20):
        dead[m, m - 16::2] = True
    keep = torch.zeros_like(dead).scatter_(1, idx.long(), True)
    keep[:, 5] = True
    dead &= ~keep
    z[dead] = -float("inf")
    for m in range(20, 28):
        z[m, m] = float("nan")
    for m in range(28, 36):
        z[m, m] = float("inf")
    _, rows, dz = B.distill_loss(z, idx, t, labels=y, temperature=T, ce_weight=0.5, kd_weight=0.5)
    assert (dz[dead] == 0).all()
    broken = torch.zeros(40, dtype=torch.bool, device="cuda")
    broken[20:36] = True
    assert torch.isnan(rows[broken]).all() and torch.isnan(dz[broken]).any(dim=1).all()
    ok = ~broken
    zz = z[ok].double().clamp(min=-1e30)
    # rows with whatever is masked left at a logit of no weight: 64-bit formulas, tolerance as above with the finite logits' spread
    rr, _, rg, size = distill64(zz, idx[ok], t[ok], y[ok], T, 0.5, 0.5, 40)
    rel = (2 * 40 / min(T, 1.0) + V / 128 + 64) * U
    check(dz[ok], rg, HALF[dtype] * rg.abs() + rel * size + 1e-40, "dlogits")
    check(rows[ok], rr, rel * (rr.abs() + 0.5 + 0.5 * T * T * 50), "rows")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 3, 8, 9, 15, 255, 256, 1023, 1024, 1025, 1031, 2047, 2048, 2056, 2063, 4103])
def test_distill_loss_around_the_widths_that_change_the_kernel(V, dtype):
    """Widths around those that a warp, its variants and a block hold, rows at every place of a vector, more rows than a block's eight."""
    z, idx, t, y = distill_case(13, V, min(V, 9), dtype, V + 3)
    for T in (1.0, 2.0, 1.3):
        for by in (0, 1):
            zz = offset(z, by)
            got = B.distill_loss(zz, idx, t, labels=y, temperature=T, ce_weight=0.4, kd_weight=0.6)
            check_distill(z, idx, t, y, T, 0.4, 0.6, got)
            same = offset(z, by)
            B.distill_loss(same, idx, t, labels=y, temperature=T, ce_weight=0.4, kd_weight=0.6, dlogits=same)
            assert by and V > 1 or torch.equal(same, got[2])
            check_distill(z, idx, t, y, T, 0.4, 0.6, (got[0], got[1], same))


@pytest.mark.parametrize("M", [300, 5000])
def test_distill_loss_of_many_rows(M):
    """More rows than blocks, and than a block looks at together; many that take no part, first and last among them."""
    g = gen(M)
    z = (2 * randn(g, M, 201)).to(torch.bfloat16)
    idx = torch.randint(-3, 201, (M, 6), device="cuda", generator=g, dtype=torch.int32)
    t = randn(g, M, 6)
    y = torch.randint(0, 201, (M,), device="cuda", generator=g, dtype=torch.int32)
    y[torch.rand(M, device="cuda", generator=g, dtype=torch.float32) < 0.6] = -1
    y[0] = y[-1] = -1
    check_distill(z, idx, t, y, 2.0, 0.5, 0.5, B.distill_loss(z, idx, t, labels=y, temperature=2.0, ce_weight=0.5, kd_weight=0.5))
    y[:] = -1
    y[M // 2] = 200
    check_distill(z, idx, t, y, 1.7, 0.5, 0.5, B.distill_loss(z, idx, t, labels=y, temperature=1.7, ce_weight=0.5, kd_weight=0.5))


def test_distill_loss_normalizer_and_no_rows():
    z, idx, t, y = distill_case(9, 500, 12, torch.float32, 6)
    check_distill(z, idx, t, y, 2.0, 0.5, 0.5, B.distill_loss(z, idx, t, labels=y, temperature=2.0, ce_weight=0.5, kd_weight=0.5, normalizer=64), n=64)
    y[:] = -100
    loss, rows, dz = B.distill_loss(z, idx, t, labels=y, temperature=2.0, ce_weight=0.5, kd_weight=0.5)
    assert float(loss) == 0 and not rows.any() and not dz.any()


def test_distill_loss_values_that_are_not_finite_stay_in_their_rows():
    z, idx, t, y = distill_case(9, 500, 12, torch.float32, 8)
    y[:] = 3
    want = B.distill_loss(z, idx, t, labels=y, temperature=2.0, ce_weight=0.5, kd_weight=0.5)
    z2, t2 = z.clone(), t.clone()
    z2[0, 499] = float("nan")
    z2[1, 0] = float("inf")
    z2[2] = -float("inf")
    t2[8, 0], idx[8, 0] = float("nan"), 7
    z2[7, idx[7, 0]] = -float("inf")                 # the student rules out what the teacher says: an infinite loss, a finite gradient
    loss, rows, dz = B.distill_loss(z2, idx, t2, labels=y, temperature=2.0, ce_weight=0.5, kd_weight=0.5)
    for m in (0, 1, 2):
        assert torch.isnan(rows[m]) and torch.isnan(dz[m]).all()
    assert torch.isnan(rows[8]) and torch.isnan(loss)
    assert torch.isinf(rows[7]) and torch.isfinite(dz[7]).all()
    for m in (3, 4, 5, 6):
        assert torch.equal(dz[m], want[2][m]) and torch.equal(rows[m], want[1][m])


def test_distill_gradient_against_differences():
    z, idx, t, y = distill_case(3, 40, 6, torch.float32, 2)
    loss, rows, dz = B.distill_loss(z, idx, t, labels=y, temperature=1.7, ce_weight=0.4, kd_weight=0.6)
    e = 1e-4
    for m, v in [(0, int(y[0])), (0, 5), (0, int(idx[0, 0])), (0, 39)]:
        hi, lo = z.double().clone(), z.double().clone()
        hi[m, v] += e
        lo[m, v] -= e
        num = float((distill64(hi, idx, t, y, 1.7, 0.4, 0.6)[1] - distill64(lo, idx, t, y, 1.7, 0.4, 0.6)[1]) / (2 * e))
        assert abs(num - float(dz[m, v])) <= e * e + 200 * U


# ---- together, streams, graphs ---------------------------------------------------------------
def block_input_projection(x, r, gain, wq, sw, wqt, A, Bm, alpha, up):
    """A training step's use of them: norm and codes, the 8-bit projection with the rank-r term as its residual, and back.  Returns y, the
    gradient with respect to the residual stream, and the adapter gradients."""
    codes, scales, h, u = B.rmsnorm_quantize(x, gain, residual=r, want_y=True)
    M, d = x.shape
    r_ = A.shape[0]
    s = alpha / r_
    low = u @ A.t()                                         # rank-r projection
    y = B.linear_i8(codes, scales, wq, sw, residual=(s * (low @ Bm.t())).contiguous())
    gq, gs = B.quantize_rows(up, col_scale=sw)
    dlow = s * (up @ Bm)
    du = B.linear_i8(gq, gs, wqt, residual=(dlow @ A).contiguous())
    dx, dg = B.rmsnorm_bwd(du, h, gain, resid=up[:, :d].contiguous(), want_dg=True)
    return y, dx, dg, dlow.t() @ u, s * up.t() @ low


def projection_case(M, d, N, seed=0):
    g = gen(seed)
    bf = torch.bfloat16
    x, r = randn(g, M, d, dtype=bf), randn(g, M, d, dtype=bf)
    gain = (1 + 0.1 * randn(g, d)).to(bf)
    W = (0.02 * randn(g, N, d)).to(bf)
    wq, sw = B.quantize_rows(W)
    wqt = B.empty_codes(d, N)
    wqt.copy_(wq.t())
    A, Bm = (0.02 * randn(g, 16, d)).to(bf), (0.02 * randn(g, N, 16)).to(bf)
    up = (1e-2 * randn(g, M, N)).to(bf)
    return (x, r, gain, wq, sw, wqt, A, Bm, 32.0, up), W


@pytest.mark.parametrize("M,d,N", [(1, 256, 768), (333, 264, 1000), (1024, 1024, 2048)])
def test_projection_and_its_gradients_together(M, d, N):
    case, W = projection_case(M, d, N)
    x, r, gain, wq, sw, wqt, A, Bm, alpha, up = case
    y, dx, dg, dA, dB = block_input_projection(*case)
    s = alpha / 16
    h = (x.double() + r.double()).requires_grad_()
    gd, Ad, Bd = gain.double().requires_grad_(), A.double().requires_grad_(), Bm.double().requires_grad_()
    u = h * (h.pow(2).mean(dim=1, keepdim=True) + 1e-5).rsqrt() * gd
    ref = u @ W.double().t() + s * (u @ Ad.t()) @ Bd.t()
    (ref * up.double()).sum().backward()
    want = [ref.detach(), h.grad + up[:, :d].double(), gd.grad, Ad.grad, Bd.grad]
    # codes are off by half a step of a row's maximum, at most 5.5 standard deviations here: rms error 5.5 / 127 / sqrt(12) = 1.25 % of
    # a row for each of the two factors of a product; bf16 roundings 0.2-0.4 % each on top: 3 % in the 2-norm
    for name, a, b in zip(("y", "dx", "dg", "dA", "dB"), (y, dx, dg, dA, dB), want):
        err = float((a.double() - b).norm() / b.norm())
        assert err <= 0.03, (name, err)


def test_two_streams_at_once_and_a_captured_step():
    case, _ = projection_case(300, 512, 768, 1)
    other, _ = projection_case(300, 512, 768, 2)
    want, want2 = block_input_projection(*case), block_input_projection(*other)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(5):
        with torch.cuda.stream(a):
            g1 = block_input_projection(*case)
        with torch.cuda.stream(b):
            g2 = block_input_projection(*other)
        got.append((g1, g2))
    torch.cuda.synchronize()
    for g1, g2 in got:
        for i in range(3):
            assert torch.equal(g1[i], want[i]) and torch.equal(g2[i], want2[i])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = block_input_projection(*case)
    for t, src in zip((case[0], case[1], case[9]), (other[0], other[1], other[9])):
        t.copy_(src)
    graph.replay()
    torch.cuda.synchronize()
    again = block_input_projection(*case)
    for i in range(3):
        assert torch.equal(held[i], again[i])
    assert B.library_status() == 0


def test_captured_loss():
    z, idx, t, y = distill_case(40, 1001, 12, torch.bfloat16, 8)
    kw = dict(temperature=2.0, ce_weight=0.5, kd_weight=0.5)
    B.distill_loss(z, idx, t, labels=y, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = B.distill_loss(z, idx, t, labels=y, **kw)
    z.copy_(z.flip(0))
    y[7] = -1
    graph.replay()
    for a, b in zip(held, B.distill_loss(z, idx, t, labels=y, **kw)):
        assert torch.equal(a, b)


def test_refusals_on_the_device():
    x = torch.zeros(8, 64, device="cuda", dtype=torch.bfloat16)
    c, s = B.quantize_rows(x)
    for f in (lambda: B.quantize_rows(x.half()), lambda: B.quantize_rows(x.t()), lambda: B.quantize_rows(x, col_scale=s[:3]),
              lambda: B.linear_i8(c, s, c[:, :32], s), lambda: B.linear_i8(c.t(), s, c, s), lambda: B.linear_i8(x, s, c, s),
              lambda: B.linear_i8(c, s[:4], c, s), lambda: B.linear_i8(c, s, c, s, dtype=torch.float16), lambda: B.linear_i8(c[:0], s[:0], c, s),
              lambda: B.linear_i8(c, s, c, s, residual=x[:, :8].float()), lambda: B.rmsnorm_quantize(x, x[0, :8]), lambda: B.rmsnorm_quantize(x, x[0].float()),
              lambda: B.rmsnorm_bwd(x, x.float(), x[0]), lambda: B.distill_loss(x, c, x.float()),
              lambda: B.distill_loss(x, torch.zeros(8, 4, dtype=torch.int64, device="cuda"), x[:, :4].float()),
              lambda: B.distill_loss(x, torch.zeros(8, 4, dtype=torch.int32, device="cuda"), torch.zeros(8, 4, device="cuda", dtype=torch.float32), ce_weight=1.0),
              lambda: B.distill_loss(x, torch.zeros(8, 4, dtype=torch.int32, device="cuda"), torch.zeros(8, 4, device="cuda", dtype=torch.float32), temperature=0.0)):
        with pytest.raises(B.SplitLoraError) as e:
            f()
        assert e.value.code == -1


def test_element_offsets_beyond_32_bits():
    """More than 2^31 elements: the last rows come out as they do by themselves, bit for bit, and the first rows with them."""
    def ends(n, k=40):
        return [slice(0, k), slice(n - k, n)]

    g = gen(5)
    M, d = 33001, 65536
    x = torch.empty(M, d, dtype=torch.bfloat16, device="cuda")
    for part in ends(M):
        x[part] = randn(g, 40, d).to(torch.bfloat16)
    codes, scales = B.quantize_rows(x)
    back = B.dequantize_rows(codes, scales, out=x.clone())
    for part in ends(M):
        c, s = B.quantize_rows(x[part])
        assert torch.equal(codes[part], c) and torch.equal(scales[part], s) and torch.equal(back[part], B.dequantize_rows(c, s))
    del codes, scales, back, x
    M, d = 131300, 16383
    x = torch.zeros(M, d, dtype=torch.bfloat16, device="cuda")
    r = torch.zeros_like(x)
    gain = randn(g, d).to(torch.bfloat16)
    for part in ends(M):
        x[part] = randn(g, 40, d).to(torch.bfloat16)
        r[part] = randn(g, 40, d).to(torch.bfloat16)
    codes, scales, h, y = B.rmsnorm_quantize(x, gain, residual=r, want_y=True)
    dx, _ = B.rmsnorm_bwd(y, h, gain, resid=x)
    dx2, dg = B.rmsnorm_bwd(y, h, gain, resid=x, want_dg=True)
    assert torch.equal(dx, dx2)
    for part in ends(M):
        # (the rows where they lie: the order of a row's sum follows its place in the 16-byte vectors)
        c, s, h1, y1 = B.rmsnorm_quantize(x[part], gain, residual=r[part], want_y=True)
        assert torch.equal(codes[part], c) and torch.equal(scales[part], s) and torch.equal(h[part], h1) and torch.equal(y[part], y1)
        assert torch.equal(dx[part], B.rmsnorm_bwd(y[part], h[part], gain, resid=x[part])[0])
    del codes, scales, h, y, dx, dx2, r, x
    M, K, N = 70001, 64, 32768
    a = torch.randint(-127, 128, (M, K), device="cuda", generator=g, dtype=torch.int8)
    w = torch.randint(-127, 128, (N, K), device="cuda", generator=g, dtype=torch.int8)
    sa, sw = randn(g, M).abs(), randn(g, N).abs()
    for dtype in (torch.bfloat16, torch.float32):
        res = torch.ones(M, N, dtype=dtype, device="cuda")
        out = B.linear_i8(a, sa, w, sw, residual=res, y=res)
        for part in ends(M):
            assert torch.equal(out[part], B.linear_i8(a[part], sa[part], w, sw, residual=torch.ones(40, N, dtype=dtype, device="cuda"), dtype=dtype))
        del res, out
    M, V = 42801, 50257
    z = torch.zeros(M, V, dtype=torch.bfloat16, device="cuda")
    idx = torch.randint(0, V, (M, 8), device="cuda", generator=g, dtype=torch.int32)
    t, lab = randn(g, M, 8), torch.randint(0, V, (M,), device="cuda", generator=g, dtype=torch.int32)
    for part in ends(M):
        z[part] = (2 * randn(g, 40, V)).to(torch.bfloat16)
    want = [B.distill_loss(z[part].clone(), idx[part], t[part], labels=lab[part], temperature=2.0, ce_weight=0.5, kd_weight=0.5, normalizer=M) for part in ends(M)]
    _, rows, dz = B.distill_loss(z, idx, t, labels=lab, temperature=2.0, ce_weight=0.5, kd_weight=0.5, dlogits=z)
    for part, (_, rows1, dz1) in zip(ends(M), want):
        assert torch.equal(rows[part], rows1) and torch.equal(dz[part], dz1)
