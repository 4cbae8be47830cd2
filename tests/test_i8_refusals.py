"""Arguments that the operators for adapters over 8-bit frozen weights refuse, through the C ABI, before anything is launched.  Every call
here fails, so the made-up addresses are never read: no GPU needed."""
import ctypes as C

import pytest

from paper_2407_00952_b200 import binding as B

P = 1 << 20             # an aligned, non-null address
ARG, ALIGN, WORKSPACE = -1, -2, -5
F32, BF16 = B.DTYPE_FP32, B.DTYPE_BF16


def call(name, *args):
    def c(a):
        return a if isinstance(a, C._SimpleCData) else C.c_void_p(0) if a is None else a
    return getattr(B.load(), name)(*[c(a) for a in args])


def p(v):
    return C.c_void_p(v)


def i64(v):
    return C.c_int64(v)


def quantize(dtype=BF16, x=P, f=0, M=4, d=64, codes=P, ld=64, scales=P):
    return call("splitlora_quantize_rows", dtype, p(x), p(f), i64(M), d, p(codes), i64(ld), p(scales), None)


def dequantize(dtype=BF16, codes=P, ld=64, scales=P, M=4, d=64, y=P):
    return call("splitlora_dequantize_rows", dtype, p(codes), i64(ld), p(scales), i64(M), d, p(y), None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), ARG), (dict(M=0), ARG), (dict(M=-1), ARG), (dict(M=1 << 31), ARG), (dict(d=0), ARG), (dict(d=65537, ld=65552), ARG),
    (dict(ld=63), ARG), (dict(codes=0), ARG), (dict(scales=0), ARG), (dict(scales=P + 2), ALIGN)])
def test_row_codec_refuses(bad, code):
    assert quantize(**bad) == code
    assert dequantize(**bad) == code


def test_row_codec_refuses_its_own():
    assert quantize(x=0) == ARG and quantize(x=P + 1) == ALIGN and quantize(dtype=F32, x=P + 2) == ALIGN and quantize(f=P + 2) == ALIGN
    assert dequantize(y=0) == ARG and dequantize(y=P + 1) == ALIGN


def norm(dtype=BF16, x=P, resid=0, g=P, eps=1e-5, M=4, d=64, h=0, y=0, codes=P, ld=64, scales=P):
    return call("splitlora_rmsnorm_quantize", dtype, p(x), p(resid), p(g), C.c_float(eps), i64(M), d, p(h), p(y), p(codes), i64(ld), p(scales), None)


def norm_bwd(dtype=BF16, dy=P, h=P, g=P, resid=0, eps=1e-5, M=4, d=64, dx=P, dg=0, ws=0, ws_bytes=0):
    return call("splitlora_rmsnorm_bwd", dtype, p(dy), p(h), p(g), p(resid), C.c_float(eps), i64(M), d, p(dx), p(dg), p(ws), C.c_size_t(ws_bytes), None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=-1), ARG), (dict(g=0), ARG), (dict(M=0), ARG), (dict(d=0), ARG), (dict(d=16385, ), ARG), (dict(eps=-1e-5), ARG),
    (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(h=P + 1), ALIGN), (dict(resid=P + 1), ALIGN)])
def test_norm_refuses(bad, code):
    assert norm(**{**bad, **({"ld": 16400} if bad.get("d", 0) > 64 else {})}) == code
    assert norm_bwd(**bad) == code


def test_norm_refuses_its_own():
    assert norm(x=0) == ARG and norm(codes=0) == ARG and norm(scales=0) == ARG and norm(ld=60) == ARG and norm(y=P + 1) == ALIGN
    assert norm_bwd(dy=0) == ARG and norm_bwd(h=0) == ARG and norm_bwd(dx=0) == ARG
    n = C.c_size_t(0)
    assert call("splitlora_rmsnorm_bwd_workspace_bytes", i64(100), 64, C.byref(n)) == 0 and n.value == 100 * 64 * 4
    assert call("splitlora_rmsnorm_bwd_workspace_bytes", i64(1 << 30), 16384, C.byref(n)) == 0 and n.value < 64 << 20
    assert call("splitlora_rmsnorm_bwd_workspace_bytes", i64(0), 64, C.byref(n)) == ARG
    assert norm_bwd(dg=P) == WORKSPACE and norm_bwd(dg=P, ws=P, ws_bytes=4 * 64 * 4 - 1) == WORKSPACE
    assert norm_bwd(dg=P, ws=P + 4, ws_bytes=1 << 20) == ALIGN


def linear(dtype=BF16, x=P, ldx=64, sx=P, W=P, ldw=64, sw=0, bias=0, resid=0, M=4, K=64, N=32, y=P):
    return call("splitlora_linear_i8", dtype, p(x), i64(ldx), p(sx), p(W), i64(ldw), p(sw), p(bias), p(resid), M, K, N, p(y), None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), ARG), (dict(x=0), ARG), (dict(sx=0), ARG), (dict(W=0), ARG), (dict(y=0), ARG), (dict(M=0), ARG), (dict(K=0), ARG), (dict(N=0), ARG),
    (dict(K=65537, ldx=65552, ldw=65552), ARG), (dict(ldx=63), ARG), (dict(ldw=63), ARG), (dict(M=2147483647, N=2147483647), ARG),
    (dict(sx=P + 1), ALIGN), (dict(sw=P + 2), ALIGN), (dict(bias=P + 1), ALIGN), (dict(resid=P + 1), ALIGN), (dict(y=P + 1), ALIGN)])
def test_linear_refuses(bad, code):
    assert linear(**bad) == code


def distill(dtype=BF16, z=P, ld=64, labels=P, idx=P, t=P, M=4, V=50, k=8, T=2.0, wc=0.5, wk=0.5, norm=0, dz=2 * P, ldg=64, rows=P, loss=P, n=P):
    return call("splitlora_distill_loss", dtype, p(z), i64(ld), p(labels), p(idx), p(t), M, V, k, C.c_float(T), C.c_float(wc), C.c_float(wk), i64(norm),
                p(dz), i64(ldg), p(rows), p(loss), p(n), None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), ARG), (dict(z=0), ARG), (dict(idx=0), ARG), (dict(t=0), ARG), (dict(dz=0), ARG), (dict(rows=0), ARG), (dict(loss=0), ARG), (dict(n=0), ARG),
    (dict(M=0), ARG), (dict(V=0), ARG), (dict(k=0), ARG), (dict(k=257), ARG), (dict(ld=49), ARG), (dict(ldg=49), ARG), (dict(norm=-1), ARG),
    (dict(norm=1 << 31), ARG), (dict(T=0.0), ARG), (dict(T=-1.0), ARG), (dict(T=float("nan")), ARG), (dict(T=1e4), ARG), (dict(wc=float("inf")), ARG),
    (dict(wk=float("nan")), ARG), (dict(labels=0), ARG), (dict(dz=P, ldg=72), ARG), (dict(z=P + 1), ALIGN), (dict(dz=P + 1), ALIGN), (dict(labels=P + 2), ALIGN),
    (dict(idx=P + 2), ALIGN), (dict(rows=P + 1), ALIGN)])
def test_distill_refuses(bad, code):
    assert distill(**bad) == code


@pytest.mark.parametrize("bad", [dict(M=2147483647, K=1, N=1), dict(M=5, K=1, N=2147483647), dict(M=(1 << 30) + 1, N=8), dict(M=8, N=(1 << 30) + 1)])
def test_linear_refuses_sizes_whose_tiles_pass_32_bits(bad):
    assert linear(**bad) == ARG


@pytest.mark.parametrize("bad", [dict(M=2147483647, V=1, ld=1, ldg=1), dict(M=(1 << 30) + 1), dict(M=1, V=(1 << 30) + 1, ld=1 << 31, ldg=1 << 31),
                                 dict(M=1, ldg=(1 << 30) + 1), dict(M=1, ldg=1 << 33), dict(M=1, ld=1 << 33)])
def test_distill_refuses_sizes_whose_indexes_pass_32_bits(bad):
    assert distill(**bad) == ARG


def test_binding_refuses_tensors_off_the_device():
    import torch
    if torch.cuda.is_available():
        x = torch.zeros(4, 64, dtype=torch.float32)                     # on the host
        for f in (lambda: B.quantize_rows(x), lambda: B.rmsnorm_quantize(x, x[0]), lambda: B.rmsnorm_bwd(x, x, x[0])):
            with pytest.raises(B.SplitLoraError) as e:
                f()
            assert e.value.code == ARG
    with pytest.raises(B.SplitLoraError):
        B.quantize_rows(torch.zeros(4, 64, dtype=torch.float64))
    with pytest.raises(B.SplitLoraError):
        B.quantize_rows(torch.zeros(64, dtype=torch.float32))
