"""Sizes that a C int does not hold: refused by the binding, where ctypes would cut them to their low 32 bits and the call would answer for a
few rows or columns only.  Stand-in tensors without memory and a stand-in library: no GPU needed."""
import types

import pytest
import torch

from paper_2407_00952_b200 import binding as B

BIG = (1 << 32) + 64
BF16, F32, I8, I32 = torch.bfloat16, torch.float32, torch.int8, torch.int32


def m(*shape, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.fixture
def calls(monkeypatch):
    """Calls that reach the library.  A meta tensor's device has the number -1."""
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: made.append(name) or 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(B, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(B, "load", lambda: Library())
    return made


def product(M, K, N):
    return lambda: B.linear_i8(m(M, K, dtype=I8), m(M, dtype=F32), m(N, K, dtype=I8), m(N, dtype=F32), y=m(M, N))


def loss(M, V, k, vocab=None, normalizer=0):
    # the row losses are made by the call: only what is refused before that, or small, can run without a device
    return lambda: B.distill_loss(m(M, V), m(M, k, dtype=I32), m(M, k, dtype=F32), vocab=vocab, normalizer=normalizer, dlogits=m(M, V))


def norm(M, d):
    return lambda: B.rmsnorm_quantize(m(M, d), m(d), codes=m(M, d, dtype=I8), scales=m(M, dtype=F32))


def norm_bwd(M, d):
    return lambda: B.rmsnorm_bwd(m(M, d), m(M, d), m(d), dx=m(M, d))


def codec(M, d):
    return lambda: B.quantize_rows(m(M, d), codes=m(M, d, dtype=I8), scales=m(M, dtype=F32))


def codec_back(M, d):
    return lambda: B.dequantize_rows(m(M, d, dtype=I8), m(M, dtype=F32), out=m(M, d))


@pytest.mark.parametrize("f", [
    product(BIG, 1, 8), product(4, 1, BIG), product(1, BIG, 1), product(1 << 31, 1, 1), loss(BIG, 1, 1), loss(1, BIG, 1), loss(1, 8, BIG), loss(4, 64, 2, vocab=BIG),
    loss(4, 64, 2, vocab=-BIG), loss(4, 64, 2, normalizer=1 << 64), loss(4, 64, 2, normalizer=1 << 31), norm(1, BIG), norm_bwd(1, BIG), codec(1, BIG),
    codec_back(1, BIG)])
def test_sizes_past_32_bits_are_refused(f, calls):
    with pytest.raises(B.SplitLoraError) as e:
        f()
    assert e.value.code == B.ERR_ARG and not calls


@pytest.mark.parametrize("f", [product(4, 16, 8), norm(4, 64), norm_bwd(4, 64), codec(4, 64), codec_back(4, 64), codec(BIG, 1), norm(BIG, 1)])
def test_others_reach_the_library(f, calls):
    """(rows of the codec and the norms are counted in 64 bits)"""
    f()
    assert len(calls) == 1


def test_a_teacher_of_too_many_entries(monkeypatch):
    e = B.SplitLoRA.__new__(B.SplitLoRA)
    e.ctx = None
    e.cfg = types.SimpleNamespace(n_clients=1, batch_per_client=1, seq=1)
    e.workspace = types.SimpleNamespace(device=torch.device("meta"))
    e.lib = types.SimpleNamespace(splitlora_set_teacher=lambda *a: pytest.fail("reached the library"))
    monkeypatch.setattr(B, "_ptr", lambda t: 0)
    with pytest.raises(B.SplitLoraError) as err:
        e.set_teacher(m(1, 1, 1, BIG, dtype=I32), m(1, 1, 1, BIG, dtype=F32))
    assert err.value.code == B.ERR_ARG
