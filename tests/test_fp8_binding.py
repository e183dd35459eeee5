"""Sizes that the C ABI's ints do not hold are refused by the 8-bit calls' binding (ctypes would drop their upper bits).  No GPU
needed: tensors of these sizes are stood in for by their shapes."""
import types

import pytest
import torch

import paper_2508_17588_b200 as H
from paper_2508_17588_b200 import binding as Bd

BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
WRAP = 1 << 32


class Shape:
    """What the binding looks at of a tensor on GPU 0: contiguous, or with a row stride of its own."""
    device = "cuda:0"

    def __init__(self, dtype, *shape, row_stride=None):
        self.dtype, self.shape = dtype, torch.Size(shape)
        self.strides = [1] * len(shape)
        for i in range(len(shape) - 2, -1, -1):
            self.strides[i] = self.strides[i + 1] * shape[i + 1]
        if row_stride is not None:
            self.strides[0] = row_stride

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return tuple(self.strides) if i is None else self.strides[i]

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def calls(monkeypatch):
    """The calls that reach the library, which is stood in for."""
    made = []
    names = ("hero_quantize_fp8", "hero_gather_ln_modulate_fp8", "hero_rms_norm", "hero_rms_norm_fp8", "hero_gemm_fp8", "hero_plan_fp8_gemm")
    lib = types.SimpleNamespace(hero_strerror=lambda code: b"", **{n: lambda *a, n=n: made.append((n, a)) or 0 for n in names})
    monkeypatch.setattr(Bd, "load", lambda: lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    return made


def quantize(rows=8, cols=64, block_rows=1):
    scales = (rows if block_rows == 1 else Bd._blocks(rows), Bd._blocks(cols))
    H.hero_quantize_fp8(Shape(BF16, rows, cols), Shape(F8, rows, cols), Shape(F32, *scales), block_rows)


def rms(rows=8, D=64):
    H.hero_rms_norm(Shape(BF16, rows, D), None, None, None, Shape(BF16, rows, D))


def rms8(rows=8, D=64):
    H.hero_rms_norm_fp8(Shape(BF16, rows, D), None, None, None, Shape(F8, rows, D), Shape(F32, rows, Bd._blocks(D)))


def gather(B=2, N=8, D=64, n_sel=4, ld=128):
    H.hero_gather_ln_modulate_fp8(Shape(BF16, B, N, D), None, Shape(torch.int32, n_sel), Shape(F32, B, D, row_stride=ld),
                                  Shape(F32, B, D, row_stride=ld), Shape(F8, B, n_sel, D), Shape(F32, B, n_sel, Bd._blocks(D)))


def gemm(M=8, N=64, K=64, act=0):
    kb = Bd._blocks(K)
    H.hero_gemm_fp8(Shape(F8, M, K), Shape(F32, M, kb), Shape(F8, N, K), Shape(F32, Bd._blocks(N), kb), None, Shape(BF16, M, N), act=act)


ORDINARY = [quantize, rms, rms8, gather, gemm]


@pytest.mark.parametrize("call", ORDINARY)
def test_ordinary_sizes_reach_the_library(calls, call):
    call()
    assert len(calls) == 1


@pytest.mark.parametrize("call,change", [
    (quantize, dict(rows=WRAP + 5)), (quantize, dict(rows=WRAP + 5, block_rows=128)), (quantize, dict(cols=WRAP + 16)),
    (quantize, dict(rows=1 << 31)), (quantize, dict(block_rows=WRAP + 1)), (quantize, dict(block_rows=1 - WRAP)),
    (rms, dict(rows=WRAP + 5)), (rms, dict(D=WRAP + 64)), (rms8, dict(rows=WRAP + 5)), (rms8, dict(D=WRAP + 64)),
    (gather, dict(B=WRAP + 2)), (gather, dict(N=WRAP + 8)), (gather, dict(D=WRAP + 64, ld=WRAP + 64)), (gather, dict(N=WRAP + 8, n_sel=WRAP + 4)),
    (gather, dict(ld=WRAP + 128)), (gather, dict(ld=1 << 31)),
    (gemm, dict(M=WRAP + 5)), (gemm, dict(N=WRAP + 64)), (gemm, dict(K=WRAP + 64)), (gemm, dict(M=1 << 31)), (gemm, dict(act=WRAP + 1))])
def test_more_than_an_int_holds(calls, call, change):
    with pytest.raises(H.HeroError) as e:
        call(**change)
    assert e.value.code == Bd.ERR_ARG
    assert not calls


@pytest.mark.parametrize("M,N,K", [(WRAP + 5, 64, 64), (5, WRAP + 64, 64), (5, 64, WRAP + 64)])
def test_the_plan_of_more_than_an_int_holds(calls, M, N, K):
    with pytest.raises(H.HeroError) as e:
        H.hero_plan_fp8_gemm(M, N, K)
    assert e.value.code == Bd.ERR_ARG
    assert not calls
