"""What the 8-bit operators refuse, before any CUDA work: the C ABI's codes and the binding's checks.  No GPU needed."""
import pytest
import torch

import paper_2508_17588_b200 as H
from paper_2508_17588_b200 import binding as Bd

P = 4096                                   # an aligned address that no call here reads
ARG, ALIGN, OK = Bd.ERR_ARG, Bd.ERR_ALIGN, Bd.OK


@pytest.mark.parametrize("want,args", [
    (OK, (0, 0, 0, 0, 64, 1, 1)),                     # no rows
    (ARG, (P, P, P, -1, 64, 1, 1)), (ARG, (P, P, P, 4, 0, 1, 1)), (ARG, (P, P, P, 4, 64, 2, 1)), (ARG, (P, P, P, 4, 64, 1, 2)),
    (ARG, (P, P, P, 4, 64, 1, -1)), (ARG, (0, P, P, 4, 64, 1, 1)), (ARG, (P, 0, P, 4, 64, 1, 1)), (ARG, (P, P, 0, 4, 64, 1, 1)),
    (ALIGN, (P, P, P, 4, 72, 1, 1)), (ALIGN, (P + 8, P, P, 4, 64, 1, 1)), (ALIGN, (P, P + 4, P, 4, 64, 128, 0)),
    (ALIGN, (P, P, P + 2, 4, 64, 1, 1))])
def test_quantize(want, args):
    assert H.load().hero_quantize_fp8(*args, None) == want


def _rms(lib, fp8, x=P, add=2 * P, gain=3 * P, total=4 * P, out=5 * P, scale=6 * P, rows=4, D=64, eps=1e-5, dtype=1):
    if fp8:
        return lib.hero_rms_norm_fp8(x, add, gain, total, out, scale, rows, D, eps, dtype, None)
    return lib.hero_rms_norm(x, add, gain, total, out, rows, D, eps, dtype, None)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("want,change", [
    (OK, dict(rows=0, x=0, out=0)), (ARG, dict(rows=-1)), (ARG, dict(D=0)), (ARG, dict(D=12288 + 16)), (ARG, dict(eps=-1e-9)),
    (ARG, dict(eps=float("nan"))), (ARG, dict(dtype=2)), (ARG, dict(x=0)), (ARG, dict(out=0)), (ARG, dict(total=5 * P)),
    (ALIGN, dict(D=60)), (ALIGN, dict(x=P + 8)), (ALIGN, dict(add=P + 4)), (ALIGN, dict(gain=P + 2)), (ALIGN, dict(total=P + 8)),
    (ALIGN, dict(out=P + 8))])
def test_rms_norm(fp8, want, change):
    assert _rms(H.load(), fp8, **change) == want


@pytest.mark.parametrize("want,change", [(ARG, dict(scale=0)), (ALIGN, dict(scale=P + 1)), (ALIGN, dict(D=72)), (ALIGN, dict(D=68, dtype=0)),
                                         (ARG, dict(out=P)), (ARG, dict(out=2 * P))])
def test_rms_norm_fp8_only(want, change):
    assert _rms(H.load(), True, **change) == want


@pytest.mark.parametrize("want,change", [
    (OK, dict(n_sel=0, x=0)), (OK, dict(B=0, x=0)), (ARG, dict(n_sel=9)), (ARG, dict(N=-1, n_sel=-1)), (ARG, dict(mod_ld=32)),
    (ARG, dict(D=12288 + 16, mod_ld=16384)), (ARG, dict(dtype=2)), (ARG, dict(x=0)), (ARG, dict(shift=0)), (ARG, dict(scale=0)),
    (ARG, dict(out=0)), (ARG, dict(out_scale=0)), (ALIGN, dict(D=56)), (ALIGN, dict(x=P + 8)), (ALIGN, dict(add=P + 8)),
    (ALIGN, dict(out=P + 8)), (ALIGN, dict(out_scale=P + 2)), (ALIGN, dict(idx=P + 2)), (ALIGN, dict(shift=P + 1)),
    (ARG, dict(B=1 << 20, N=1 << 20, n_sel=1 << 20))])
def test_gather_ln_modulate(want, change):
    a = dict(x=P, add=0, idx=P, shift=P, scale=P, mod_ld=64, out=P, out_scale=P, B=1, N=8, n_sel=4, D=64, dtype=1)
    a.update(change)
    assert H.load().hero_gather_ln_modulate_fp8(*a.values(), None) == want


@pytest.mark.parametrize("want,change", [
    (OK, dict(M=0, a=0)), (ARG, dict(M=-1)), (ARG, dict(N=0)), (ARG, dict(K=0)), (ARG, dict(act=2)), (ARG, dict(out_dtype=3)),
    (ARG, dict(a=0)), (ARG, dict(a_scale=0)), (ARG, dict(w=0)), (ARG, dict(w_scale=0)), (ARG, dict(c=0)), (ARG, dict(c_scale=P)),
    (ARG, dict(out_dtype=2)), (ALIGN, dict(K=72)), (ALIGN, dict(out_dtype=2, c_scale=P, N=24)), (ALIGN, dict(a=P + 8)),
    (ALIGN, dict(w=P + 8)), (ALIGN, dict(c=P + 8)), (ALIGN, dict(a_scale=P + 2)), (ALIGN, dict(w_scale=P + 2)),
    (ALIGN, dict(out_dtype=2, c_scale=P + 2)), (ALIGN, dict(bias=P + 1))])
def test_gemm(want, change):
    a = dict(a=P, a_scale=P, w=P, w_scale=P, bias=P, c=P, c_scale=0, M=4, N=32, K=64, act=0, out_dtype=1)
    a.update(change)
    assert H.load().hero_gemm_fp8(*a.values(), None) == want


def test_the_binding_refuses_what_is_not_on_a_gpu_or_of_another_shape():
    f8, f32 = torch.float8_e4m3fn, torch.float32
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    calls = [lambda: H.hero_quantize_fp8(x, x.to(f8), torch.zeros(4, 1)),
             lambda: H.hero_quantize_fp8(x.half(), x.to(f8), torch.zeros(4, 1)),
             lambda: H.hero_quantize_fp8(x[0], x.to(f8), torch.zeros(4, 1)),
             lambda: H.hero_rms_norm(x, None, None, None, torch.empty_like(x)),
             lambda: H.hero_rms_norm_fp8(x, None, None, None, x.to(f8), torch.zeros(4, 1)),
             lambda: H.hero_gather_ln_modulate_fp8(x[None], None, None, torch.zeros(1, 64), torch.zeros(1, 64), x[None].to(f8),
                                                   torch.zeros(1, 4, 1)),
             lambda: H.hero_gather_ln_modulate_fp8(x[None], None, None, torch.zeros(1, 32), torch.zeros(1, 64), x[None].to(f8),
                                                   torch.zeros(1, 4, 1)),
             lambda: H.hero_gemm_fp8(x.to(f8), torch.zeros(4, 1), x.to(f8), torch.zeros(1, 1), None, torch.zeros(4, 4, dtype=f32)),
             lambda: H.hero_gemm_fp8(x.to(f8), torch.zeros(4, 1), x.to(f8), torch.zeros(1, 1), None, torch.zeros(4, 4).half())]
    for call in calls:
        with pytest.raises(H.HeroError) as e:
            call()
        assert e.value.code == ARG


def test_the_rule_on_sizes_names_what_there_is():
    for M in (1, 16, 17, 32, 33, 64, 65, 200, 1000, 9000):
        for N in (1, 16, 129, 1000, 12288):
            for K in (16, 128, 1040, 12288):
                for f8 in (False, True):
                    columns, ctas, swap = H.hero_plan_fp8_gemm(M, N, K, f8)
                    if swap:
                        assert columns in (16, 32, 64) and ctas in (1, 2, 4, 8)
                    elif ctas == 0:
                        assert columns == 256 or (columns == 128 and not f8)
                    else:
                        assert ctas in (1, 2, 4) and (columns == 128 or (columns == 64 and not f8))
                    assert ctas <= -(-K // 128)
    with pytest.raises(H.HeroError):
        H.hero_plan_fp8_gemm(0, 1, 16)
