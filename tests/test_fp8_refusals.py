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


BIG = 1 << 40                              # (addresses so far apart that nothing of these calls meets)


@pytest.mark.parametrize("change", [
    dict(q=BIG), dict(q=BIG + 496), dict(x=2 * BIG + 240), dict(scale=2 * BIG + 128), dict(scale=BIG + 508), dict(q=3 * BIG - 240)])
def test_quantize_results_apart(change):
    a = dict(x=BIG, q=2 * BIG, scale=3 * BIG, rows=4, cols=64, block_rows=1, dtype=1)
    a.update(change)
    assert H.load().hero_quantize_fp8(*a.values(), None) == ARG


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("change", [dict(total=P + 128), dict(out=2 * P - 16), dict(total=5 * P + 240), dict(gain=4 * P + 496),
                                    dict(gain=5 * P - 112), dict(total=2 * P + 16, add=2 * P), dict(add=P + 64, total=P)])
def test_rms_norm_results_apart(fp8, change):
    assert _rms(H.load(), fp8, **change) == ARG


@pytest.mark.parametrize("change", [dict(scale=P), dict(scale=2 * P + 508), dict(scale=3 * P + 64), dict(scale=4 * P), dict(scale=5 * P + 252),
                                    dict(out=P + 496)])
def test_rms_norm_fp8_results_apart(change):
    assert _rms(H.load(), True, **change) == ARG


@pytest.mark.parametrize("change", [
    dict(out=BIG), dict(out=2 * BIG + 2 * 8 * 64 * 2 - 16), dict(out=3 * BIG), dict(out=4 * BIG + (64 + 64) * 4 - 16), dict(out=5 * BIG),
    dict(out=7 * BIG - 2 * 4 * 64 + 16), dict(out_scale=BIG + 4), dict(out_scale=3 * BIG + 12)])
def test_gather_ln_modulate_results_apart(change):
    a = dict(x=BIG, add=2 * BIG, idx=3 * BIG, shift=4 * BIG, scale=5 * BIG, mod_ld=64, out=6 * BIG, out_scale=7 * BIG, B=2, N=8, n_sel=4, D=64,
             dtype=1)
    a.update(change)
    assert H.load().hero_gather_ln_modulate_fp8(*a.values(), None) == ARG


@pytest.mark.parametrize("change", [
    dict(c=BIG + 240), dict(c=2 * BIG), dict(c=3 * BIG + 32 * 64 - 16), dict(c=4 * BIG), dict(c=5 * BIG + 48), dict(c=7 * BIG - 112),
    dict(c_scale=BIG), dict(c_scale=2 * BIG + 12), dict(c_scale=3 * BIG), dict(c_scale=5 * BIG)])
def test_gemm_results_apart(change):
    a = dict(a=BIG, a_scale=2 * BIG, w=3 * BIG, w_scale=4 * BIG, bias=5 * BIG, c=6 * BIG, c_scale=7 * BIG, M=4, N=32, K=64, act=0, out_dtype=2)
    a.update(change)
    assert H.load().hero_gemm_fp8(*a.values(), None) == ARG


def test_sizes_that_an_int_does_not_hold_when_rounded_up_to_tiles():
    lib, top = H.load(), 2 ** 31 - 1
    assert lib.hero_quantize_fp8(BIG, 2 * BIG, 3 * BIG, top, 16, 128, 1, None) == ARG
    assert lib.hero_quantize_fp8(BIG, 2 * BIG, 3 * BIG, 1, top - 15, 1, 1, None) == ARG
    for M, N, K, out in ((top, 1, 16, 1), (1, top, 16, 1), (1, 16, top - 15, 1), (1, 1 << 29, 16, 0), (1, 1 << 30, 16, 1)):
        assert lib.hero_gemm_fp8(BIG, 2 * BIG, 3 * BIG, 4 * BIG, 0, 5 * BIG, 0, M, N, K, 0, out, None) == ARG


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
                        assert columns == 16 and ctas in (1, 2, 4, 8)
                    elif ctas == 0:
                        assert columns == 256
                    else:
                        assert ctas in (1, 2, 4) and (columns == 128 or (columns == 64 and not f8))
                    assert ctas <= -(-K // 128)
    with pytest.raises(H.HeroError):
        H.hero_plan_fp8_gemm(0, 1, 16)
