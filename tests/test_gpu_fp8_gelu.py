"""GELU in the 8-bit product against the formula in 64 bits, to what an fp32 evaluation leaves, whatever the result's type and
whatever stands beside a value: four neighbours of a row share a reciprocal."""
import math

import numpy as np
import pytest
import torch

from tests import fp8_ref as R

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": F8}
# (tile, thread blocks per tile, exchanged), M, N, K: every epilogue
CASES = [((16, 1, True), 40, 304, 16, "bf16"), ((16, 1, True), 40, 304, 16, "fp32"), ((16, 1, True), 40, 304, 16, "e4m3"),
         ((64, 1, False), 600, 1200, 144, "bf16"), ((64, 1, False), 600, 1200, 144, "fp32"),
         ((128, 1, False), 51, 9584, 176, "bf16"), ((128, 1, False), 51, 9584, 176, "fp32"), ((128, 1, False), 51, 9584, 176, "e4m3"),
         ((256, 0, False), 2600, 2608, 16, "bf16"), ((256, 0, False), 2600, 2608, 16, "fp32"), ((256, 0, False), 2600, 2608, 16, "e4m3")]
# e4m3 numbers whose products with an argument of 16 bits are exact in fp32
FACTORS = np.array([1, -1, 0.5, -0.5, 2, -2, 1.5, -1.25, 448, -448, 2.0 ** -6, -2.0 ** -6, 0.75, -0.875, 3, -3.5], np.float64)


def H():
    import paper_2508_17588_b200 as h
    return h


def gelu64(t):
    """t (1 + tanh u) / 2 = t / (1 + exp(-2 u)), which does not cancel below zero."""
    with np.errstate(over="ignore", invalid="ignore"):
        return t / (1.0 + np.exp(-2.0 * math.sqrt(2.0 / math.pi) * (t + 0.044715 * t ** 3)))


def room(want, t):
    """What an fp32 evaluation of t / (1 + 2^x), x = -2 log2(e) u, is off by, for exact t.

    x: two rounded constants, t^2, a multiply-add and a product of terms of one sign, at most 4 * 2^-24 of it; it is at most 30 down to
    t = -5.52, so that 2^x is off by 30 * 4 * 2^-24 * ln 2 = 83.2 * 2^-24 of itself, and 4 * 2^-24 for the exponential instruction.  The
    sum, the product of four denominators, its reciprocal (2^-23) and the products that take the other three out again: 10 * 2^-24.
    Together less than 100 * 2^-24.  Below -5.52 the exponential is cut off at 2^30 and t at -16: at most 16 * 2^-30, as it is evaluated:
    2^30 carries the exponential instruction's 4 * 2^-24, and the sum, reciprocal and products their 10 * 2^-24."""
    return 100 * 2.0 ** -24 * np.abs(want) + np.where(t < -5.5, 2.0 ** -26 * (1 + 14 * 2.0 ** -24), 0.0)


def run(arguments, factors, K, out):
    """GELU of arguments[m] * factors[n]: one element of each row of A and W is not zero."""
    M, N = len(arguments), len(factors)
    a = torch.zeros(M, K, device="cuda")
    a[:, 5] = 1.0
    w = torch.zeros(N, K, device="cuda")
    w[:, 5] = torch.from_numpy(factors.astype(np.float32)).cuda()
    a_s = torch.from_numpy(arguments.astype(np.float32)).cuda()[:, None].repeat(1, R.blocks(K)).contiguous()
    c = torch.full((M, N), float("nan"), device="cuda").to(TORCH[out])
    c_scale = torch.full((M, R.blocks(N)), float("nan"), device="cuda") if out == "e4m3" else None
    H().hero_gemm_fp8(a.to(F8), a_s, w.to(F8), torch.ones(R.blocks(N), R.blocks(K), device="cuda"), None, c, c_scale, act=1)
    H().hero_isolated_status()
    return c.double().cpu().numpy() if out != "e4m3" else c.float().cpu().numpy(), None if c_scale is None else c_scale.double().cpu().numpy()


@pytest.mark.parametrize("plan,M,N,K,out", CASES)
def test_gelu_to_fp32_accuracy(plan, M, N, K, out):
    """Arguments from -8.5 to 8.5 in the factors of magnitude 1, and of a few hundred, nearly zero and both signs beside them."""
    assert H().hero_plan_fp8_gemm(M, N, K, out == "e4m3") == plan
    rng = np.random.default_rng(M + N)
    s = np.round((np.arange(M) + 1) / M * 8.5 * 4096) / 4096            # 16 bits
    f = FACTORS[rng.integers(0, len(FACTORS), N)]
    t = s[:, None] * f[None, :]
    assert (t.astype(np.float32).astype(np.float64) == t).all()
    want = gelu64(t)
    err = room(want, t)
    got, scale = run(s, f, K, out)
    if out == "e4m3":
        R.check_quantized(got, scale, want, err)
    else:
        tol = err + R.HALF[out] * (np.abs(want) + err)
        off = np.abs(got - want)
        assert (off <= tol).all(), (float((off / tol).max()), t.flat[(off / tol).argmax()], got.flat[(off / tol).argmax()])


@pytest.mark.parametrize("plan,M,N,K,out", [c for c in CASES if c[-1] != "e4m3"])
def test_gelu_beside_what_is_not_finite(plan, M, N, K, out):
    """Infinity stays, its negative becomes zero, NaN stays, and their neighbours are what they are without them."""
    assert H().hero_plan_fp8_gemm(M, N, K, False) == plan
    rng = np.random.default_rng(M + N)
    s = np.where(np.arange(M) % 2 == 0, 2.0 ** 127, 1.5)                # times 448: an infinity
    f = np.array([448, -448, 2.0 ** -6, -2.0 ** -6, 1, -1, np.nan])[rng.integers(0, 7, N)]
    with np.errstate(over="ignore"):
        t = (s[:, None] * f[None, :]).astype(np.float32).astype(np.float64)
    assert np.isinf(t).any() and np.isnan(t).any()
    want = np.where(t == -np.inf, 0.0, gelu64(np.where(t == -np.inf, -1.0, t)))
    want = np.where(t < -1e3, 0.0, want)
    got, _ = run(s, f, K, out)
    assert np.array_equal(np.isnan(got), np.isnan(t))
    assert np.array_equal(got == np.inf, want == np.inf)
    finite = np.isfinite(want)
    w, g = want[finite], got[finite]
    err = room(w, t[finite])
    assert (np.abs(g - w) <= err + R.HALF[out] * (np.abs(w) + err)).all()


@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_gelu_repeats_whatever_its_neighbours(out):
    """An argument's result beside others of the same size and beside far ones differs by no more than the evaluation may be off."""
    t = np.round(np.linspace(-5.4, 5.4, 64) * 4096) / 4096
    alone = run(t, np.ones(16), 16, out)[0][:, 0]
    beside = run(t, np.tile([1.0, 448.0, -448.0, 2.0 ** -6], 4), 16, out)[0][:, 0]
    want = np.abs(gelu64(t))
    assert (np.abs(alone - beside) <= 2 * (room(want, t) + R.HALF[out] * (want + room(want, t)))).all()
