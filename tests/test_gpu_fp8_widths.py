"""The row kernels of the 8-bit path at the last width of every variant that a row's length chooses, and at the first of the next."""
import numpy as np
import pytest
import torch

from tests import fp8_ref as R
from tests.util import to_dev, to_host
from workloads import synthetic as S

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}
STEPS = [1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 96]             # warps times pieces a lane


def H():
    import paper_2508_17588_b200 as h
    return h


def widths(unit):
    """unit: columns that a warp holds with one piece a lane."""
    return sorted({w for s in STEPS for w in (s * unit, s * unit + 16) if w <= 12288})


def values(rng, shape, dtype):
    v = (rng.standard_normal(shape) * np.exp(rng.standard_normal((*shape[:-1], 1)))).astype(np.float32)
    return S.round_bf16(v) if dtype == "bf16" else v


def empty(shape, dtype=None):
    return torch.full(shape, float("nan"), device="cuda").to(dtype or torch.float32)


# The errors of an fp32 evaluation: sums of at most 96 terms a lane and 13 steps over lanes and warps.
LN_ERR, RMS_ERR = 120 * 2.0 ** -24, (110 / 2 + 6) * 2.0 ** -24


@pytest.mark.parametrize("dtype,D", [("bf16", w) for w in widths(256)] + [("fp32", w) for w in widths(128)])
def test_gather_ln_modulate(dtype, D):
    B, N, n_sel = 2, 23, 19
    rng = np.random.default_rng(D)
    x, add = values(rng, (B, N, D), dtype), values(rng, (B, N, D), dtype)
    idx = np.sort(rng.choice(N, n_sel, replace=False)).astype(np.int32)
    mod = (0.5 * rng.standard_normal((B, 2 * D))).astype(np.float32)
    m, q, s = torch.from_numpy(mod).cuda(), empty((B, n_sel, D), F8), empty((B, n_sel, R.blocks(D)))
    H().hero_gather_ln_modulate_fp8(to_dev(x, dtype), to_dev(add, dtype), torch.from_numpy(idx).cuda(), m[:, :D], m[:, D:], q, s)
    for b in range(B):
        h = x[b, idx].astype(np.float64) + add[b, idx].astype(np.float64)
        centred = h - h.mean(-1, keepdims=True)
        sd = np.sqrt((centred ** 2).mean(-1, keepdims=True) + 1e-5)
        g = 1.0 + mod[b, D:].astype(np.float64)
        want = centred / sd * g + mod[b, :D].astype(np.float64)
        err = LN_ERR * ((np.abs(h).max(-1, keepdims=True) / sd + np.abs(centred) / sd) * np.abs(g) + np.abs(want))
        R.check_quantized(q[b].float().cpu().numpy(), s[b].double().cpu().numpy(), want, err)


@pytest.mark.parametrize("dtype,D", [("bf16", w) for w in widths(512)] + [("fp32", w) for w in widths(256)])
def test_rms_norm(dtype, D):
    rows = 19
    rng = np.random.default_rng(D)
    x, add, gain = values(rng, (rows, D), dtype), values(rng, (rows, D), dtype), values(rng, (1, D), dtype)[0]
    dev = [to_dev(t, dtype) for t in (x, add, gain)]
    q, s, o, total = empty((rows, D), F8), empty((rows, R.blocks(D))), empty((rows, D), TORCH[dtype]), empty((rows, D), TORCH[dtype])
    H().hero_rms_norm_fp8(*dev, None, q, s)
    H().hero_rms_norm(*dev, total, o)
    y = R.rms_norm(x, add, gain, 1e-5)[1]
    R.check_quantized(q.float().cpu().numpy(), s.double().cpu().numpy(), y, RMS_ERR * np.abs(y))
    assert (np.abs(to_host(o) - y) <= (R.HALF[dtype] + RMS_ERR * 1.01) * np.abs(y) + 1e-37).all()
    assert torch.equal(total.cpu(), (torch.from_numpy(x) + torch.from_numpy(add)).to(TORCH[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [640, 12288])
def test_rms_norm_of_large_magnitudes(D, dtype):
    """Up to the largest whose squares fp32 holds the norm is what it is of ordinary rows; beyond, zeros; the sum is kept all the same."""
    x = values(np.random.default_rng(D), (5, D), dtype)
    x[1] = S.round_bf16(np.float32([1e16])) * np.sign(x[1])
    x[3] = S.round_bf16(np.float32([1e20])) * np.sign(x[3])
    d, q, s, o, total = to_dev(x, dtype), empty((5, D), F8), empty((5, R.blocks(D))), empty((5, D), TORCH[dtype]), empty((5, D), TORCH[dtype])
    H().hero_rms_norm_fp8(d, None, None, None, q, s)
    H().hero_rms_norm(d, None, None, total, o)
    y = R.rms_norm(x, None, None, 1e-5)[1]
    y[3] = 0.0
    R.check_quantized(q.float().cpu().numpy(), s.double().cpu().numpy(), y, RMS_ERR * np.abs(y))
    assert (np.abs(to_host(o) - y) <= (R.HALF[dtype] + RMS_ERR * 1.01) * np.abs(y) + 1e-37).all()
    assert torch.equal(total, d)
