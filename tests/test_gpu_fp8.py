"""The 8-bit operators on the GPU against plain implementations in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

from oracle import hero_oracle as O
from tests import fp8_ref as R
from tests.util import to_dev, to_host
from workloads import synthetic as S

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": F8}


def H():
    import paper_2508_17588_b200 as h
    return h


def values(rng, rows, cols, dtype, spread=1.0):
    v = (rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal((rows, 1)))).astype(np.float32)
    return S.round_bf16(v) if dtype == "bf16" else v


def new(shape, dtype):
    """An output that holds NaN (e4m3: the byte of NaN) until it is written."""
    t = torch.empty(shape, device="cuda", dtype=TORCH[dtype])
    (t.view(torch.uint8).fill_(0x7F) if dtype == "e4m3" else t.fill_(float("nan")))
    return t


def host32(t):
    return t.float().cpu().numpy()


# ------------------------------------------------------------------ quantiser
QUANT_SHAPES = [(1, 16), (1, 128), (3, 144), (5, 240), (127, 256), (128, 272), (129, 1040), (300, 3072), (7, 12304)]


@pytest.mark.parametrize("rows,cols", QUANT_SHAPES)
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantize(rows, cols, block_rows, dtype):
    v = values(np.random.default_rng(rows * 31 + cols), rows, cols, dtype, 2.0)
    q, s = new((rows, cols), "e4m3"), new((rows if block_rows == 1 else R.blocks(rows), R.blocks(cols)), "fp32")
    H().hero_quantize_fp8(to_dev(v, dtype), q, s, block_rows)
    want_q, want_s = R.quantize32(v, block_rows)
    assert np.array_equal(host32(s), want_s)
    assert np.array_equal(host32(q), want_q)
    # and what it stands for is the value to half a step
    got = R.dequantize(host32(q), host32(s), block_rows)
    room = R.spread(want_s.astype(np.float64), block_rows, rows, cols) * R.SUBNORMAL
    assert (np.abs(got - v) <= (R.HALF["e4m3"] + 2.0 ** -20) * np.abs(v) + 1.001 * room).all()


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantize_extremes(block_rows, dtype):
    """Blocks of zeros, of the smallest and of the largest magnitudes, with one infinity, with one NaN; their neighbours untouched."""
    rows, cols = 260, 640
    v = values(np.random.default_rng(5), rows, cols, dtype)
    v[:, :128] = 0.0
    v[:128, 128:256] = S.round_bf16(np.float32([[1e-39]])) if dtype == "bf16" else np.float32(1e-44)
    v[128:256, 128:256] = np.float32(2.0 ** 127)
    v[3, 300], v[131, 301], v[259, 500] = np.inf, -np.inf, np.nan
    q, s = new((rows, cols), "e4m3"), new((rows if block_rows == 1 else 3, 5), "fp32")
    H().hero_quantize_fp8(to_dev(v, dtype), q, s, block_rows)
    want_q, want_s = R.quantize32(v, block_rows)
    assert np.array_equal(host32(s), want_s, equal_nan=True)
    assert np.array_equal(host32(q), want_q, equal_nan=True)
    assert np.isnan(want_s).sum() == 3                    # one block each, and the whole block
    assert (host32(q)[:, :128] == 0).all() and (host32(s)[:, 0] == np.float32(R.FLOOR)).all()


# ------------------------------------------------------------------ root-mean-square norm
# Sums of squares: a lane adds at most 96 in a row, 14 more steps over lanes and warps, all of one sign; the root halves that;
# sum, root, division, norm and gain round once more each.
RMS_ERR = (110 / 2 + 6) * 2.0 ** -24
RMS_WIDTHS = [16, 128, 144, 512, 1024, 1040, 1536, 2064, 3072, 4096, 4112, 6144, 8208, 12288]


def check_rms(rows, D, dtype, out, with_add, with_gain, keep, eps=1e-5, alias=None):
    rng = np.random.default_rng(rows + D)
    x = values(rng, rows, D, dtype, 2.0)
    add = values(rng, rows, D, dtype) if with_add else None
    gain = values(rng, 1, D, dtype)[0] if with_gain else None
    dev = [None if t is None else to_dev(t, dtype) for t in (x, add, gain)]
    total = {"x": dev[0], "add": dev[1], None: new((rows, D), dtype) if keep else None}[alias]
    h, y = R.rms_norm(x, add, gain, eps)
    if out == "e4m3":
        o, s = new((rows, D), "e4m3"), new((rows, R.blocks(D)), "fp32")
        H().hero_rms_norm_fp8(*dev, total, o, s, eps)
        # (an added-up h is off by half a step of fp32 itself)
        R.check_quantized(host32(o), host32(s).astype(np.float64), y, RMS_ERR * np.abs(y))
    else:
        o = new((rows, D), dtype)
        H().hero_rms_norm(*dev, total, o, eps)
        assert (np.abs(to_host(o) - y) <= (R.HALF[dtype] + RMS_ERR * 1.01) * np.abs(y) + 1e-37).all()
    if keep:
        want = torch.from_numpy(x).float() + (0 if add is None else torch.from_numpy(add).float())
        assert torch.equal(total.cpu(), want.to(TORCH[dtype]))


@pytest.mark.parametrize("D", RMS_WIDTHS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("quantized", [False, True])
def test_rms_norm_widths(D, dtype, quantized):
    check_rms(37, D, dtype, "e4m3" if quantized else dtype, True, True, True)


@pytest.mark.parametrize("rows", [1, 7, 8, 9, 1700])
@pytest.mark.parametrize("with_add,with_gain,keep", list(itertools.product([False, True], repeat=3)))
def test_rms_norm_options(rows, with_add, with_gain, keep):
    for dtype, out in (("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32"), ("fp32", "e4m3")):
        check_rms(rows, 400, dtype, out, with_add, with_gain, keep)


def test_rms_norm_narrow_widths_that_only_the_run_dtype_takes():
    check_rms(9, 8, "bf16", "bf16", True, True, True)
    check_rms(9, 1032, "bf16", "bf16", True, True, True)
    check_rms(9, 4, "fp32", "fp32", True, True, True)
    check_rms(9, 2052, "fp32", "fp32", True, False, True)


@pytest.mark.parametrize("alias", ["x", "add"])
@pytest.mark.parametrize("D", [400, 3072])
def test_rms_norm_sum_in_place(alias, D):
    for dtype, out in (("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32")):
        check_rms(70, D, dtype, out, True, True, True, alias=alias)


def test_rms_norm_sum_and_result_in_place():
    """sum over one input and, in the run dtype, the result over the other, on rows of one warp and of several."""
    for D, dtype in ((400, "bf16"), (6144, "fp32")):
        rng = np.random.default_rng(D)
        x, add = values(rng, 70, D, dtype, 2.0), values(rng, 70, D, dtype)
        y = R.rms_norm(x, add, None, 1e-5)[1]
        total = (torch.from_numpy(x) + torch.from_numpy(add)).to(TORCH[dtype])
        for over in ("x", "add"):
            dx, da = to_dev(x, dtype), to_dev(add, dtype)
            s, o = (dx, da) if over == "x" else (da, dx)
            H().hero_rms_norm(dx, da, None, s, o, 1e-5)
            assert torch.equal(s.cpu(), total)
            assert (np.abs(to_host(o) - y) <= (R.HALF[dtype] + RMS_ERR * 1.01) * np.abs(y) + 1e-37).all()


def test_rms_norm_rows_of_zeros_and_rows_that_are_not_finite():
    D = 640
    x = values(np.random.default_rng(1), 6, D, "bf16")
    x[1] = 0.0
    x[3, 17], x[4, 300] = np.nan, np.inf
    q, s, o = new((6, D), "e4m3"), new((6, 5), "fp32"), new((6, D), "bf16")
    H().hero_rms_norm_fp8(to_dev(x, "bf16"), None, None, None, q, s)
    H().hero_rms_norm(to_dev(x, "bf16"), None, None, None, o)
    q, s, o = host32(q), host32(s), to_host(o)
    assert (q[1] == 0).all() and (o[1] == 0).all() and (s[1] == np.float32(R.FLOOR)).all()
    assert np.isnan(q[3]).all() and np.isnan(s[3]).all() and np.isnan(o[3]).all()
    assert np.isnan(o[4, 300]) and np.isnan(q[4, 256:384]).all()      # Inf / Inf; the rest of the row is divided by infinity
    assert (np.delete(o[4], 300) == 0).all()
    for r in (0, 2, 5):
        R.check_quantized(q[r:r + 1], s[r:r + 1].astype(np.float64), R.rms_norm(x[r:r + 1], None, None, 1e-5)[1],
                          RMS_ERR * np.abs(R.rms_norm(x[r:r + 1], None, None, 1e-5)[1]))


# ------------------------------------------------------------------ gather + LayerNorm + modulate
@pytest.mark.parametrize("dtype,B,N,D,n_sel,with_add,with_idx,mod_pad", [
    ("bf16", 1, 1, 16, 1, False, True, 0), ("bf16", 2, 50, 256, 17, True, True, 0), ("fp32", 1, 40, 128, 9, False, True, 0),
    ("fp32", 2, 33, 272, 33, True, False, 0), ("bf16", 3, 300, 1024, 77, False, True, 0), ("bf16", 2, 123, 2064, 50, True, True, 0),
    ("bf16", 2, 500, 3072, 259, True, True, 0), ("bf16", 1, 40, 4096, 13, True, True, 0), ("fp32", 1, 30, 2048, 30, True, True, 0),
    ("bf16", 2, 20, 4112, 13, True, True, 0), ("fp32", 2, 20, 2064, 13, False, True, 0),
    ("bf16", 1, 9, 12288, 9, True, False, 0), ("fp32", 1, 9, 12288, 9, True, False, 0),
    ("bf16", 2, 50, 256, 17, True, True, 1), ("fp32", 2, 50, 144, 17, False, True, 3),        # vectors that are not 16-byte aligned
    ("bf16", 2, 17776, 256, 4387, True, True, 0)])
def test_gather_ln_modulate(dtype, B, N, D, n_sel, with_add, with_idx, mod_pad):
    rng = np.random.default_rng(N * 7 + D + n_sel)
    x = (values(rng, B * N, D, dtype, 1.0) + 0.5 * (dtype == "fp32")).reshape(B, N, D).astype(np.float32)
    add = values(rng, B * N, D, dtype, 0.0).reshape(B, N, D) if with_add else None
    idx = np.sort(rng.choice(N, n_sel, replace=False)).astype(np.int32) if with_idx else None
    mod = rng.standard_normal((B, 4 * D + mod_pad)).astype(np.float32) * 0.5
    mod_d = torch.from_numpy(mod).cuda()
    q, s = new((B, n_sel, D), "e4m3"), new((B, n_sel, R.blocks(D)), "fp32")
    H().hero_gather_ln_modulate_fp8(to_dev(x, dtype), None if add is None else to_dev(add, dtype),
                                    None if idx is None else torch.from_numpy(idx).cuda(), mod_d[:, :D], mod_d[:, D:2 * D], q, s)
    for b in range(B):
        rows = np.arange(n_sel) if idx is None else idx
        h = x[b, rows].astype(np.float64) + (0.0 if add is None else add[b, rows].astype(np.float64))
        mean = h.mean(-1, keepdims=True)
        sd = np.sqrt(((h - mean) ** 2).mean(-1, keepdims=True) + 1e-5)
        g = 1.0 + mod[b, D:2 * D].astype(np.float64)
        want = (h - mean) / sd * g + mod[b, :D].astype(np.float64)
        # fp32: mean and variance from sums of at most 96 + 13 steps; h and the difference are off by that much of the row's largest
        # magnitude, the quotient by half of it besides
        err = 120 * 2.0 ** -24 * ((np.abs(h).max(-1, keepdims=True) / sd + np.abs(h - mean) / sd) * np.abs(g) + np.abs(want))
        R.check_quantized(host32(q[b]), host32(s[b]).astype(np.float64), want, err)


def test_gather_ln_modulate_the_same_row_twice():
    x = values(np.random.default_rng(2), 40, 512, "bf16")
    mod = torch.zeros(1, 1024, device="cuda")
    idx = torch.tensor([7, 7, 39, 7], dtype=torch.int32, device="cuda")
    q, s = new((1, 4, 512), "e4m3"), new((1, 4, 4), "fp32")
    H().hero_gather_ln_modulate_fp8(to_dev(x[None], "bf16"), None, idx, mod[:, :512], mod[:, 512:], q, s)
    assert torch.equal(q[0, 0].float(), q[0, 1].float()) and torch.equal(s[0, 0], s[0, 3]) and not torch.equal(s[0, 0], s[0, 2])


def test_gather_ln_modulate_rows_that_are_not_finite():
    """NaN for the row that holds one, or an infinity, whatever the modulation; its neighbours and rows off the list as without it."""
    for D, dtype in ((256, "bf16"), (3072, "bf16"), (1040, "fp32")):
        x = values(np.random.default_rng(D), 40, D, dtype)
        bad = x.copy()
        bad[3, D - 1], bad[5, 0], bad[9, 7] = np.nan, np.inf, -np.inf
        bad[11:13] = np.nan                                    # not on the list
        idx = torch.tensor([2, 3, 4, 5, 6, 8, 9, 10, 13], dtype=torch.int32, device="cuda")
        mod = 0.2 * torch.randn(1, 2 * D, device="cuda", generator=torch.Generator("cuda").manual_seed(D))
        got = []
        for v in (x, bad):
            q, s = new((1, 9, D), "e4m3"), new((1, 9, R.blocks(D)), "fp32")
            H().hero_gather_ln_modulate_fp8(to_dev(v[None], dtype), None, idx, mod[:, :D], mod[:, D:], q, s)
            got.append((host32(q[0]), host32(s[0])))
        hit = np.isin(idx.cpu().numpy(), (3, 5, 9))
        assert np.isnan(got[1][0][hit]).all() and np.isnan(got[1][1][hit]).all()
        assert (got[1][0][~hit] == got[0][0][~hit]).all() and (got[1][1][~hit] == got[0][1][~hit]).all()


@pytest.mark.parametrize("dtype,B,N,D,n_sel,with_idx", [("bf16", 1, 700000, 16, 600001, True), ("bf16", 2, 31000, 3072, 30007, True),
                                                        ("fp32", 1, 33000, 2064, 33000, False)])
def test_gather_ln_modulate_long_lists(dtype, B, N, D, n_sel, with_idx):
    """Lists so long that a thread block takes more than 32 rows (what it reads of the list at a time): as in calls of a few rows."""
    g = torch.Generator("cuda").manual_seed(D)
    x = torch.randn(B, N, D, device="cuda", generator=g).to(TORCH[dtype])
    mod = 0.3 * torch.randn(B, 2 * D, device="cuda", generator=g)
    idx = torch.randperm(N, device="cuda", generator=g)[:n_sel].int() if with_idx else None
    q, s = new((B, n_sel, D), "e4m3"), new((B, n_sel, R.blocks(D)), "fp32")
    h = H()
    h.hero_gather_ln_modulate_fp8(x, None, idx, mod[:, :D], mod[:, D:], q, s)
    rows = torch.arange(n_sel, device="cuda", dtype=torch.int32) if idx is None else idx
    for at in range(0, n_sel, 5000):
        part = rows[at:at + 5000].contiguous()
        q1, s1 = new((B, len(part), D), "e4m3"), new((B, len(part), R.blocks(D)), "fp32")
        h.hero_gather_ln_modulate_fp8(x, None, part, mod[:, :D], mod[:, D:], q1, s1)
        assert torch.equal(q[:, at:at + 5000].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[:, at:at + 5000], s1)


def test_many_small_batch_items():
    """More items than thread blocks fit the chip, a row or two of each."""
    B, D = 5000, 144
    x = values(np.random.default_rng(1), B * 3, D, "bf16").reshape(B, 3, D)
    mod = torch.from_numpy((0.3 * np.random.default_rng(2).standard_normal((B, 2 * D))).astype(np.float32)).cuda()
    q, s = new((B, 2, D), "e4m3"), new((B, 2, 2), "fp32")
    idx = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    xd, h = to_dev(x, "bf16"), H()
    h.hero_gather_ln_modulate_fp8(xd, None, idx, mod[:, :D], mod[:, D:], q, s)
    for b in (0, 1, 2500, B - 1):                              # the same rows alone
        q1, s1 = new((1, 2, D), "e4m3"), new((1, 2, 2), "fp32")
        h.hero_gather_ln_modulate_fp8(xd[b:b + 1], None, idx, mod[b:b + 1, :D], mod[b:b + 1, D:], q1, s1)
        assert torch.equal(q[b].float(), q1[0].float()) and torch.equal(s[b], s1[0])
    assert torch.isfinite(q.float()).all() and torch.isfinite(s).all()


# ------------------------------------------------------------------ product
def operands(rng, M, N, K, bias):
    a, a_s = R.quantize32(values(rng, M, K, "fp32", 0.5), 1)
    w, w_s = R.quantize32(values(rng, N, K, "fp32", 0.0) * np.float32(0.05), 128)
    b = S.round_bf16(rng.standard_normal(N).astype(np.float32) * 0.1) if bias else None
    dev = (torch.from_numpy(a).cuda().to(F8), torch.from_numpy(a_s).cuda(), torch.from_numpy(w).cuda().to(F8), torch.from_numpy(w_s).cuda(),
           None if b is None else to_dev(b, "bf16"))
    return (a, a_s, w, w_s, b), dev


def check_gemm(M, N, K, out, bias=True, act=0, seed=0):
    host, dev = operands(np.random.default_rng(seed + M * 7 + N * 3 + K), M, N, K, bias)
    c, c_scale = new((M, N), out), new((M, R.blocks(N)), "fp32") if out == "e4m3" else None
    H().hero_gemm_fp8(*dev, c, c_scale, act)
    H().hero_isolated_status()
    want, err = R.gemm(*host, act)
    got = host32(c).astype(np.float64)
    if out == "e4m3":
        R.check_quantized(got, host32(c_scale).astype(np.float64), want, err)
    else:
        tol = err + R.HALF[out] * (np.abs(want) + err)
        assert (np.abs(got - want) <= tol).all(), (M, N, K, float((np.abs(got - want) / tol).max()))


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 32, 33, 63, 64, 65, 127, 128, 129, 257])
@pytest.mark.parametrize("N,K", [(16, 16), (128, 128), (144, 272), (400, 1040), (1280, 2064)])
def test_gemm_row_counts(M, N, K):
    for out in ("bf16", "fp32", "e4m3"):
        check_gemm(M, N, K, out)


@pytest.mark.parametrize("N", [1, 2, 3, 7, 17, 63, 127, 129, 255, 1001])
@pytest.mark.parametrize("M", [1, 40, 200])
def test_gemm_odd_widths(M, N):
    for out in ("bf16", "fp32"):
        check_gemm(M, N, 336, out, act=1)


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("bias,act", [(False, 0), (False, 1), (True, 1)])
def test_gemm_bias_and_activation(out, bias, act):
    for M in (5, 50, 150):
        check_gemm(M, 272, 640, out, bias, act)


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("M,N,K", [(2600, 2608, 272), (2305, 2064, 128), (1793, 4112, 16), (5000, 3072, 400)])
def test_gemm_that_fills_the_chip(out, M, N, K):
    assert H().hero_plan_fp8_gemm(M, N, K, out == "e4m3")[1] == 0
    check_gemm(M, N, K, out, act=1)


def test_gemm_that_fills_the_chip_odd_width():
    for out in ("bf16", "fp32"):
        check_gemm(2600, 2601, 272, out)


@pytest.mark.parametrize("M", [3, 40, 130])
def test_gemm_what_is_not_finite_stays_in_its_row(M):
    rng = np.random.default_rng(M)
    host, dev = operands(rng, M, 272, 640, True)
    for out in ("bf16", "e4m3"):
        clean, dirty = new((M, 272), out), new((M, 272), out)
        s1, s2 = (new((M, 3), "fp32"), new((M, 3), "fp32")) if out == "e4m3" else (None, None)
        H().hero_gemm_fp8(*dev, clean, s1)
        a_s = dev[1].clone()
        a_s[1, 2] = float("nan")
        a = dev[0].clone()
        a.view(torch.uint8)[2, 639] = 0x7F
        H().hero_gemm_fp8(a, a_s, *dev[2:], dirty, s2)
        got, ref = host32(dirty), host32(clean)
        assert np.isnan(got[1:3]).all() and np.array_equal(np.delete(got, [1, 2], 0), np.delete(ref, [1, 2], 0))
        assert np.isfinite(ref).all()
        if s2 is not None:
            assert torch.isnan(s2[1:3]).all() and torch.isfinite(s2[3:]).all()


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("M", [3, 70, 2600])
def test_gemm_gelu_of_large_magnitudes(M, out):
    """Far below zero GELU is zero and far above it the identity, whatever the magnitude: sums of 1e2, 1e10 and 1e20, one sign a row."""
    N, K = 2608 if M > 2000 else 272, 144
    a = np.ones((M, K), np.float32)
    a_s = np.repeat(np.array([[1e0], [-1e0], [-1e8], [1e8], [-1e18], [1e18]], np.float32), 2, 1)[np.arange(M) % 6]
    w, w_s = np.ones((N, K), np.float32), np.ones((R.blocks(N), 2), np.float32)
    c, c_scale = new((M, N), out), new((M, R.blocks(N)), "fp32") if out == "e4m3" else None
    up = lambda t: torch.from_numpy(np.ascontiguousarray(t)).cuda()  # noqa: E731
    H().hero_gemm_fp8(up(a).to(F8), up(a_s), up(w).to(F8), up(w_s), None, c, c_scale, act=1)
    got = host32(c).astype(np.float64) if out != "e4m3" else R.dequantize(host32(c), host32(c_scale), 1)
    want = np.maximum(a_s[:, :1].astype(np.float64) * K, 0.0)
    # sums of equal terms, exact but for the scales' product; 16 * 2^-30 is what a value far below zero may leave; half a step of the type
    assert (np.abs(got - want) <= 2.0 ** -25 + (R.HALF[out] + 2.0 ** -22) * want).all()


def test_gemm_leaves_what_is_behind_its_result_alone():
    for M, N, out in ((3, 130, "bf16"), (70, 130, "fp32"), (200, 1001, "bf16"), (200, 272, "e4m3"), (9, 272, "e4m3")):
        _, dev = operands(np.random.default_rng(3), M, N, 272, True)
        room = new((M + 3, N), out)
        c_scale = new((M + 3, R.blocks(N)), "fp32") if out == "e4m3" else None
        H().hero_gemm_fp8(*dev, room[:M], None if c_scale is None else c_scale[:M])
        assert torch.isnan(room[M:].float()).all() and torch.isfinite(room[:M].float()).all()
        assert c_scale is None or (torch.isnan(c_scale[M:]).all() and torch.isfinite(c_scale[:M]).all())


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes of input and 2^31 elements: the last rows come out as they do alone."""
    h, rows, D, last = H(), 700001, 4096, 5
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.zeros(rows, D, device="cuda", dtype=torch.bfloat16)
    x[-200:].normal_(generator=g)
    tail = x[-last:].clone()
    # a scale per row, and per 128 x 128: 700001 = 128 * 5468 + 97, the last block by itself
    for block_rows, n in ((1, last), (128, 97)):
        q, s = torch.zeros(rows, D, device="cuda", dtype=F8), new((rows if block_rows == 1 else R.blocks(rows), D // 128), "fp32")
        q1, s1 = new((n, D), "e4m3"), new((n if block_rows == 1 else 1, D // 128), "fp32")
        h.hero_quantize_fp8(x, q, s, block_rows)
        h.hero_quantize_fp8(x[-n:].clone(), q1, s1, block_rows)
        assert torch.equal(q[-n:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[-s1.shape[0]:], s1)
        assert torch.isfinite(s).all() and (q[:1000].view(torch.uint8) == 0).all()
    # the norm, its sum over x, and the same in 8 bits
    o, o1 = torch.empty_like(x), torch.empty_like(tail)
    h.hero_rms_norm_fp8(x, None, None, None, q, s_rows := new((rows, D // 128), "fp32"))
    h.hero_rms_norm_fp8(tail, None, None, None, q1[:last], s1 := new((last, D // 128), "fp32"))
    assert torch.equal(q[-last:].view(torch.uint8), q1[:last].view(torch.uint8)) and torch.equal(s_rows[-last:], s1)
    h.hero_rms_norm(x, None, None, x, o)
    h.hero_rms_norm(tail, None, None, None, o1)
    assert torch.equal(o[-last:], o1) and torch.equal(x[-last:], tail) and (o[:1000] == 0).all()
    # rows from the end of a long matrix; the second of two items
    mod = 0.2 * torch.randn(2, 2 * D, device="cuda", generator=g)
    idx = torch.arange(350000 - last, 350000, dtype=torch.int32, device="cuda")
    both = x[1:].view(2, 350000, D)
    q2, s2 = new((2, last, D), "e4m3"), new((2, last, D // 128), "fp32")
    h.hero_gather_ln_modulate_fp8(both, None, idx, mod[:, :D], mod[:, D:], q2, s2)
    qa, sa = new((1, last, D), "e4m3"), new((1, last, D // 128), "fp32")
    h.hero_gather_ln_modulate_fp8(tail[None], None, None, mod[1:, :D], mod[1:, D:], qa, sa)
    assert torch.equal(q2[1].view(torch.uint8), qa[0].view(torch.uint8)) and torch.equal(s2[1], sa[0])
    del x, o, both
    # a product of more than 2^31 results from an operand of more than 2^31 elements: integers, exact in whatever order
    a = torch.zeros(rows, D, device="cuda", dtype=F8)
    a[-last:, -128:] = torch.randint(-3, 4, (last, 128), device="cuda", generator=g).float().to(F8)
    w = torch.randint(-3, 4, (3200, D), device="cuda", generator=g).float().to(F8)
    ones = lambda *shape: torch.ones(*shape, device="cuda")  # noqa: E731
    for out in (torch.float32, torch.bfloat16):
        c = torch.empty(rows, 3200, device="cuda", dtype=out)
        h.hero_gemm_fp8(a, ones(rows, D // 128), w, ones(25, D // 128), None, c)
        want = a[-last:, -128:].float().cpu() @ w[:, -128:].float().cpu().t()
        assert torch.equal(c[-last:].cpu(), want.to(out)) and (c[-1000:-last] == 0).all() and (c[:1000] == 0).all()
        del c


def test_gemm_repeats_bit_for_bit():
    for M, N, K in ((1, 4096, 4096), (48, 1000, 2064), (300, 400, 4096), (2600, 2608, 640)):
        _, dev = operands(np.random.default_rng(9), M, N, K, True)
        first, again = new((M, N), "fp32"), new((M, N), "fp32")
        H().hero_gemm_fp8(*dev, first)
        for _ in range(5):
            H().hero_gemm_fp8(*dev, again)
            assert torch.equal(first, again)


def test_gemm_random_shapes():
    rng = np.random.default_rng(77)
    for _ in range(25):
        M, N, K = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (900, 1500, 150))
        out = ["bf16", "fp32", "e4m3"][int(rng.integers(3))]
        check_gemm(M, N * 16 if out == "e4m3" and N < 90 else (max(16, N // 16 * 16) if out == "e4m3" else N), 16 * K, out,
                   bool(rng.integers(2)), int(rng.integers(2)), int(rng.integers(1000)))


# ------------------------------------------------------------------ streams, graphs, no rows
def ffn(x, add, gain, dev_w1, dev_w2, bufs):
    """Norm, up-projection with GELU, down-projection: the run of calls that a serving loop makes."""
    h = H()
    h.hero_rms_norm_fp8(x, add, gain, bufs["sum"], bufs["n"], bufs["n_s"])
    h.hero_gemm_fp8(bufs["n"], bufs["n_s"], *dev_w1, bufs["u"], bufs["u_s"], act=1)
    h.hero_gemm_fp8(bufs["u"], bufs["u_s"], *dev_w2, bufs["y"])
    return bufs["y"]


def ffn_case(rows, D, F, seed):
    rng = np.random.default_rng(seed)
    host = dict(x=values(rng, rows, D, "bf16", 0.5), add=values(rng, rows, D, "bf16", 0.0), gain=values(rng, 1, D, "bf16")[0])
    weights = []
    for n, k in ((F, D), (D, F)):
        w = to_dev(S.round_bf16(rng.standard_normal((n, k)).astype(np.float32) / np.float32(np.sqrt(k))), "bf16")
        q, s = new((n, k), "e4m3"), new((R.blocks(n), R.blocks(k)), "fp32")
        H().hero_quantize_fp8(w, q, s, 128)
        weights.append((q, s, to_dev(S.round_bf16(rng.standard_normal(n).astype(np.float32) * 0.1), "bf16")))
    bufs = dict(sum=new((rows, D), "bf16"), n=new((rows, D), "e4m3"), n_s=new((rows, R.blocks(D)), "fp32"), u=new((rows, F), "e4m3"),
                u_s=new((rows, R.blocks(F)), "fp32"), y=new((rows, D), "bf16"))
    return host, [to_dev(host[k], "bf16") for k in ("x", "add", "gain")], weights, bufs


@pytest.mark.parametrize("rows,D,F", [(1, 256, 1024), (33, 400, 912), (310, 512, 2048), (1200, 1152, 4608)])
def test_ffn_together(rows, D, F):
    host, dev, (w1, w2), bufs = ffn_case(rows, D, F, rows)
    y = to_host(ffn(*dev, w1, w2, bufs))
    # each product on what the call before it wrote
    _, n = R.rms_norm(host["x"], host["add"], host["gain"], 1e-5)
    R.check_quantized(host32(bufs["n"]), host32(bufs["n_s"]).astype(np.float64), n, RMS_ERR * np.abs(n))
    t1 = [host32(t) for t in w1]
    u, err = R.gemm(host32(bufs["n"]), host32(bufs["n_s"]), *t1, 1)
    R.check_quantized(host32(bufs["u"]), host32(bufs["u_s"]).astype(np.float64), u, err)
    t2 = [host32(t) for t in w2]
    want, err = R.gemm(host32(bufs["u"]), host32(bufs["u_s"]), *t2, 0)
    assert (np.abs(y - want) <= err + R.HALF["bf16"] * (np.abs(want) + err)).all()


def test_two_streams_at_once_and_a_replayed_graph():
    cases = [ffn_case(rows, 512, 2048, 40 + rows) for rows in (1, 310)]
    alone = [ffn(*dev, w1, w2, bufs).clone() for _, dev, (w1, w2), bufs in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (_, dev, (w1, w2), bufs) in zip(streams, cases):
            with torch.cuda.stream(st):
                ffn(*dev, w1, w2, bufs)
    torch.cuda.synchronize()
    for want, (_, _, _, bufs) in zip(alone, cases):
        assert torch.equal(bufs["y"], want)
    # both captured, replayed on two streams at once, on inputs that changed after the capture
    graphs = []
    for _, dev, (w1, w2), bufs in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ffn(*dev, w1, w2, bufs)
        graphs.append(g)
    for _, dev, _, bufs in cases:
        dev[0].mul_(-1)
        dev[1].mul_(-1)
        bufs["y"].fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(3):
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for _, dev, (w1, w2), bufs in cases:
        replayed = bufs["y"].clone()
        assert torch.equal(ffn(*dev, w1, w2, bufs), replayed)
    H().hero_isolated_status()


def test_calls_wait_for_the_work_in_front_of_them_on_their_stream():
    """Inputs written, and outputs read, by kernels right before and after on a side stream."""
    _, dev, (w1, w2), bufs = ffn_case(310, 512, 2048, 3)
    want = ffn(*dev, w1, w2, bufs).clone()
    x, kept = dev[0], dev[0].clone()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        for _ in range(20):
            x.fill_(float("nan"))
            x.copy_(kept)
            got = ffn(*dev, w1, w2, bufs).clone()
            bufs["u"].view(torch.uint8).fill_(0x7F)
            bufs["n_s"].fill_(float("nan"))
            st.synchronize()
            assert torch.equal(got, want)


def test_no_rows():
    w = torch.zeros(32, 64, device="cuda", dtype=F8)
    f = lambda *shape: torch.zeros(*shape, device="cuda")  # noqa: E731
    H().hero_gemm_fp8(torch.zeros(0, 64, device="cuda", dtype=F8), f(0, 1), w, f(1, 1), None, f(0, 32))
    H().hero_quantize_fp8(f(0, 64), torch.zeros(0, 64, device="cuda", dtype=F8), f(0, 1))
    H().hero_rms_norm(f(0, 64), None, None, None, f(0, 64))
    H().hero_gather_ln_modulate_fp8(f(2, 5, 64), None, torch.zeros(0, device="cuda", dtype=torch.int32), f(2, 64), f(2, 64),
                                    torch.zeros(2, 0, 64, device="cuda", dtype=F8), f(2, 0, 1))
    torch.cuda.synchronize()


def test_the_binding_refuses_other_strides_types_and_shapes():
    h = H()
    x = torch.zeros(8, 128, device="cuda", dtype=torch.bfloat16)
    q, s = new((8, 128), "e4m3"), new((8, 1), "fp32")
    for bad in (lambda: h.hero_quantize_fp8(x.t(), new((128, 8), "e4m3"), new((128, 1), "fp32")),
                lambda: h.hero_quantize_fp8(x, q, s[:4]), lambda: h.hero_quantize_fp8(x, x, s),
                lambda: h.hero_quantize_fp8(x[:, ::2], q[:, :64].contiguous(), s),
                lambda: h.hero_rms_norm(x, x.float(), None, None, torch.empty_like(x)),
                lambda: h.hero_rms_norm(x, None, x[0, :64], None, torch.empty_like(x)),
                lambda: h.hero_gemm_fp8(q, s, q, s[:1], None, torch.zeros(8, 9, device="cuda")),
                lambda: h.hero_gemm_fp8(q, s, q, s[:1], None, q.clone()),              # e4m3 result without scales
                lambda: h.hero_gemm_fp8(q, s.bfloat16(), q, s[:1], None, torch.zeros(8, 8, device="cuda"))):
        with pytest.raises(h.HeroError):
            bad()


# ------------------------------------------------------------------ the FFN branch of a refresh block in 8 bits
def test_refresh_ffn_branch_in_8_bits():
    """Gather + LayerNorm + modulate, FFN-up with GELU, FFN-down, scatter into the feature cache, on a drawn list, against the
    oracle's LayerNorm and the plain product on what each call before wrote."""
    B, N, D, F, n_sel = 2, 307, 256, 768, 77
    rng = np.random.default_rng(4)
    x = values(rng, B * N, D, "bf16", 0.3).reshape(B, N, D)
    add = values(rng, B * N, D, "bf16", 0.0).reshape(B, N, D)
    idx = np.sort(rng.choice(N, n_sel, replace=False)).astype(np.int32)
    mod = (0.3 * rng.standard_normal((B, 2 * D))).astype(np.float32)
    mod_d, idx_d = torch.from_numpy(mod).cuda(), torch.from_numpy(idx).cuda()
    _, _, (w1, w2), _ = ffn_case(1, D, F, 11)
    n, n_s = new((B, n_sel, D), "e4m3"), new((B, n_sel, R.blocks(D)), "fp32")
    u, u_s = new((B * n_sel, F), "e4m3"), new((B * n_sel, R.blocks(F)), "fp32")
    y, cache = new((B, n_sel, D), "bf16"), torch.zeros(B, N, D, device="cuda", dtype=torch.bfloat16)
    h = H()
    h.hero_gather_ln_modulate_fp8(to_dev(x, "bf16"), to_dev(add, "bf16"), idx_d, mod_d[:, :D], mod_d[:, D:], n, n_s)
    h.hero_gemm_fp8(n.view(-1, D), n_s.view(-1, R.blocks(D)), *w1, u, u_s, act=1)
    h.hero_gemm_fp8(u, u_s, *w2, y.view(-1, D))
    h.hero_scatter_rows(y, idx_d, cache)
    cfg = O.Config(n_blocks=1, n_shallow=1, hidden=D, n_heads=1, head_dim=D, ffn_dim=8, temb_dim=8, batch=B, frames=1, grid_h=1,
                   grid_w=1, n_text=0, patch_h=1, patch_w=1, ratio_num=1, ratio_den=1)
    for b in range(B):
        rows = x[b, idx].astype(np.float64) + add[b, idx].astype(np.float64)
        want = O.layernorm_modulate(cfg, rows, mod[b, :D].astype(np.float64), mod[b, D:].astype(np.float64))
        sd = np.sqrt(rows.var(-1, keepdims=True) + 1e-5)
        err = 120 * 2.0 ** -24 * (2 * np.abs(rows).max(-1, keepdims=True) / sd * (1 + np.abs(mod[b, D:])) + np.abs(want))
        R.check_quantized(host32(n[b]), host32(n_s[b]).astype(np.float64), want, err)
    up, err = R.gemm(host32(n).reshape(-1, D), host32(n_s).reshape(-1, R.blocks(D)), *[host32(t) for t in w1], 1)
    R.check_quantized(host32(u), host32(u_s).astype(np.float64), up, err)
    down, err = R.gemm(host32(u), host32(u_s), *[host32(t) for t in w2], 0)
    got = to_host(cache)
    assert (np.abs(got[:, idx].reshape(-1, D) - down) <= err + R.HALF["bf16"] * (np.abs(down) + err)).all()
    assert (np.delete(got, idx, 1) == 0).all()
