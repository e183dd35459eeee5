"""Every variant of the 8-bit product that the rule on sizes chooses, against the product in 64 bits: scales that differ from block to
block, so that one that is stale, swapped or shifted shows."""
import pytest
import torch

from tests import fp8_ref as R

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "e4m3": F8}


def H():
    import paper_2508_17588_b200 as h
    return h


def new(shape, dtype):
    """An output that holds NaN (e4m3: the byte of NaN) until it is written."""
    t = torch.empty(shape, device="cuda", dtype=TORCH[dtype])
    (t.view(torch.uint8).fill_(0x7F) if dtype == "e4m3" else t.fill_(float("nan")))
    return t


def operands(M, N, K, seed, bias=True):
    """Random e4m3 numbers and, per block, random scales that span a factor of about 50."""
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    a, w = ((60.0 * normal(r, K)).clamp(-448, 448).to(F8) for r in (M, N))
    a_s, w_s = 0.01 * torch.exp(normal(M, R.blocks(K))), 0.001 * torch.exp(normal(R.blocks(N), R.blocks(K)))
    return a, a_s, w, w_s, normal(N).bfloat16() if bias else None


def product(a, a_s, w, w_s, bias):
    """(result, error of an fp32 evaluation in front of the last rounding) in 64 bits; the error as in fp8_ref.gemm: 128 additions of a
    block that each lose a unit in the last place, one multiply-add a block with a factor rounded once, the bias' addition."""
    M, K = a.shape
    N = w.shape[0]
    c, size = (torch.zeros(M, N, device="cuda", dtype=torch.float64) for _ in range(2))
    for j in range(R.blocks(K)):
        part = slice(j * R.BLOCK, (j + 1) * R.BLOCK)
        left = a[:, part].double() * a_s[:, j:j + 1].double()
        right = w[:, part].double() * w_s[:, j].double().repeat_interleave(R.BLOCK)[:N, None]
        c.addmm_(left, right.T)
        size.addmm_(left.abs(), right.abs().T)
    err = (128 + R.blocks(K) + 2) * 2.0 ** -23 * size
    if bias is not None:
        c += bias.double()
        err += 2.0 ** -23 * c.abs()
    return c, err


def call(dev, out, act=0):
    M, N = dev[0].shape[0], dev[2].shape[0]
    c, c_scale = new((M, N), out), new((M, R.blocks(N)), "fp32") if out == "e4m3" else None
    H().hero_gemm_fp8(*dev, c, c_scale, act)
    H().hero_isolated_status()
    return c, c_scale


def check(got, want, err, out):
    c, c_scale = got
    if out == "e4m3":
        R.check_quantized(c.float().cpu().numpy(), c_scale.double().cpu().numpy(), want.cpu().numpy(), err.cpu().numpy())
    else:
        off, tol = (c.double() - want).abs(), err + R.HALF[out] * (want.abs() + err)
        assert bool((off <= tol).all()), float((off / tol).max())


# Rows that end inside a tile, columns that end inside a block, K that ends inside a block and, where it is shared, is no multiple of the
# thread blocks'; of each variant a short K and one that takes a thread block through more than two windows of 16 blocks of scales.
# (tile, thread blocks per tile, exchanged), M, N, K
WIDE = [  # any result
    ((16, 1, True), 5, 272, 272), ((16, 1, True), 19, 6416, 4272), ((16, 2, True), 3, 1136, 1104), ((16, 2, True), 7, 7312, 9056),
    ((16, 4, True), 3, 1424, 1888), ((16, 4, True), 6, 3216, 16960), ((16, 8, True), 13, 144, 9040), ((16, 8, True), 17, 400, 9040),
    ((128, 1, False), 51, 9584, 176), ((128, 1, False), 33, 9776, 4896), ((128, 2, False), 49, 6000, 1808), ((128, 2, False), 39, 4752, 9552),
    ((128, 4, False), 36, 2096, 3920), ((128, 4, False), 33, 2352, 18000)]
RAGGED = [  # rows that start anywhere: bf16 and fp32
    ((16, 1, True), 5, 141, 144), ((16, 2, True), 2, 1121, 1104), ((16, 4, True), 2, 1401, 1888), ((16, 8, True), 9, 143, 9040),
    ((64, 1, False), 371, 1401, 656), ((64, 1, False), 515, 1811, 4368), ((64, 2, False), 50, 1561, 1376), ((64, 2, False), 33, 4559, 8512),
    ((64, 4, False), 150, 301, 1040), ((64, 4, False), 168, 141, 17552), ((128, 1, False), 51, 9589, 176), ((128, 1, False), 1753, 1001, 1040),
    ((128, 2, False), 49, 5997, 1808), ((128, 4, False), 36, 2101, 3920)]
NARROW = [  # rows on multiples of 16 bytes, tiles of 64 columns: bf16 and fp32
    ((64, 1, False), 371, 2304, 768), ((64, 1, False), 371, 1400, 656), ((64, 2, False), 50, 1560, 1376), ((64, 4, False), 150, 312, 1040)]
CASES = ([(*c, out) for c in WIDE for out in ("bf16", "fp32", "e4m3")] + [(*c, out) for c in RAGGED + NARROW for out in ("bf16", "fp32")])


def plan_of(M, N, K, out):
    columns, ctas, swap = H().hero_plan_fp8_gemm(M, N, K, out == "e4m3")
    return columns, ctas, swap


@pytest.mark.parametrize("plan,M,N,K,out", CASES)
def test_one_tile_a_thread_block(plan, M, N, K, out):
    assert plan_of(M, N, K, out) == plan
    dev = operands(M, N, K, M * 7 + N * 3 + K)
    check(call(dev, out), *product(*dev), out)


# More tiles (of 256 x 256) than pairs of SMs, so that a pair goes on to a second one; blocks of K just below, at and above one, two and more
# windows of scales.
@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("K", [1920, 2032, 2048, 2064, 2176, 4080, 4096, 4112, 12288, 12304])
def test_pairs_windows_of_scales(K, out):
    M, N = 2600, 2608
    assert plan_of(M, N, K, out) == (256, 0, False)
    dev = operands(M, N, K, K)
    check(call(dev, out), *product(*dev), out)


@pytest.mark.parametrize("out", ["bf16", "fp32"])
@pytest.mark.parametrize("N", [2601, 2604])
def test_pairs_rows_that_start_anywhere(N, out):
    M, K = 2601, 4112
    assert plan_of(M, N, K, out) == (256, 0, False)
    dev = operands(M, N, K, N, bias=False)
    check(call(dev, out), *product(*dev), out)


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
def test_pairs_what_is_not_finite_stays_in_its_row(out):
    """NaN among a row's values and among another's scales, in windows of scales behind the first: every other row bit for bit as
    without them."""
    M, N, K = 2600, 2608, 4112
    dev = operands(M, N, K, 5)
    a, a_s = dev[0].clone(), dev[1].clone()
    a.view(torch.uint8)[1999, 2500] = 0x7F
    a_s[2000, 32] = float("nan")
    clean, dirty = call(dev, out), call((a, a_s, *dev[2:]), out)
    hit = torch.zeros(M, dtype=torch.bool, device="cuda")
    hit[1999:2001] = True
    for t, u in zip(clean, dirty):
        if t is not None:
            assert bool(torch.isnan(u[hit].float()).all()) and bool(torch.isfinite(t.float()).all())
            assert torch.equal(t[~hit].float(), u[~hit].float())


@pytest.mark.parametrize("M,N,K", [(17, 400, 9040), (39, 4752, 9552), (33, 2352, 18000), (515, 1811, 4368), (2600, 2608, 4112)])
def test_long_sums_repeat_bit_for_bit(M, N, K):
    dev = operands(M, N, K, 3)
    first = call(dev, "fp32")[0]
    for _ in range(5):
        assert torch.equal(first, call(dev, "fp32")[0])


@pytest.mark.parametrize("out", ["bf16", "fp32", "e4m3"])
@pytest.mark.parametrize("which", ["row", "columns"])
def test_what_these_tests_would_notice(which, out):
    """One scale of the plain product taken from the window before: the kernel's result is outside the tolerances."""
    a, a_s, w, w_s, bias = operands(70, 272, 4112, 1)
    got = call((a, a_s, w, w_s, bias), out)
    check(got, *product(a, a_s, w, w_s, bias), out)
    if which == "row":
        a_s = a_s.clone()
        a_s[41, 20] = a_s[41, 4]
    else:
        w_s = w_s.clone()
        w_s[1, 32] = w_s[1, 0]
    with pytest.raises(AssertionError):
        check(got, *product(a, a_s, w, w_s, bias), out)
