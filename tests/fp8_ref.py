"""Plain statements of the 8-bit operators in 64 bits (numpy), for the parity tests."""
import math

import numpy as np
import torch

BLOCK = 128
FLOOR = 2.0 ** -126
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -4}     # half a step, relative to the value
SUBNORMAL = 2.0 ** -10                                                # half of e4m3's smallest step


def blocks(n):
    return -(-n // BLOCK)


def block_scale32(v, block_rows):
    """The scales as the definition rounds them: amax * fp32(1 / 448) in fp32, at least 2^-126, NaN for a block that is not finite."""
    rows, cols = v.shape
    s = np.empty((-(-rows // block_rows), blocks(cols)), np.float32)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            amax = np.abs(v[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]).max().astype(np.float32)
            s[i, j] = max(amax * np.float32(1.0 / 448.0), np.float32(FLOOR)) if np.isfinite(amax) else np.nan
    return s


def spread(scale, block_rows, rows, cols):
    """A scale per element."""
    return np.repeat(np.repeat(scale, block_rows, 0)[:rows], BLOCK, 1)[:, :cols]


def quantize32(v, block_rows):
    """(q as fp32 numbers, scale): the definition in fp32 step by step, which the kernels follow bit for bit on given inputs."""
    v = v.astype(np.float32)
    s = block_scale32(v, block_rows)
    with np.errstate(all="ignore"):
        scaled = v * (np.float32(1.0) / spread(s, block_rows, *v.shape)).astype(np.float32)
    return torch.from_numpy(scaled).to(torch.float8_e4m3fn).float().numpy(), s


def dequantize(q, scale, block_rows):
    return q.astype(np.float64) * spread(scale.astype(np.float64), block_rows, *q.shape)


def rms_norm(x, add, gain, eps):
    h = x.astype(np.float64) + (0.0 if add is None else add.astype(np.float64))
    y = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h, y if gain is None else y * gain.astype(np.float64)


def gelu(t):
    return 0.5 * t * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (t + 0.044715 * t ** 3)))


def gemm(a, a_scale, w, w_scale, bias, act):
    """(result, error of an fp32 evaluation in front of the last rounding) of the block-scaled product, from dequantised operands.

    The error: at most 128 additions inside a block that each lose a unit in the last place of fp32 (2^-23: nothing says that the
    tensor core rounds to nearest) and one multiply-add per block, of terms whose magnitudes sum up to |A| |W|; the bias' addition.
    GELU has a slope below 1.13 and, evaluated in fp32, an error of 2^-20 of its argument (the exponential's argument is at most 40
    where it matters and carries 2^-24 of itself); what bf16 results take, the hardware's tanh, adds half of 2^-10 of it."""
    A, W = dequantize(a, a_scale, 1), dequantize(w, w_scale, BLOCK)
    c = A @ W.T
    err = (128 + blocks(a.shape[1]) + 2) * 2.0 ** -23 * (np.abs(A) @ np.abs(W).T)
    if bias is not None:
        c = c + bias.astype(np.float64)
        err = err + 2.0 ** -23 * np.abs(c)
    if act:
        t = c
        c = gelu(t)
        err = 1.13 * err + (2.0 ** -20 + 2.0 ** -11) * np.abs(t)
    return c, err


def check_quantized(q, scale, want, err):
    """e4m3 values with a scale per row and 128 columns against 64-bit values that an fp32 evaluation has to `err`."""
    rows, cols = want.shape
    amax = np.zeros((rows, blocks(cols)))
    room = np.zeros_like(amax)
    for j in range(blocks(cols)):
        piece = slice(j * BLOCK, (j + 1) * BLOCK)
        amax[:, j], room[:, j] = np.abs(want[:, piece]).max(1), err[:, piece].max(1)
    # the scale: the largest magnitude is off by at most the largest error, and three roundings follow
    assert (np.abs(scale - np.maximum(amax / 448.0, FLOOR)) <= room / 448.0 + 4 * 2.0 ** -24 * amax / 448.0 + 2e-45).all()
    # a value: half a step of e4m3 on what is scaled, half of the smallest step, the error, and the roundings of scale and inverse
    got = dequantize(q, scale, 1)
    tol = (HALF["e4m3"] + 2.0 ** -20) * (np.abs(want) + err) + SUBNORMAL * 1.001 * spread(scale.astype(np.float64), 1, rows, cols) + err
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
