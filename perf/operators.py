"""Performance cases of the 8-bit linear path: the operators that feed, and are, a matrix product in e4m3 with a scale
for each block of 128.

  gemm       `hero_gemm_fp8`: C = act(A W^T + bias), A with a scale per row and 128 columns, W with one per 128 x 128;
             C in bf16, in fp32, or in e4m3 with scales of its own (what the next product reads).
  rms        `hero_rms_norm` / `hero_rms_norm_fp8`: residual addition and root-mean-square norm, the output in the
             input's type or in e4m3 with a scale for each 128 columns of a row.
  quantize   `hero_quantize_fp8`: a matrix to e4m3, blocks of 1 x 128 (activations) or 128 x 128 (weights).
  gather_ln  `hero_gather_ln_modulate_fp8`: the refreshed rows gathered, normalised and modulated, in e4m3 with scales.

A scale is max(largest magnitude / 448, 2^-126), a value is stored as the nearest e4m3 to value * (1 / scale).  Inputs:
weights N(0, 0.02^2), activations N(0, 1) with a spread of magnitudes between rows, as after a few residual blocks.
"""
import math

import torch

own = False

BLOCK = 128
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
SCALE_FLOOR = 2.0 ** -126
_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": E4M3}
_BYTES = {"bf16": 2, "fp32": 4, "e4m3": 1}


def listed():
    return [
        # One row through the up-projection of the 5B video block: a single conditioning token, weights read once.
        dict(name="gemm_row1", op="gemm", m=1, n=12288, k=3072, bias=True, act=1, out="bf16"),
        # The QKV projection of a small one-frame model, 371 refreshed rows of width 768.
        dict(name="gemm_rows371", op="gemm", m=371, n=2304, k=768, bias=True, act=0, out="bf16"),
        # Odd everything: a width that ends inside a block of 128 and a column count that is no multiple of anything,
        # in fp32 for a numerics run.
        dict(name="gemm_ragged", op="gemm", m=1753, n=1001, k=1040, bias=False, act=0, out="fp32"),
        # FFN-up of a refresh block of the 5B video model at 25 %, GELU, written in 8 bits for FFN-down.
        dict(name="gemm_ffn_up", op="gemm", m=8774, n=12288, k=3072, bias=True, act=1, out="e4m3"),
        # FFN-down of the same block.
        dict(name="gemm_ffn_down", op="gemm", m=8774, n=3072, k=12288, bias=True, act=0, out="bf16"),
        # One row: the norm in front of gemm_row1.
        dict(name="rms_row1", op="rms", rows=1, d=3072, dtype="bf16", add=True, gain=True, keep=True, out="e4m3"),
        # An fp32 model of width 1152, one latent frame of 34 x 51 tokens, norm without quantisation.
        dict(name="rms_fp32_1734", op="rms", rows=1734, d=1152, dtype="fp32", add=True, gain=True, keep=True, out="fp32"),
        # Every row of the guidance pair of the 5B video model: residual written back, output in 8 bits.
        dict(name="rms_full", op="rms", rows=35552, d=3072, dtype="bf16", add=True, gain=True, keep=True, out="e4m3"),
        # The weights of an FFN-up, once at load.
        dict(name="quantize_weights", op="quantize", rows=12288, cols=3072, block_rows=128, dtype="bf16"),
        # The attention's output of a refresh block at 25 %, before the out-projection.
        dict(name="quantize_rows", op="quantize", rows=8774, cols=3072, block_rows=1, dtype="bf16"),
        # The prologue of a small fp32 model's refresh: 310 of 1319 rows of the pair.
        dict(name="gather_ln_fp32", op="gather_ln", batch=2, n=1319, n_sel=310, d=512, dtype="fp32", add=False),
        # The FFN branch's prologue of a refresh block of the 5B video model at 25 %.
        dict(name="gather_ln_video", op="gather_ln", batch=2, n=17776, n_sel=4387, d=3072, dtype="bf16", add=True),
    ]


def _log(rng, low, high):
    """A whole number from low to high, spread over its logarithm."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["gemm", "gemm", "gemm", "rms", "quantize", "gather_ln"])
    if op == "gemm":
        out = rng.choice(["bf16", "bf16", "fp32", "e4m3"])
        m, k = _log(rng, 1, 9000), 16 * _log(rng, 4, 768)
        n = 16 * _log(rng, 4, 768) if out == "e4m3" else _log(rng, 64, 12288)
        return dict(op=op, m=m, n=n, k=k, bias=rng.random() < 0.7, act=rng.randint(0, 1), out=out)
    if op == "rms":
        dtype = rng.choice(["bf16", "fp32"])
        return dict(op=op, rows=_log(rng, 1, 20000), d=16 * rng.randint(4, 256), dtype=dtype, add=rng.random() < 0.7,
                    gain=rng.random() < 0.8, keep=rng.random() < 0.7, out=rng.choice([dtype, "e4m3"]))
    if op == "quantize":
        return dict(op=op, rows=_log(rng, 1, 12000), cols=16 * rng.randint(4, 256), block_rows=rng.choice([1, 128]),
                    dtype=rng.choice(["bf16", "fp32"]))
    n = _log(rng, 8, 17776)
    return dict(op=op, batch=rng.randint(1, 3), n=n, n_sel=max(1, int(n * rng.uniform(0.05, 0.6))), d=16 * rng.randint(4, 192),
                dtype=rng.choice(["bf16", "fp32"]), add=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _blocks(n):
    return -(-n // BLOCK)


def _rows(gen, rows, cols):
    """Activations: N(0, 1) times a magnitude of the row's own."""
    x = torch.randn(rows, cols, device="cuda", generator=gen)
    return x * torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=gen))


def _by_rows(x):
    """x in e4m3 with a scale per row and 128 columns (the last block of a row may be shorter)."""
    rows, cols = x.shape
    padded = torch.nn.functional.pad(x, (0, _blocks(cols) * BLOCK - cols)).view(rows, -1, BLOCK)
    amax = padded.abs().amax(-1)
    scale = torch.where(torch.isfinite(amax), (amax / E4M3_MAX).clamp_min(SCALE_FLOOR), math.nan)
    q = (padded * (1.0 / scale).unsqueeze(-1)).view(rows, -1)[:, :cols]
    return q.to(E4M3).contiguous(), scale


def _by_tiles(x):
    """x in e4m3 with a scale per 128 x 128 elements."""
    rows, cols = x.shape
    br, bc = _blocks(rows), _blocks(cols)
    padded = torch.nn.functional.pad(x, (0, bc * BLOCK - cols, 0, br * BLOCK - rows)).view(br, BLOCK, bc, BLOCK)
    amax = padded.abs().amax((1, 3))
    scale = torch.where(torch.isfinite(amax), (amax / E4M3_MAX).clamp_min(SCALE_FLOOR), math.nan)
    q = (padded * (1.0 / scale).view(br, 1, bc, 1)).view(br * BLOCK, bc * BLOCK)[:rows, :cols]
    return q.to(E4M3).contiguous(), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *shape, dtype: torch.empty(*shape, device="cuda", dtype=dtype)  # noqa: E731
    s = dict(case)
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"], s["a_scale"] = _by_rows(_rows(gen, m, k))
        s["w"], s["w_scale"] = _by_tiles(0.02 * torch.randn(n, k, device="cuda", generator=gen))
        s["b"] = (0.02 * torch.randn(n, device="cuda", generator=gen)).bfloat16() if case["bias"] else None
        s["c"] = new(m, n, dtype=_DTYPES[case["out"]])
        s["c_scale"] = new(m, _blocks(n), dtype=torch.float32) if case["out"] == "e4m3" else None
        return s
    dt = _DTYPES[case["dtype"]]
    if case["op"] == "rms":
        rows, d = case["rows"], case["d"]
        s["x"] = _rows(gen, rows, d).to(dt)
        s["r"] = torch.randn(rows, d, device="cuda", generator=gen).to(dt) if case["add"] else None
        s["g"] = (1.0 + 0.1 * torch.randn(d, device="cuda", generator=gen)).to(dt) if case["gain"] else None
        s["sum"] = new(rows, d, dtype=dt) if case["keep"] else None
        s["y"] = new(rows, d, dtype=_DTYPES[case["out"]])
        s["y_scale"] = new(rows, _blocks(d), dtype=torch.float32) if case["out"] == "e4m3" else None
    elif case["op"] == "quantize":
        rows, cols, br = case["rows"], case["cols"], case["block_rows"]
        s["x"] = (_rows(gen, rows, cols) if br == 1 else 0.02 * torch.randn(rows, cols, device="cuda", generator=gen)).to(dt)
        s["y"] = new(rows, cols, dtype=E4M3)
        s["y_scale"] = new(rows if br == 1 else _blocks(rows), _blocks(cols), dtype=torch.float32)
    else:
        b, n, d, n_sel = case["batch"], case["n"], case["d"], case["n_sel"]
        s["x"] = _rows(gen, b * n, d).view(b, n, d).to(dt)
        s["r"] = torch.randn(b, n, d, device="cuda", generator=gen).to(dt) if case["add"] else None
        order = torch.randperm(n, device="cuda", generator=gen)[:n_sel]
        s["idx"] = torch.sort(order).values.to(torch.int32)
        mod = 0.3 * torch.randn(b, 4 * d, device="cuda", generator=gen)        # shift | scale | the other branch's
        s["shift"], s["scale"] = mod[:, :d], mod[:, d:2 * d]
        s["y"] = new(b, n_sel, d, dtype=E4M3)
        s["y_scale"] = new(b, n_sel, _blocks(d), dtype=torch.float32)
    return s


# ------------------------------------------------------------------ one pass
_EPS = 1e-5


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2508_17588_b200 as H
    if s["op"] == "gemm":
        H.hero_gemm_fp8(s["a"], s["a_scale"], s["w"], s["w_scale"], s["b"], s["c"], s["c_scale"], act=s["act"])
        return {"c": s["c"], "c_scale": s["c_scale"]}
    if s["op"] == "rms":
        if s["out"] == "e4m3":
            H.hero_rms_norm_fp8(s["x"], s["r"], s["g"], s["sum"], s["y"], s["y_scale"], _EPS)
        else:
            H.hero_rms_norm(s["x"], s["r"], s["g"], s["sum"], s["y"], _EPS)
        return {"sum": s["sum"], "y": s["y"], "y_scale": s["y_scale"]}
    if s["op"] == "quantize":
        H.hero_quantize_fp8(s["x"], s["y"], s["y_scale"], s["block_rows"])
    else:
        H.hero_gather_ln_modulate_fp8(s["x"], s["r"], s["idx"], s["shift"], s["scale"], s["y"], s["y_scale"])
    return {"y": s["y"], "y_scale": s["y_scale"]}


def _plain(s):
    if s["op"] == "gemm":
        n, k = s["n"], s["k"]
        a = s["a"].float() * s["a_scale"].repeat_interleave(BLOCK, 1)[:, :k]
        w = s["w"].float() * s["w_scale"].repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]
        c = a @ w.T
        if s["b"] is not None:
            c = c + s["b"].float()
        if s["act"]:
            c = 0.5 * c * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (c + 0.044715 * c ** 3)))
        if s["out"] == "e4m3":
            c, c_scale = _by_rows(c)
            return {"c": c, "c_scale": c_scale}
        return {"c": c.to(_DTYPES[s["out"]]), "c_scale": None}
    if s["op"] == "rms":
        h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + _EPS)
        if s["g"] is not None:
            y = y * s["g"].float()
        kept = h.to(_DTYPES[s["dtype"]]) if s["keep"] else None
        if s["out"] == "e4m3":
            q, scale = _by_rows(y)
            return {"sum": kept, "y": q, "y_scale": scale}
        return {"sum": kept, "y": y.to(_DTYPES[s["out"]]), "y_scale": None}
    if s["op"] == "quantize":
        q, scale = (_by_rows if s["block_rows"] == 1 else _by_tiles)(s["x"].float())
        return {"y": q, "y_scale": scale}
    h = s["x"][:, s["idx"].long()].float()
    if s["r"] is not None:
        h = h + s["r"][:, s["idx"].long()].float()
    h = h - h.mean(-1, keepdim=True)
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + _EPS) * (1.0 + s["scale"].unsqueeze(1)) + s["shift"].unsqueeze(1)
    b, n_sel, d = y.shape
    q, scale = _by_rows(y.view(b * n_sel, d))
    return {"y": q.view(b, n_sel, d), "y_scale": scale.view(b, n_sel, -1)}


def work(case):
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        scales = 4 * (m * _blocks(k) + _blocks(n) * _blocks(k) + (m * _blocks(n) if case["out"] == "e4m3" else 0))
        return {"bytes": m * k + n * k + m * n * _BYTES[case["out"]] + scales + (2 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    size = _BYTES[case["dtype"]]
    if case["op"] == "rms":
        rows, d = case["rows"], case["d"]
        each = size * (1 + case["add"] + case["keep"]) + _BYTES[case["out"]]
        scales = 4 * rows * _blocks(d) if case["out"] == "e4m3" else 0
        return {"bytes": rows * d * each + scales + (size * d if case["gain"] else 0), "flops": 4 * rows * d}
    if case["op"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        return {"bytes": rows * cols * (size + 1) + 4 * -(-rows // case["block_rows"]) * _blocks(cols), "flops": 3 * rows * cols}
    b, n_sel, d = case["batch"], case["n_sel"], case["d"]
    return {"bytes": b * n_sel * (d * (size * (1 + case["add"]) + 1) + 4 * _blocks(d)) + 4 * n_sel + 8 * b * d,
            "flops": 10 * b * n_sel * d}


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_quantized(v, block_rows):
    """Values and scales of a matrix in 64 bits, block by block of rows."""
    rows, cols = v.shape
    br, bc = -(-rows // block_rows), _blocks(cols)
    scale = torch.empty(br, bc, device=v.device, dtype=torch.float64)
    q = torch.empty(rows, cols, device=v.device, dtype=torch.float64)
    for j in range(bc):
        piece = v[:, j * BLOCK:(j + 1) * BLOCK]
        largest = piece.abs().max(dim=1).values
        if block_rows > 1:
            largest = torch.stack([p.max() for p in largest.split(block_rows)])
        scale[:, j] = torch.clamp(largest / 448.0, min=SCALE_FLOOR)
        of_row = scale[:, j].repeat_interleave(block_rows)[:rows].unsqueeze(1)
        q[:, j * BLOCK:(j + 1) * BLOCK] = _nearest_e4m3(piece / of_row)
    return q, scale


def _nearest_e4m3(v):
    """The nearest number with three bits behind the leading one (exponents from -6 on), ties to even, in 64 bits."""
    exponent = torch.clamp(torch.frexp(v).exponent - 1, min=-6)
    step = torch.ldexp(torch.ones_like(v), exponent - 3)
    return torch.clamp(torch.round(v / step) * step, -448.0, 448.0)


def exact(case, seed):
    s = prepare(case, seed)
    f64 = lambda t: t.to(torch.float64)  # noqa: E731
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        c = torch.zeros(m, n, device="cuda", dtype=torch.float64)
        tile_of = torch.arange(n, device="cuda") // BLOCK
        for j in range(_blocks(k)):
            part = slice(j * BLOCK, (j + 1) * BLOCK)
            left = f64(s["a"][:, part]) * f64(s["a_scale"][:, j:j + 1])
            right = f64(s["w"][:, part]) * f64(s["w_scale"][:, j])[tile_of].unsqueeze(1)
            c.addmm_(left, right.T)
        if s["b"] is not None:
            c += f64(s["b"])
        if case["act"]:
            inner = math.sqrt(2.0 / math.pi) * (c + 0.044715 * c * c * c)
            c = c / (1.0 + torch.exp(-2.0 * inner))
        if case["out"] != "e4m3":
            return {"c": c, "c_scale": None}
        q, scale = _exact_quantized(c, 1)
        return {"c": q, "c_scale": scale}
    if case["op"] == "quantize":
        q, scale = _exact_quantized(f64(s["x"]), case["block_rows"])
        return {"y": q, "y_scale": scale}
    if case["op"] == "rms":
        h = f64(s["x"])
        if s["r"] is not None:
            h = h + f64(s["r"])
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["d"] + _EPS)
        if s["g"] is not None:
            y = y * f64(s["g"])
        q, scale = _exact_quantized(y, 1) if case["out"] == "e4m3" else (y, None)
        return {"sum": h if case["keep"] else None, "y": q, "y_scale": scale}
    d = case["d"]
    out, scales = [], []
    for b in range(case["batch"]):
        h = f64(s["x"][b].index_select(0, s["idx"]))
        if s["r"] is not None:
            h = h + f64(s["r"][b].index_select(0, s["idx"]))
        var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
        y = (h - mean) / torch.sqrt(var + _EPS) * (1.0 + f64(s["scale"][b])) + f64(s["shift"][b])
        q, scale = _exact_quantized(y, 1)
        out.append(q)
        scales.append(scale)
    return {"y": torch.stack(out), "y_scale": torch.stack(scales)}
