"""Microscaled 4-bit floating point as timed cases: quantization of rows and its inverse, the decode product of 16-bit
activations with 4-bit weights, and the product of quantized activations with 4-bit weights.

Format.  A matrix of `rows` rows is cut along K into blocks of 32 or 16 values.  A value is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6
and their negatives) times its block's scale times its row's scale:
  block 32   the scale is a power of two (e8m0), 2^(floor(log2 max|block|) - 2); row scales are 1
  block 16   the scale is e4m3, round(max|block| / (6 r)); the row scale r is the least power of two with max|row| <= 2688 r
Roundings are to nearest, ties to even, and saturate.

A case is a dict of plain values:
  op      "roundtrip"  tman_quantize_rows_f4, then tman_dequant_rows_f4: rows as a 4-bit product sees them
          "dequant"    tman_dequant_rows_f4 of a stored weight matrix
          "gemv"       tman_mpgemv_f4: y = x . W^T, x in 16 bits, M in 1..8
          "linear"     tman_quantize_rows_f4 of x, then tman_mpgemm_f4: both operands in 4 bits
  M, K, N rows, reduction, output channels;  block 32 or 16;  dtype "f16" or "bf16" of x and y
  pad     values by which a row of x is longer than K (x is a slice of a wider matrix)
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
MAX_FLOPS = 2.0 * 8192 * 18944 * 3584      # the largest listed case
MAX_CELLS = 18944 * 3584                   # weights of its matrix


def listed():
    return [
        # One token's hidden state quantized and read back: the smallest call, launch cost.
        dict(name="roundtrip_m1_b32", op="roundtrip", M=1, K=4096, N=0, block=32, dtype="f16", pad=0),
        # A long prompt's activations in front of a down projection, as a slice of the wider gate-and-up output.
        dict(name="roundtrip_m2048_b16", op="roundtrip", M=2048, K=14336, N=0, block=16, dtype="bf16", pad=14336),
        # A stored weight matrix back in 16 bits, as a program that inspects, merges or exports weights asks for it.
        dict(name="dequant_14336x4096_b32", op="dequant", M=14336, K=4096, N=0, block=32, dtype="bf16", pad=0),
        # One token through the smallest projection of a layer (key or value): fixed costs of a decode call.
        dict(name="gemv_m1_4096x1024_b32", op="gemv", M=1, K=4096, N=1024, block=32, dtype="f16", pad=0),
        # One token through gate or up, the weights' bytes.
        dict(name="gemv_m1_4096x14336_b16", op="gemv", M=1, K=4096, N=14336, block=16, dtype="bf16", pad=0),
        # The widest decode batch through the long reduction of a down projection.
        dict(name="gemv_m8_14336x4096_b32", op="gemv", M=8, K=14336, N=4096, block=32, dtype="f16", pad=0),
        # Three sequences, a reduction that is no multiple of 128 and an odd number of channels.
        dict(name="gemv_m3_1040x1001_b16", op="gemv", M=3, K=1040, N=1001, block=16, dtype="f16", pad=8),
        # One token with both operands in 4 bits.
        dict(name="linear_m1_4096x14336_b16", op="linear", M=1, K=4096, N=14336, block=16, dtype="bf16", pad=0),
        # A batch just beyond the decode call's rows, or a very short prompt, ragged.
        dict(name="linear_m40_4096x14336_b32", op="linear", M=40, K=4096, N=14336, block=32, dtype="f16", pad=0),
        # An ordinary prompt of odd length through an attention projection.
        dict(name="linear_m777_3584x4608_b16", op="linear", M=777, K=3584, N=4608, block=16, dtype="f16", pad=0),
        # A long prompt through gate or up.
        dict(name="linear_m2048_3584x18944_b32", op="linear", M=2048, K=3584, N=18944, block=32, dtype="bf16", pad=0),
        # A long batch of prompts through the longest reduction.
        dict(name="linear_m8192_18944x3584_b16", op="linear", M=8192, K=18944, N=3584, block=16, dtype="f16", pad=0),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    op = rng.choice(("roundtrip", "dequant", "gemv", "gemv", "linear", "linear"))
    block = rng.choice((32, 16))
    c = dict(op=op, M=1, K=_log(rng, 8 * block, 18944, block), N=0, block=block, dtype=rng.choice(("f16", "bf16")),
             pad=rng.choice((0, 0, 8, 264)))
    if op in ("roundtrip", "dequant"):
        c["M"] = _log(rng, 1, min(16384, MAX_CELLS // c["K"]))
    else:
        c["N"] = _log(rng, 64, min(32768, MAX_CELLS // c["K"]), rng.choice((1, 8, 64)))
        c["M"] = rng.randint(1, 8) if op == "gemv" else _log(rng, 1, min(8192, int(MAX_FLOPS / (2.0 * c["K"] * c["N"]))))
    return c


# ---- the format in elementary operations, in the type of its arguments --------------------------------------------------


def _pow2(e):
    """2^e of an integer tensor of exponents in [-127, 127], exactly: the bits of a number of 32 bits."""
    e = e.to(torch.int32)
    return torch.where(e < -126, 1 << 22, (e + 127).clamp(min=1) << 23).view(torch.float32)


def _floor_log2(v):
    """floor(log2 v) of positive values, exactly."""
    return torch.frexp(v)[1] - 1


def _round_e2m1(v):
    """Codes of v: sign in bit 3, magnitude index below; nearest, ties to the even index, saturating."""
    a = v.abs()
    i = (a > 0.25).to(torch.uint8)
    for at, even_below in ((0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        i += (a > at) if even_below else (a >= at)
    return i | (torch.signbit(v).to(torch.uint8) << 3)


def _round_e4m3(v):
    """v >= 0 rounded to a value of e4m3 (448 at most)."""
    step = _pow2(torch.where(v > 0, _floor_log2(v), -6).clamp(-6, 8) - 3)
    return torch.clamp(torch.round(v / step) * step, max=448.0)


def _quantize(x, block):
    """Codes [rows][K], block scales [rows][K / block], row scales [rows] of x (32 bits)."""
    rows, K = x.shape
    b = x.view(rows, K // block, block)
    top = b.abs().amax(-1)
    if block == 32:
        e = torch.where(top > 0, _floor_log2(top) - 2, -127).clamp(min=-127)
        scale, r = _pow2(e), torch.ones(rows, device=x.device)
    else:
        m = top.amax(-1)
        e = _floor_log2(m) - 11
        r = torch.where(m > 0, _pow2((e + (m > 2688.0 * _pow2(e))).clamp(min=-126)), 1.0)
        scale = _round_e4m3(top / r[:, None] / 6.0)
    d = scale[..., None]
    v = torch.where(d > 0, b / r[:, None, None] / torch.where(d > 0, d, 1.0), 0.0)
    return _round_e2m1(v).view(rows, K), scale, r


def _values(codes, scale, r):
    """What codes and scales stand for, in the scales' type."""
    rows, K = codes.shape
    mags = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=scale.dtype, device=codes.device)
    v = mags[codes.long()].view(rows, scale.shape[1], -1) * scale[..., None] * r[:, None, None]
    return v.view(rows, K)


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _activations(case, g):
    """A normal hidden state with 1 % of channels 20 times as large, in a matrix whose rows are `pad` longer."""
    M, K = case["M"], case["K"]
    x = torch.randn(M, K + case["pad"], generator=g, device="cuda")
    loud = torch.randperm(K, generator=g, device="cuda")[: max(1, K // 100)]
    x[:, loud] *= 20.0
    return x.to(DTYPES[case["dtype"]])[:, :K]


def _weights(rows, K, block, g):
    """A weight matrix as a checkpoint holds it: codes two to a byte (the even k in the low half), scales, row scales."""
    codes, scale, r = _quantize(torch.randn(rows, K, generator=g, device="cuda") * 0.02, block)
    return {"codes": codes[:, 0::2] | (codes[:, 1::2] << 4), "scale": scale, "row_scale": r}


def _plain_codes(w):
    return torch.stack((w["codes"] & 15, w["codes"] >> 4), -1).flatten(1)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, M, K, N, block = (case[k] for k in ("op", "M", "K", "N", "block"))
    s = {"case": case, "dtype": DTYPES[case["dtype"]]}
    rows = M if op == "dequant" else N
    if op != "dequant":
        s["x"] = _activations(case, g)
    if rows:
        s["w"] = _weights(rows, K, block, g)
    out = (M, N) if N else (M, K)
    s["y"] = torch.empty(out, dtype=s["dtype"], device="cuda")
    if own:
        # what a program that serves a model keeps: the weights in the library's layout (laid out once, when the
        # checkpoint is loaded), the buffer that quantized activations go to, and a workspace
        from paper_2511_11248_b200 import binding as B
        if rows:
            w = s["w"]
            kind = torch.float8_e8m0fnu if block == 32 else torch.float8_e4m3fn
            s["packed"] = torch.empty(B.tman_packed_bytes_f4(rows, K, block), dtype=torch.uint8, device="cuda")
            B.tman_pack_f4(w["codes"], w["scale"].to(kind).view(torch.uint8), w["row_scale"], rows, K, block, s["packed"])
        if op in ("roundtrip", "linear"):
            s["a"] = torch.empty(B.tman_packed_bytes_f4(M, K, block), dtype=torch.uint8, device="cuda")
        which = {"gemv": B.OP_GEMV, "linear": B.OP_GEMM}.get(op, B.OP_AUX)
        s["ws"] = torch.empty(B.tman_workspace_bytes_f4(which, M, K, max(N, 1), block), dtype=torch.uint8, device="cuda")
        B.tman_workspace_init(s["ws"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    op, M, K, N, block = (c[k] for k in ("op", "M", "K", "N", "block"))
    if own:
        from paper_2511_11248_b200 import binding as B
        dt = B.DTYPE_F16 if c["dtype"] == "f16" else B.DTYPE_BF16
        y = s["y"]
        if op == "roundtrip":
            B.tman_quantize_rows_f4(s["x"], K + c["pad"], dt, M, K, block, s["a"])
            B.tman_dequant_rows_f4(s["a"], M, K, block, y, K, dt, s["ws"])
        elif op == "dequant":
            B.tman_dequant_rows_f4(s["packed"], M, K, block, y, K, dt, s["ws"])
        elif op == "gemv":
            B.tman_mpgemv_f4(s["packed"], s["x"], K + c["pad"], y, N, dt, M, K, N, block, s["ws"])
        else:
            B.tman_quantize_rows_f4(s["x"], K + c["pad"], dt, M, K, block, s["a"])
            B.tman_mpgemm_f4(s["packed"], s["a"], y, N, dt, M, K, N, block, s["ws"])
        return y
    if op == "roundtrip":
        return _values(*_quantize(s["x"].float(), block)).to(s["dtype"])
    w = _values(_plain_codes(s["w"]), s["w"]["scale"], s["w"]["row_scale"])
    if op == "dequant":
        return w.to(s["dtype"])
    x = s["x"].float()
    if op == "linear":
        x = _values(*_quantize(x, block))
    return (x @ w.T).to(s["dtype"])


def exact(case, seed):
    """The same from the definitions in 64 bits: scales from their closed forms, every value from the nearest entry of the
    table of all values that its block can hold."""
    s = prepare(case, seed)
    op, block = case["op"], case["block"]
    table = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")

    def binade(v):                                     # floor(log2 v): the exponent of a number of 64 bits
        return (v.view(torch.int64) >> 52) - 1023

    def two_to(e):
        return ((e + 1023) << 52).view(torch.float64)

    def quantized(x):
        b = x.double().view(x.shape[0], -1, block)
        top = b.abs().amax(-1, keepdim=True)
        if block == 32:
            unit = torch.where(top > 0, two_to(binade(top) - 2), 0.0)
        else:
            m = top.amax(1, keepdim=True)
            r = torch.where(m > 0, two_to(binade(m) - 12), 1.0)
            r = torch.where(m > 2688.0 * r, 2.0 * r, r)
            r = torch.where(m > 2688.0 * r, 2.0 * r, r)
            grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
            q = (top / (6.0 * r)).contiguous()
            hi = torch.searchsorted(grid, q).clamp(1, 126)
            below, above = q - grid[hi - 1], grid[hi] - q
            up = (above < below) | ((above == below) & (hi % 2 == 0))
            unit = torch.where(up, grid[hi], grid[hi - 1]) * r
        out = torch.empty_like(b)
        for i in range(0, b.shape[0], 1024):           # (in pieces, for the memory of the searches)
            part, u = b[i:i + 1024], unit[i:i + 1024]
            a = torch.where(u > 0, part.abs() / torch.where(u > 0, u, 1.0), 0.0)
            hi = torch.searchsorted(table, a.contiguous()).clamp(1, 7)
            below, above = a - table[hi - 1], table[hi] - a
            up = (above < below) | ((above == below) & (hi % 2 == 0))
            out[i:i + 1024] = torch.sign(part) * torch.where(up, table[hi], table[hi - 1]) * u
        return out.view(x.shape)

    if op == "roundtrip":
        return quantized(s["x"])
    c = s["w"]["codes"]
    both = torch.stack((c % 16, torch.div(c, 16, rounding_mode="floor")), -1).flatten(1).long()
    w = torch.where(both >= 8, -1.0, 1.0).double() * table[both % 8]
    w = (w.view(w.shape[0], -1, block) * (s["w"]["scale"].double() * s["w"]["row_scale"].double()[:, None])[..., None]).view(w.shape)
    if op == "dequant":
        return w
    return torch.einsum("mk,nk->mn", quantized(s["x"]) if op == "linear" else s["x"].double(), w)


def work(case):
    """Each operator's inputs read once and its outputs written once; products count two operations a weight and row."""
    op, M, K, N = case["op"], case["M"], case["K"], case["N"]
    f4 = 0.5 + (1 / 32 if case["block"] == 32 else 1 / 16)
    if op == "roundtrip":
        return {"bytes": M * K * (2 + f4 + f4 + 2), "flops": 6.0 * M * K}
    if op == "dequant":
        return {"bytes": M * K * (f4 + 2), "flops": 2.0 * M * K}
    if op == "gemv":
        return {"bytes": N * K * f4 + 2 * M * (K + N), "flops": 2.0 * M * K * N}
    return {"bytes": N * K * f4 + M * K * (2 + 2 * f4) + 2 * M * N, "flops": 2.0 * M * K * N}
