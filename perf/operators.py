"""What is timed of the microscaled 4-bit floating point path: quantiser, expansion, product and prepared layer.

Three kinds of case.

``quantize``  rows to 4-bit codes with block scales and back to the values they stand for: activations of a step, or the
              rows of a weight matrix when a model is prepared and checked.
``product``   two quantised operands to a bf16 output: a linear whose weights and activations are in 4 bits already.
``linear``    the prepared layer as a serving engine calls it: bf16 activations are rotated by the Kronecker factors,
              quantised and multiplied with 4-bit weights in one call.

Two formats: ``mx`` has blocks of 32 values with a power-of-two scale (E8M0), ``nv`` blocks of 16 with an E4M3 scale and
one fp32 scale a row.  Codes are two e2m1 values a byte, the even one in the low half.  Scale bytes lie in tiles of 128
rows x 4 blocks, 512 bytes each: block j of row r at (r % 32) * 16 + (r / 32) * 4 + j, the tiles of 128 rows one after
the other along the row; rows are filled up to 128, blocks to 4 with zeros.

Activations are heavy-tailed with a few outlier channels (Student-t, nu = 3), weights Gaussian with row scales that
spread log-normally, Kronecker factors Haar-orthogonal.
"""
import math

import numpy as np
import torch

own = False                      # whether run() makes the framework's calls

DEV = "cuda"
BLOCK = {"mx": 32, "nv": 16}
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FORMATS = {"mx": 0, "nv": 1}

# (n1, n2) of the layers' input widths
FACTORS = [(32, 64), (64, 64), (64, 80), (64, 88), (64, 128), (86, 128), (108, 128), (112, 128), (160, 160)]
LARGEST = 2.0 * 4096 * 5120 * 25600


def listed():
    return [
        # one token's activations: latency
        {"name": "quantize_token", "kind": "quantize", "format": "mx", "dtype": "bf16", "M": 1, "K": 5120, "pad": 0},
        # a ragged chunk of a prompt in half precision, read out of a wider buffer
        {"name": "quantize_ragged", "kind": "quantize", "format": "mx", "dtype": "f16", "M": 333, "K": 11008, "pad": 24},
        # a long prompt
        {"name": "quantize_prompt", "kind": "quantize", "format": "nv", "dtype": "bf16", "M": 4096, "K": 5120, "pad": 0},
        # offline: the up projection's fp32 weights
        {"name": "quantize_weights", "kind": "quantize", "format": "nv", "dtype": "f32", "M": 25600, "K": 5120, "pad": 0},
        # one sequence being decoded
        {"name": "product_token", "kind": "product", "format": "mx", "M": 1, "K": 5120, "N": 5120},
        # a decode batch on the widest weights
        {"name": "product_batch", "kind": "product", "format": "nv", "M": 16, "K": 5120, "N": 25600},
        # a ragged chunk against an odd number of outputs
        {"name": "product_ragged", "kind": "product", "format": "mx", "M": 333, "K": 11008, "N": 4095},
        # a prompt through the down projection
        {"name": "product_down", "kind": "product", "format": "nv", "M": 1024, "K": 25600, "N": 5120},
        # a long prompt through the up projection
        {"name": "product_up", "kind": "product", "format": "mx", "M": 4096, "K": 5120, "N": 25600},
        # the layer: one token, a decode batch, a prompt
        {"name": "linear_token", "kind": "linear", "format": "mx", "n1": 64, "n2": 64, "M": 1, "N": 4096},
        {"name": "linear_batch", "kind": "linear", "format": "nv", "n1": 86, "n2": 128, "M": 50, "N": 4096},
        {"name": "linear_prompt", "kind": "linear", "format": "mx", "n1": 64, "n2": 80, "M": 2048, "N": 8192},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["quantize", "product", "product", "linear"])
    c = {"kind": kind, "format": rng.choice(["mx", "nv"])}
    if kind == "quantize":
        c["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        c["K"] = 32 * _log_int(rng, 2, 800)
        c["M"] = _log_int(rng, 1, min(32768, 25600 * 5120 // c["K"]))
        c["pad"] = rng.choice([0, 0, 8, 24])
        return c
    if kind == "product":
        c["K"] = 32 * _log_int(rng, 8, 800)
    else:
        c["n1"], c["n2"] = rng.choice(FACTORS)
    K = c["K"] if kind == "product" else c["n1"] * c["n2"]
    c["N"] = _log_int(rng, 64, 25600)
    c["M"] = _log_int(rng, 1, max(1, min(4096, int(LARGEST / 2 / K / c["N"]))))
    return c


# ---- the formats -------------------------------------------------------------------------------------------------
def _pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e2m1(a):
    """|values| rounded to 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to even codes)."""
    return torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2)).clamp(max=6)


def _quantize(x, fmt):
    """(values of the codes [M][K], block scales [M][K / block], row scales [M]), in 64 bits: which of two codes a value
    gets is decided at a border."""
    M, K = x.shape
    b = x.double().reshape(M, K // BLOCK[fmt], BLOCK[fmt])
    amax = b.abs().amax(-1)
    if fmt == "mx":
        e = torch.frexp(amax).exponent - 3
        scale = _pow2(torch.where(amax == 0, torch.full_like(e, -127), e.clamp(min=-127)))
        row = torch.ones(M, dtype=torch.float64, device=x.device)
    else:
        m, e = torch.frexp(amax.amax(-1) / 2688)
        row = _pow2(torch.where(m == 0.5, e - 1, e).clamp(min=-126))
        row = torch.where(m == 0, torch.ones_like(row), row)
        t = amax / 6 / row[:, None]
        q = _pow2((torch.frexp(t).exponent - 1).clamp(min=-6) - 3)
        scale = (torch.round(t / q) * q).clamp(min=2.0 ** -9, max=448)
        scale = torch.where(amax == 0, torch.zeros_like(scale), scale)
    div = scale * row[:, None]
    v = b / torch.where(div == 0, torch.ones_like(div), div)[..., None]
    return (torch.copysign(_e2m1(v.abs()), v)).reshape(M, K), scale, row


def _expand(values, scale, row, fmt):
    M, K = values.shape
    return (values.reshape(M, -1, BLOCK[fmt]) * (scale * row[:, None])[..., None]).reshape(M, K)


def _pack(values):
    """Values of codes to bytes, two a byte."""
    a = values.abs()
    c = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    c = c | (torch.signbit(values).to(torch.uint8) << 3)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).contiguous()


def _unpack(codes):
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32, device=codes.device)
    c = torch.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    return table[c.int()]


def _tile(scale, fmt):
    """Block scales [M][nb] to bytes in tiles of 128 x 4."""
    if fmt == "mx":
        byte = (torch.frexp(scale).exponent + 126).to(torch.uint8)
    else:
        byte = scale.float().to(torch.float8_e4m3fn).view(torch.uint8)
    M, nb = byte.shape
    full = torch.zeros(-(-M // 128) * 128, -(-nb // 4) * 4, dtype=torch.uint8, device=byte.device)
    full[:M, :nb] = byte
    return full.reshape(-1, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1).contiguous()


def _untile(tiles, M, nb, fmt):
    cols = -(-nb // 4)
    byte = tiles.reshape(-1, cols, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, cols * 4)[:M, :nb]
    if fmt == "mx":
        return _pow2(byte.int() - 127).float()
    return byte.contiguous().view(torch.float8_e4m3fn).float()


# ---- inputs ------------------------------------------------------------------------------------------------------
def _haar(n, rng):
    q, r = np.linalg.qr(rng.standard_normal((n, n)))
    return torch.from_numpy(np.ascontiguousarray(q * np.sign(np.diag(r))[None, :], dtype=np.float32)).to(DEV)


def _activations(M, K, g):
    z = torch.randn(M, K, device=DEV, generator=g)
    chi = sum(torch.randn(M, K, device=DEV, generator=g).square_() for _ in range(3))
    z *= torch.rsqrt(chi / 3)
    z[:, torch.randint(0, K, (8,), device=DEV, generator=g)] *= 50
    return z


def _weights(N, K, g):
    w = torch.randn(N, K, device=DEV, generator=g)
    return w * torch.exp(0.3 * torch.randn(N, 1, device=DEV, generator=g) - 4)


def _operand(x, fmt):
    """Codes, tiled scales and row scales of the rows of x, some rows at a time."""
    codes, scales, rows = [], [], []
    for p in x.split(4096):
        v, s, r = _quantize(p, fmt)
        codes.append(_pack(v))
        scales.append(s)
        rows.append(r.float())
    return torch.cat(codes), _tile(torch.cat(scales), fmt), torch.cat(rows) if fmt == "nv" else None


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 13)
    fmt, M = case["format"], case["M"]
    if case["kind"] == "quantize":
        K, dtype = case["K"], DTYPES[case["dtype"]]
        x = torch.zeros(M, K + case["pad"], dtype=dtype, device=DEV)
        x[:, :K] = (_weights(M, K, g) if case["dtype"] == "f32" else _activations(M, K, g)).to(dtype)
        return {"kind": "quantize", "format": fmt, "x": x[:, :K]}
    N = case["N"]
    if case["kind"] == "product":
        K = case["K"]
        s = {"kind": "product", "format": fmt, "a": _operand(_activations(M, K, g), fmt), "w": _operand(_weights(N, K, g), fmt)}
        if own:                  # scratch that a program allocates once
            from paper_2605_00422_b200 import bwla
            s["workspace"] = bwla.new_fp4_workspace(M, K, N, DEV)
        return s
    n1, n2 = case["n1"], case["n2"]
    K = n1 * n2
    rng = np.random.default_rng([422, int(seed), n1, n2])
    s = {"kind": "linear", "format": fmt, "P1": _haar(n1, rng), "P2": _haar(n2, rng), "x": _activations(M, K, g).bfloat16(),
         "w": _operand(_weights(N, K, g), fmt)}
    if own:                      # the handle that a program keeps for a layer, and its scratch
        from paper_2605_00422_b200 import bwla
        s["layer"] = bwla.bwla_fp4_layer_create(s["P1"], s["P2"], FORMATS[fmt], *s["w"])
        s["workspace"] = bwla.new_fp4_layer_workspace(s["layer"], M, DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------
def _rotate(x, P1, P2):
    M, n1, n2 = x.shape[0], P1.shape[0], P2.shape[0]
    return (P1.double().t() @ x.double().reshape(M, n1, n2) @ P2.double()).reshape(M, n1 * n2)


def _values(codes, tiles, rows, fmt):
    M, K = codes.shape[0], 2 * codes.shape[1]
    v = _unpack(codes).reshape(M, -1, BLOCK[fmt]) * _untile(tiles, M, K // BLOCK[fmt], fmt)[..., None]
    v = v.reshape(M, K)
    return v if rows is None else v * rows[:, None]


def run(state):
    fmt = state["format"]
    if own:
        from paper_2605_00422_b200 import bwla
        if state["kind"] == "quantize":
            codes, scales, rows = bwla.bwla_fp4_quantize_rows(state["x"], FORMATS[fmt])
            return bwla.bwla_fp4_expand_rows(codes, scales, rows, FORMATS[fmt])
        if state["kind"] == "product":
            return bwla.bwla_fp4_gemm_codes(*state["a"], *state["w"], FORMATS[fmt], workspace=state["workspace"])
        return bwla.bwla_fp4_layer_linear(state["layer"], state["x"], workspace=state["workspace"])
    if state["kind"] == "quantize":
        return _expand(*_quantize(state["x"], fmt), fmt).bfloat16()
    if state["kind"] == "product":
        return (_values(*state["a"], fmt) @ _values(*state["w"], fmt).t()).bfloat16()
    a = _expand(*_quantize(_rotate(state["x"], state["P1"], state["P2"]), fmt), fmt).float()
    return (a @ _values(*state["w"], fmt).t()).bfloat16()


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def _operand_bytes(rows, K, fmt):
    return rows * K // 2 + rows * K // BLOCK[fmt] + (4 * rows if fmt == "nv" else 0)


def work(case):
    fmt, M = case["format"], case["M"]
    if case["kind"] == "quantize":
        K = case["K"]
        # the rows, their codes and scales, and the values
        return {"bytes": M * K * DTYPES[case["dtype"]].itemsize + _operand_bytes(M, K, fmt) + 2 * M * K, "flops": 4 * M * K}
    N = case["N"]
    if case["kind"] == "product":
        K = case["K"]
        return {"bytes": _operand_bytes(M, K, fmt) + _operand_bytes(N, K, fmt) + 2 * M * N, "flops": 2 * M * N * K}
    n1, n2 = case["n1"], case["n2"]
    K = n1 * n2
    return {"bytes": 2 * M * K + 4 * (n1 * n1 + n2 * n2) + _operand_bytes(N, K, fmt) + 2 * M * N,
            "flops": 2 * M * N * K + 2 * M * K * (n1 + n2)}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------
def _nearest(a, grid):
    """a >= 0 to the nearest entry of the sorted grid, ties to the even entry, beyond the last one to the last."""
    mid = (grid[1:] + grid[:-1]) / 2
    i = torch.searchsorted(mid, a.contiguous())
    tie = (i < len(mid)) & (mid[i.clamp(max=len(mid) - 1)] == a)
    return grid[torch.where(tie & (i % 2 == 1), i + 1, i)]


def _two(e):
    return ((e.to(torch.int64) + 1023) * 2 ** 52).view(torch.float64)        # (a power function may be off by a bit, and move ties)


def _grid(exponent_bits, mantissa_bits, bias, count):
    v = []
    for c in range(count):
        e, m = c >> mantissa_bits, c & ((1 << mantissa_bits) - 1)
        v.append(m / (1 << mantissa_bits) * 2.0 ** (1 - bias) if e == 0 else (1 + m / (1 << mantissa_bits)) * 2.0 ** (e - bias))
    return torch.tensor(v, dtype=torch.float64, device=DEV)


def _exact_rows(x, fmt):
    """The values that the rows' codes stand for."""
    M, K = x.shape
    x = x.double()
    out = torch.empty(M, K, dtype=torch.float64, device=DEV)
    four, eight = _grid(2, 1, 1, 8), _grid(4, 3, 7, 127)
    size = BLOCK[fmt]
    for lo in range(0, M, 2048):
        b = x[lo:lo + 2048].reshape(-1, K // size, size)
        top = b.abs().max(-1, keepdim=True).values
        if fmt == "mx":
            step = _two(((top.view(torch.int64) >> 52) - 1025).clamp(min=-127))
        else:
            row = top.max(1, keepdim=True).values
            E = torch.ceil(torch.log2(row / 2688))
            E = torch.where(row > 2688 * _two(E), E + 1, E)
            E = torch.where(row <= 2688 * _two(E - 1), E - 1, E).clamp(min=-126)
            E = torch.where(row == 0, torch.zeros_like(E), E)
            step = _nearest(top / 6 / _two(E), eight)
            step = torch.where((top > 0) & (step == 0), torch.full_like(step, 2.0 ** -9), step) * _two(E)
        q = _nearest(torch.where(step > 0, b.abs() / step, torch.zeros_like(b)), four)
        out[lo:lo + 2048] = (torch.sign(b) * q * step).reshape(-1, K)
    return out


def _exact_operand(codes, tiles, rows, fmt):
    M, K = codes.shape[0], 2 * codes.shape[1]
    k = torch.arange(K, device=DEV)
    nib = (codes[:, k // 2].int() >> (4 * (k % 2)).int()) & 15
    q = _grid(2, 1, 1, 8)[(nib & 7).long()] * (1 - 2 * (nib >> 3).double())
    r, j = torch.arange(M, device=DEV)[:, None], (k // BLOCK[fmt])[None, :]
    col_tiles = -(-(K // BLOCK[fmt]) // 4)
    byte = tiles[((r // 128) * col_tiles + j // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + j % 4].long()
    q *= _two(byte - 127) if fmt == "mx" else _grid(4, 3, 7, 127)[byte]
    return q if rows is None else q * rows.double()[:, None]


def exact(case, seed):
    if case["kind"] != "quantize" and work(case)["flops"] > 3e14:      # (a product in 64 bits of that size takes too long)
        return None
    s, fmt = prepare(case, seed), case["format"]
    if case["kind"] == "quantize":
        return _exact_rows(s["x"], fmt)
    if case["kind"] == "product":
        a = _exact_operand(*s["a"], fmt)
    else:
        M, n1, n2 = case["M"], case["n1"], case["n2"]
        y = torch.einsum("ac,mab,bd->mcd", s["P1"].double(), s["x"].double().reshape(M, n1, n2), s["P2"].double())
        a = _exact_rows(y.reshape(M, n1 * n2), fmt)
    return a @ _exact_operand(*s["w"], fmt).t()
