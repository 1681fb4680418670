"""Microscaled 4-bit floating point in 64 bits with numpy: the definition that the kernels are compared with.

Formats: "mx" (blocks of 32, scales 2^n; OCP Microscaling Formats 1.0) and "nv" (blocks of 16, e4m3 scales, a scale a row).
Values of codes, block scales and row scales are kept apart; `pack` and `unpack`, `tile` and `untile` go to the stored bytes.
"""
import numpy as np

BLOCK = {"mx": 32, "nv": 16}
E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
E4M3 = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def nearest(a, grid):
    """Index of the grid entry nearest to a >= 0: ties to the even one, beyond the last to the last."""
    mid = (grid[1:] + grid[:-1]) / 2
    lo, hi = np.searchsorted(mid, a, side="left"), np.searchsorted(mid, a, side="right")
    return np.where((lo != hi) & (lo % 2 == 1), hi, lo)


def mx_exponent(top):
    """of a block's scale, from its largest magnitude"""
    _, e = np.frexp(top)
    return np.where(top == 0, -127, np.maximum(e - 1 - 2, -127))


def nv_exponent(top):
    """of a row's scale"""
    m, e = np.frexp(top / 2688)
    return np.where(top == 0, 0, np.maximum(np.where(m == 0.5, e - 1, e), -126))


def nv_scale(top, row):
    """a block's scale, from its largest magnitude and the row's scale"""
    s = E4M3[nearest(top / 6 / row, E4M3)]
    return np.where(top == 0, 0.0, np.maximum(s, 2.0 ** -9))


def codes_of(x, div):
    """Values of the codes of x / div (zeros where div is zero)."""
    q = np.divide(x, div, out=np.zeros_like(x), where=div != 0)
    return np.copysign(E2M1[nearest(np.abs(q), E2M1)], x)


def quantize(x, fmt):
    """(values of the codes [M][K], block scales [M][K / block], row scales [M]) of rows x in fp64."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    b = x.reshape(M, -1, BLOCK[fmt])
    finite = np.isfinite(b).all(-1)
    if fmt == "nv":
        finite = np.repeat(finite.all(-1, keepdims=True), b.shape[1], 1)
    b = np.where(finite[..., None], b, 0.0)
    top = np.abs(b).max(-1)
    if fmt == "mx":
        row = np.ones(M)
        scale = np.where(finite, np.ldexp(1.0, mx_exponent(top)), np.nan)
    else:
        row = np.ldexp(1.0, nv_exponent(top.max(-1)))
        scale = nv_scale(top, row[:, None])
        row = np.where(finite[:, 0], row, np.nan)
    div = scale * (1.0 if fmt == "mx" else row[:, None])
    v = codes_of(b, np.where(finite, div, 1.0)[..., None])
    return v.reshape(M, K), scale, row


def expand(values, scale, row, fmt):
    M, K = values.shape
    return (values.reshape(M, -1, BLOCK[fmt]) * (scale * row[:, None])[..., None]).reshape(M, K)


def pack(values):
    c = nearest(np.abs(values), E2M1) | (np.signbit(values).astype(np.int64) << 3)
    return (c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)


def unpack(codes):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    return np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]


def _at(rows, nb):
    r, j = np.arange(rows)[:, None], np.arange(nb)[None, :]
    return (r // 128 * -(-nb // 4) + j // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + j % 4


def scale_bytes(scale, fmt):
    if fmt == "mx":
        return np.where(np.isnan(scale), 255, np.frexp(np.where(np.isnan(scale), 1.0, scale))[1] + 126).astype(np.uint8)
    return nearest(scale, E4M3).astype(np.uint8)


def tile(bytes_, fill=0):
    """Scale bytes [rows][blocks] into tiles of 128 x 4; `fill`: rows beyond the last (blocks beyond the last are zeros)."""
    rows, nb = bytes_.shape
    out = np.zeros(-(-rows // 128) * -(-nb // 4) * 512, np.uint8)
    if rows % 128:
        out[_at(-(-rows // 128) * 128, nb)[rows:]] = fill
    out[_at(rows, nb)] = bytes_
    return out


def untile(tiles, rows, nb):
    return tiles[_at(rows, nb)]


def scales_of(bytes_, fmt):
    return np.where(bytes_ == 255, np.nan, np.ldexp(1.0, bytes_.astype(np.int64) - 127)) if fmt == "mx" else E4M3[bytes_]
