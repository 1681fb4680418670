"""Microscaled 4-bit floating point on the GPU against oracle/fp4.py (64 bits).

Tolerances:
  * quantiser and expansion: bit-exact, whatever the type and layout of the rows.
  * product: within half a bf16 step of the exact sum (2^-8 relative: `torch.finfo(bf16).eps / 2`, counted once) plus what fp32
    sums can be off: products of two codes and their scales are exact, the tensor core adds 64 of them at a time to its
    accumulator and truncates (below 2^-22 of the largest partial sum, which is at most S = sum |a||w|), so (K/64 + 4) 2^-22 S,
    the 4 for the row scales' multiplications and sums of split K (at most 8 parts, each rounded to 2^-24).
    Where all partial sums are integers below 2^24 nothing is lost: outputs are the rounded exact ones.
  * rotation: Y is within E = 1e-6 of a token's largest magnitude (the bound that the rotation's own tests hold); rounding is
    monotone, so a scale must lie between those of (top - E) and (top + E), and a code between those of y - E and y + E.
"""
import numpy as np
import pytest
import torch

from oracle import fp4

pytestmark = pytest.mark.gpu

FORMATS = {"mx": 0, "nv": 1}


@pytest.fixture(scope="module")
def bwla():
    from paper_2605_00422_b200 import bwla
    return bwla


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def rows_like(rng, M, K):
    """Rows of many magnitudes with what rounding can go wrong at: ties, zeros of both signs, equal blocks, a lone large value."""
    x = rng.standard_t(3, (M, K)) * np.exp2(rng.integers(-12, 12, (M, 1)))
    flat = x.reshape(-1)
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0])
    at = rng.integers(0, flat.size, flat.size // 4)
    flat[at] = rng.choice(grid, at.size) * np.exp2(rng.integers(-3, 3, at.size)) * rng.choice([-1, 1], at.size)
    if M > 2:
        x[1] = 0.0
        x[2, ::2] = -0.0
    if M > 3:
        x[3, : min(K, 64)] = 0.0
    return x


def quantised(bwla, x, fmt):
    codes, scales, rows = bwla.bwla_fp4_quantize_rows(x, FORMATS[fmt])
    M, nb = x.shape[0], x.shape[1] // fp4.BLOCK[fmt]
    s = scales.cpu().numpy()
    got = fp4.untile(s, M, nb)
    pad = fp4.untile(s, M, -(-nb // 4) * 4)[:, nb:]
    assert not pad.any(), "blocks that fill the last tile must be zero"
    return codes.cpu().numpy(), got, None if rows is None else rows.cpu().numpy()


def check_quantiser(bwla, x, fmt):
    codes, s, rows = quantised(bwla, x, fmt)
    v, scale, row = fp4.quantize(x.double().cpu().numpy(), fmt)
    if fmt == "nv":
        assert np.array_equal(rows, row.astype(np.float32), equal_nan=True)
    bad = np.isnan(row)
    want = fp4.scale_bytes(np.where(bad[:, None], 0.0, scale), fmt)
    assert np.array_equal(s, want)
    assert np.array_equal(codes, fp4.pack(v))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K", [(1, 32), (5, 96), (129, 2048), (3, 2080), (33, 5120), (2, 8192), (7, 8224), (2, 25600), (2, 32768), (1, 32800), (300, 160)])
def test_quantiser_is_exact(bwla, fmt, dtype, M, K):
    x = dev(rows_like(np.random.default_rng([M, K]), M, K)).to(dtype)
    check_quantiser(bwla, x, fmt)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (3, 1), (24, 5)])
def test_strided_and_unaligned_rows(bwla, fmt, dtype, pad, shift):
    big = dev(rows_like(np.random.default_rng(7), 17, 352 + pad)).to(dtype)
    flat = torch.zeros(big.numel() + shift, dtype=dtype, device="cuda")
    flat[shift:] = big.reshape(-1)
    x = flat[shift:].view(17, 352 + pad)[:, :352]
    assert x.stride(0) == 352 + pad
    check_quantiser(bwla, x, fmt)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_values_next_to_borders(bwla, fmt):
    """fp32 values one step beside a border between two codes or two scales, and on it."""
    rng = np.random.default_rng(3)
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    blocks = []
    for _ in range(4096):
        # the block's scale from its largest value, then borders of that scale
        top = np.float32(rng.uniform(0.01, 2688))
        s = fp4.nv_scale(np.float64(top), 1.0) if fmt == "nv" else 2.0 ** float(fp4.mx_exponent(np.float64(top)))
        b = np.float32(s) * rng.choice(mid, fp4.BLOCK[fmt]).astype(np.float32)
        b = np.where(rng.random(b.size) < 0.3, np.nextafter(b, np.float32(np.inf)), np.where(rng.random(b.size) < 0.4, np.nextafter(b, np.float32(0)), b))
        b[0] = top
        blocks.append(np.minimum(b, top))
    if fmt == "nv":        # largest values beside 6 times a border of e4m3
        for i in range(0, 2048):
            m = np.float32(6 * (fp4.E4M3[i % 126] + fp4.E4M3[i % 126 + 1]) / 2)
            blocks[i] = np.minimum(blocks[i], m)
            blocks[i][0] = (m, np.nextafter(m, np.float32(np.inf)), np.nextafter(m, np.float32(0)))[i % 3]
    x = np.stack(blocks).reshape(-1, 32 * fp4.BLOCK[fmt])
    if fmt == "nv":
        x[:, 5] = 2688.0    # the row's scale is 1
    check_quantiser(bwla, dev(x), fmt)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_ends_of_the_range(bwla, fmt):
    f = np.finfo(np.float32)
    x = np.zeros((14, 64), np.float32)
    x[0] = f.max
    x[1, 3] = f.tiny
    x[2, 5] = f.smallest_subnormal
    x[3, ::3] = -f.max
    x[4, :32] = np.linspace(-f.max, f.max, 32, dtype=np.float32)
    x[5, 40] = np.inf
    x[6, 40] = -np.inf
    x[7, 2] = np.nan
    x[8] = np.float32(2.0 ** -126) * np.linspace(0, 5, 64, dtype=np.float32)
    x[9] = np.float32(2.0 ** -140) * np.arange(64, dtype=np.float32)
    x[10, 0], x[10, 20] = f.max, f.smallest_subnormal
    x[11, 0], x[11, 50] = 1.0, 2.0 ** -14
    x[12, 0], x[12, 50] = 2688.0, 0.004
    check_quantiser(bwla, dev(x), fmt)
    y = bwla.bwla_fp4_expand_rows(*bwla.bwla_fp4_quantize_rows(dev(x), FORMATS[fmt]), FORMATS[fmt], dtype=torch.float32).cpu().numpy()
    want = fp4.expand(*fp4.quantize(x.astype(np.float64), fmt), fmt)
    assert np.array_equal(y, want.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,K,pad", [(1, 32, 0), (130, 96, 0), (3, 2080, 5), (257, 5120, 8), (2, 25600, 1)])
def test_expansion_is_exact(bwla, fmt, M, K, pad):
    x = dev(rows_like(np.random.default_rng([M, K, 2]), M, K)).bfloat16()
    q = bwla.bwla_fp4_quantize_rows(x, FORMATS[fmt])
    want = fp4.expand(*fp4.quantize(x.double().cpu().numpy(), fmt), fmt)
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.full((M, K + pad), 7.0, dtype=dtype, device="cuda")
        got = bwla.bwla_fp4_expand_rows(*q, FORMATS[fmt], out=out[:, :K])
        assert np.array_equal(got.double().cpu().numpy(), want)
        assert (out[:, K:] == 7).all()
    # row scales of any value: two roundings
    r = torch.rand(M, device="cuda") + 0.5
    got = bwla.bwla_fp4_expand_rows(q[0], q[1], r, FORMATS[fmt], dtype=torch.float32).double().cpu().numpy()
    v, s, _ = fp4.quantize(x.double().cpu().numpy(), fmt)
    want = fp4.expand(v, s, r.double().cpu().numpy(), fmt)
    assert (np.abs(got - want) <= 2.0 ** -24 * np.abs(want)).all()


def operand(rng, rows, K, fmt, integers=False, fill=0):
    """Codes, scale tiles, row scales on the device and the values (fp64) without row scales."""
    codes = rng.integers(0, 256, (rows, K // 2), dtype=np.uint8)
    nb = K // fp4.BLOCK[fmt]
    if fmt == "mx":
        s = (127 + rng.integers(0, 2, (rows, nb))) if integers else rng.integers(118, 130, (rows, nb))
    else:
        s = rng.choice([56, 64] if integers else np.arange(40, 80), (rows, nb))       # 56: 1, 64: 2
    s = s.astype(np.uint8)
    values = fp4.unpack(codes).reshape(rows, nb, -1) * fp4.scales_of(s, fmt)[..., None]
    return dev(codes), dev(fp4.tile(s, fill)), dev(values.reshape(rows, K))


def check_product(out, a, w, ra=None, rw=None, exact=False):
    """a, w: values fp64 on the device."""
    y = a @ w.t()
    S = a.abs() @ w.abs().t()
    f = torch.ones_like(y)
    if ra is not None:
        f = f * ra.double()[:, None]
    if rw is not None:
        f = f * rw.double()[None, :]
    y, S = y * f, S * f.abs()
    if exact:
        assert torch.equal(out, y.bfloat16()), f"{int((out != y.bfloat16()).sum())} of {out.numel()} differ"
        return
    K = a.shape[1]
    tol = 2.0 ** -8 * y.abs() + (K / 64 + 4) * 2.0 ** -22 * S
    off = (out.double() - y).abs()
    assert (off <= tol).all(), f"{int((off > tol).sum())} of {out.numel()} off, worst {float((off / tol).max()):.3g} of the tolerance"


SIZES = [(1, 1, 32), (1, 77, 64), (1, 128, 256), (3, 300, 160), (8, 129, 2080), (9, 257, 512), (16, 5120, 5120), (17, 100, 4096), (31, 4095, 96), (32, 640, 11008),
         (33, 256, 8192), (64, 1000, 5120), (65, 512, 288), (100, 130, 25600), (128, 2048, 4096), (129, 129, 1056), (200, 777, 5120), (257, 256, 512), (333, 4095, 2048),
         (512, 512, 4096), (1000, 1030, 544), (1024, 5120, 5120), (2048, 256, 25600), (2500, 3000, 1024)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product_of_integers_is_exact(bwla, fmt, M, N, K):
    """Codes times 2 scaled by 1 or 2: sums of quarters below 2^24, so every order of adding gives the exact sum."""
    rng = np.random.default_rng([M, N, K])
    a, sa, va = operand(rng, M, K, fmt, integers=True)
    w, sw, vw = operand(rng, N, K, fmt, integers=True)
    ws = bwla.new_fp4_workspace(M, K, N)
    out = bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, FORMATS[fmt], workspace=ws)
    assert bwla.bwla_check_status(ws) == 0
    check_product(out, va, vw, exact=True)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(bwla, fmt, M, N, K):
    """Row scales, an output inside a wider buffer, rows beyond the last with NaN scale bytes."""
    rng = np.random.default_rng([M, N, K, 1])
    a, sa, va = operand(rng, M, K, fmt, fill=255 if fmt == "mx" else 127)
    w, sw, vw = operand(rng, N, K, fmt, fill=255 if fmt == "mx" else 127)
    ra = torch.rand(M, device="cuda") + 0.5 if (M + N) % 3 else None
    rw = torch.rand(N, device="cuda") - 0.5 if (M + N) % 2 else None
    pad = (M + K // 32) % 4 * 4 + N % 2
    wide = torch.full((M + 1, N + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = bwla.new_fp4_workspace(M, K, N)
    out = bwla.bwla_fp4_gemm_codes(a, sa, ra, w, sw, rw, FORMATS[fmt], out=wide[:M, :N], workspace=ws)
    assert bwla.bwla_check_status(ws) == 0
    check_product(out, va, vw, ra, rw)
    assert (wide[:, N:] == 7).all() and (wide[M] == 7).all()
    again = bwla.bwla_fp4_gemm_codes(a, sa, ra, w, sw, rw, FORMATS[fmt], workspace=ws)
    assert torch.equal(again, out), "a call must repeat itself bit for bit"


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M", [1, 40, 300, 600])
def test_a_nan_block_stays_in_its_row(bwla, fmt, M):
    rng = np.random.default_rng(M)
    K, N = 512, 200
    x = dev(rng.standard_normal((M, K))).bfloat16()
    x[M // 2, 100] = float("nan")
    w = dev(rng.standard_normal((N, K))).bfloat16()
    w[7, 3] = float("inf")
    out = bwla.bwla_fp4_gemm_codes(*bwla.bwla_fp4_quantize_rows(x, FORMATS[fmt]), *bwla.bwla_fp4_quantize_rows(w, FORMATS[fmt]), FORMATS[fmt])
    nan = torch.isnan(out)
    assert nan[M // 2].all() and nan[:, 7].all()
    nan[M // 2] = False
    nan[:, 7] = False
    assert not nan.any()


def haar(rng, n):
    q, r = np.linalg.qr(rng.standard_normal((n, n)))
    return (q * np.sign(np.diag(r))).astype(np.float32)


def check_rotated(bwla, x, P1, P2, fmt, q):
    codes, scales, rows = q
    M, K = x.shape
    n1, n2 = P1.shape[0], P2.shape[0]
    Y = np.einsum("ac,mab,bd->mcd", P1.astype(np.float64), x.double().cpu().numpy().reshape(M, n1, n2), P2.astype(np.float64), optimize=True).reshape(M, K)
    err = 1e-6 * np.abs(Y).max(1, keepdims=True)
    nb = K // fp4.BLOCK[fmt]
    byte = fp4.untile(scales.cpu().numpy(), M, nb)
    assert not fp4.untile(scales.cpu().numpy(), M, -(-nb // 4) * 4)[:, nb:].any()
    s = fp4.scales_of(byte, fmt)
    top = np.abs(Y).reshape(M, nb, -1).max(-1)
    if fmt == "mx":
        lo, hi = np.ldexp(1.0, fp4.mx_exponent(np.maximum(top - err, 0))), np.ldexp(1.0, fp4.mx_exponent(top + err))
        div = s
    else:
        r = rows.double().cpu().numpy()[:, None]
        big = np.abs(Y).max(1, keepdims=True)
        assert (r >= np.ldexp(1.0, fp4.nv_exponent(big - err))).all() and (r <= np.ldexp(1.0, fp4.nv_exponent(big + err))).all()
        lo, hi = fp4.nv_scale(np.maximum(top - err, 0), r), fp4.nv_scale(top + err, r)
        div = s * r
    assert (s >= lo).all() and (s <= hi).all()
    v = fp4.unpack(codes.cpu().numpy())
    d = np.repeat(div, fp4.BLOCK[fmt], 1)
    assert (v >= fp4.codes_of(Y - err, d)).all() and (v <= fp4.codes_of(Y + err, d)).all()


FACTORS = [(4, 8), (3, 32), (32, 64), (64, 64), (64, 80), (40, 88), (86, 128), (108, 128), (112, 128), (160, 160), (128, 64), (16, 136)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2", FACTORS)
@pytest.mark.parametrize("M", [1, 5, 50, 300, 700])
def test_rotation(bwla, fmt, n1, n2, M):
    if n1 * n2 > 20000 and M > 300:
        M = 301
    rng = np.random.default_rng([n1, n2, M])
    K = n1 * n2
    x = dev(rng.standard_t(3, (M, K)) * np.where(rng.random(K) < 0.01, 50, 1)).bfloat16()
    if M > 3:
        x[2] = 0
    P1, P2 = haar(rng, n1), haar(rng, n2)
    check_rotated(bwla, x, P1, P2, fmt, bwla.bwla_rotate_quant_fp4(x, dev(P1), dev(P2), FORMATS[fmt]))
    w = bwla.bwla_fp4_quantize_rows(torch.randn(72, K, device="cuda"), FORMATS[fmt])
    layer = bwla.bwla_fp4_layer_create(dev(P1), dev(P2), FORMATS[fmt], *w)
    ws = bwla.new_fp4_layer_workspace(layer, M)
    q = bwla.bwla_fp4_layer_rotate_quant(layer, x, workspace=ws)
    assert bwla.bwla_check_status(ws) == 0
    check_rotated(bwla, x, P1, P2, fmt, q)
    # the layer in one call is the two steps
    out = bwla.bwla_fp4_layer_linear(layer, x, workspace=ws)
    assert bwla.bwla_check_status(ws) == 0
    assert torch.equal(out, bwla.bwla_fp4_gemm_codes(*q, *w, FORMATS[fmt]))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2", [(64, 64), (86, 128), (64, 88), (160, 160)])
@pytest.mark.parametrize("M", [4, 400])
def test_rotation_of_tokens_with_infinities(bwla, fmt, n1, n2, M):
    rng = np.random.default_rng([n1, M])
    K = n1 * n2
    x = dev(rng.standard_normal((M, K))).bfloat16()
    x[1, 5] = float("inf")
    x[3, K - 1] = float("nan")
    P1, P2 = haar(rng, n1), haar(rng, n2)
    w = bwla.bwla_fp4_quantize_rows(torch.randn(40, K, device="cuda"), FORMATS[fmt])
    layer = bwla.bwla_fp4_layer_create(dev(P1), dev(P2), FORMATS[fmt], *w)
    out = torch.isnan(bwla.bwla_fp4_layer_linear(layer, x))
    assert out[[1, 3]].all()
    out[[1, 3]] = False
    assert not out.any()


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_rotated_weights_meet_rotated_activations(bwla, fmt):
    """The whole path as a user goes it: weights through the rotation and the quantiser, a layer, tokens; against the dense product.
    Orthogonal factors leave x . w as it is, and 4-bit codes of both sides are off by about 0.1 of it."""
    rng = np.random.default_rng(5)
    n1, n2, N, M = 64, 64, 384, 70
    K = n1 * n2
    P1, P2 = haar(rng, n1), haar(rng, n2)
    W = dev(rng.standard_normal((N, K))).bfloat16()
    x = dev(rng.standard_t(3, (M, K))).bfloat16()
    w = bwla.bwla_rotate_quant_fp4(W, dev(P1), dev(P2), FORMATS[fmt])
    layer = bwla.bwla_fp4_layer_create(dev(P1), dev(P2), FORMATS[fmt], *w)
    out = bwla.bwla_fp4_layer_linear(layer, x).double()
    dense = x.double() @ W.double().t()
    rel = float((out - dense).norm() / dense.norm())
    # a code is off by at most a sixth of the value or a quarter of the scale (which is at most half of top / 2): each side below
    # 1/4 of its rms in the 2-norm, and the two are independent
    assert rel < (2 * 0.25 ** 2) ** 0.5


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M", [1, 16, 200, 700])
def test_captured_and_replayed(bwla, fmt, M):
    rng = np.random.default_rng([M, 9])
    n1, n2, N = 64, 64, 640
    K = n1 * n2
    P1, P2 = dev(haar(rng, n1)), dev(haar(rng, n2))
    w = bwla.bwla_fp4_quantize_rows(torch.randn(N, K, device="cuda"), FORMATS[fmt])
    layer = bwla.bwla_fp4_layer_create(P1, P2, FORMATS[fmt], *w)
    ws = bwla.new_fp4_layer_workspace(layer, M)
    x = torch.randn(M, K, device="cuda").bfloat16()
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bwla.bwla_fp4_layer_linear(layer, x, out=out, workspace=ws)
        side.synchronize()
        graphs = []
        for _ in range(2):                        # two graphs on one workspace, replayed in turn
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                bwla.bwla_fp4_layer_linear(layer, x, out=out, workspace=ws)
            graphs.append(g)
        for i in range(4):
            x.copy_(torch.randn(M, K, device="cuda").bfloat16())
            graphs[i % 2].replay()
            side.synchronize()
            got = out.clone()
            want = bwla.bwla_fp4_layer_linear(layer, x)
            side.synchronize()
            assert torch.equal(got, want)
    assert bwla.bwla_check_status(ws) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [(1, 5120, 5120), (600, 1024, 2048)])
def test_weights_and_tokens_made_by_the_kernel_before(bwla, fmt, M, N, K):
    """No synchronisation between the quantiser and the product that reads what it made, on either side, again and again."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = [torch.randn(M, K, device="cuda", generator=g).bfloat16() for _ in range(4)]
    w = [torch.randn(N, K, device="cuda", generator=g).bfloat16() for _ in range(4)]
    want = []
    for a, b in zip(x, w):
        qa, qb = bwla.bwla_fp4_quantize_rows(a, FORMATS[fmt]), bwla.bwla_fp4_quantize_rows(b, FORMATS[fmt])
        torch.cuda.synchronize()
        want.append(bwla.bwla_fp4_gemm_codes(*qa, *qb, FORMATS[fmt]))
        torch.cuda.synchronize()
    qa, qb = bwla.bwla_fp4_quantize_rows(x[0], FORMATS[fmt]), bwla.bwla_fp4_quantize_rows(w[0], FORMATS[fmt])
    ws = bwla.new_fp4_workspace(M, K, N)
    outs = [torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, b, out in zip(x, w, outs):
            bwla.bwla_fp4_quantize_rows(b, FORMATS[fmt], *qb)
            bwla.bwla_fp4_gemm_codes(*qa, *qb, FORMATS[fmt], out=out, workspace=ws)       # (tokens of the round before: overwritten next)
            bwla.bwla_fp4_quantize_rows(a, FORMATS[fmt], *qa)
            bwla.bwla_fp4_gemm_codes(*qa, *qb, FORMATS[fmt], out=out, workspace=ws)
        torch.cuda.synchronize()
        for out, y in zip(outs, want):
            assert torch.equal(out, y)


def test_empty_calls_and_destroyed_layers(bwla):
    K, N = 64, 40
    w = bwla.bwla_fp4_quantize_rows(torch.randn(N, K, device="cuda"), 0)
    x0 = torch.empty(0, K, dtype=torch.bfloat16, device="cuda")
    q0 = bwla.bwla_fp4_quantize_rows(x0, 0)
    assert q0[0].shape == (0, 32) and q0[1].numel() == 0
    assert bwla.bwla_fp4_expand_rows(*q0, 0).shape == (0, K)
    assert bwla.bwla_fp4_gemm_codes(*q0, *w, 0).shape == (0, N)
    eye = torch.eye(8, device="cuda")
    layer = bwla.bwla_fp4_layer_create(eye, eye.clone(), 0, *w)
    assert bwla.bwla_fp4_layer_linear(layer, x0).shape == (0, N)
    x, out = torch.zeros(2, K, dtype=torch.bfloat16, device="cuda"), torch.empty(2, N, dtype=torch.bfloat16, device="cuda")
    ws = bwla.new_fp4_layer_workspace(layer, 2)
    with pytest.raises(bwla.BwlaError) as e:
        bwla.bwla_fp4_layer_linear(layer, x, out, ws[:256])
    assert e.value.status == bwla.BWLA_ERR_WORKSPACE
    for bad in (dict(x=x[:, :32]), dict(out=out[:, :8]), dict(out=out[:1]), dict(x=x.float()), dict(workspace=ws.cpu())):
        with pytest.raises(TypeError):
            bwla.bwla_fp4_layer_linear(layer, **{**dict(x=x, out=out, workspace=ws), **bad})
    for bad in ((w[0][:, ::2], w[1], None), (w[0], w[1][:100], None), (w[0], w[1], torch.ones(3, device="cuda")), (w[0].cpu(), w[1], None)):
        with pytest.raises(TypeError):
            bwla.bwla_fp4_gemm_codes(*bad, *w, 0, out=torch.empty(N, N, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises((AttributeError, TypeError)):        # (a layer of the other kind)
        bwla.bwla_w1ax_linear_group([layer], x, [out], ws)
    bwla.bwla_fp4_layer_destroy(layer)
    with pytest.raises(bwla.BwlaError) as e:
        bwla.bwla_fp4_layer_linear(layer, x, out, ws)
    assert e.value.status == bwla.BWLA_ERR_INVALID_ARG
    with pytest.raises(bwla.BwlaError) as e:                # factor sizes that the rotation does not take
        bwla.bwla_rotate_quant_fp4(x, torch.eye(16, device="cuda"), torch.eye(4, device="cuda"), 0)
    assert e.value.status == bwla.BWLA_ERR_UNSUPPORTED


def test_a_failed_workspace_keeps_its_word(bwla):
    """The status word set by an earlier call: later calls skip their work until it has been read."""
    M, N, K = 64, 256, 512
    rng = np.random.default_rng(0)
    a, sa, va = operand(rng, M, K, "mx", integers=True)
    w, sw, vw = operand(rng, N, K, "mx", integers=True)
    ws = bwla.new_fp4_workspace(M, K, N)
    ws[:4].view(torch.int32)[0] = 1
    bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, 0, workspace=ws)
    assert bwla.bwla_check_status(ws) == bwla.BWLA_ERR_DEVICE_TIMEOUT
    check_product(bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, 0, workspace=ws), va, vw, exact=True)
    assert bwla.bwla_check_status(ws) == 0


@pytest.mark.parametrize("M,N,K", [(40, 256, 512), (700, 1024, 1024), (1100, 5120, 25600)])
def test_a_failed_workspace_keeps_its_word_whatever_the_kernel(bwla, M, N, K):
    """The same for the kernels of many tokens, cut tiles among them: no output is written, and after the check the call is right."""
    rng = np.random.default_rng(M)
    a, sa, va = operand(rng, M, K, "nv", integers=True)
    w, sw, vw = operand(rng, N, K, "nv", integers=True)
    ws = bwla.new_fp4_workspace(M, K, N)
    ws[:4].view(torch.int32)[0] = 1
    out = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, 1, out=out, workspace=ws)
    assert bwla.bwla_check_status(ws) == bwla.BWLA_ERR_DEVICE_TIMEOUT and (out == 7).all()
    check_product(bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, 1, out=out, workspace=ws), va, vw, exact=True)
    assert bwla.bwla_check_status(ws) == 0 and not ws[:256].any()      # (arrival counters are back at zero)


# tiles of 256 x 256 in one round and a half, in fewer halves than pairs, cut in three; more than one round of whole tiles
CUT = [(1024, 5120, 25600), (1000, 1000, 32000), (250, 1030, 25600), (500, 3333, 20480), (2048, 2600, 12800), (1300, 4096, 8192), (2304, 2304, 512)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", CUT)
def test_product_of_tiles_cut_by_k(bwla, fmt, M, N, K):
    rng = np.random.default_rng([M, N, K, 3])
    a, sa, va = operand(rng, M, K, fmt)
    w, sw, vw = operand(rng, N, K, fmt)
    ra, rw = torch.rand(M, device="cuda") + 0.5, torch.rand(N, device="cuda") - 0.5
    ws = bwla.new_fp4_workspace(M, K, N)
    ws[256:].fill_(255)                              # what was in the scratch before is not looked at
    out = bwla.bwla_fp4_gemm_codes(a, sa, ra, w, sw, rw, FORMATS[fmt], workspace=ws)
    assert bwla.bwla_check_status(ws) == 0 and not ws[:256].any()
    check_product(out, va, vw, ra, rw)
    for _ in range(5):
        assert torch.equal(bwla.bwla_fp4_gemm_codes(a, sa, ra, w, sw, rw, FORMATS[fmt], workspace=ws), out)


@pytest.mark.parametrize("M", [1, 20, 130, 600])
@pytest.mark.parametrize("shift", [1, 2, 4, 8])
def test_outputs_off_16_bytes(bwla, M, shift):
    """The output begins anywhere on 2 bytes inside its rows; what is beside it stays."""
    rng = np.random.default_rng([M, shift])
    N, K = 520, 1024
    a, sa, va = operand(rng, M, K, "mx", integers=True)
    w, sw, vw = operand(rng, N, K, "mx", integers=True)
    wide = torch.full((M, N + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, 0, out=wide[:, shift:N + shift])
    check_product(wide[:, shift:N + shift], va, vw, exact=True)
    assert (wide[:, :shift] == 7).all() and (wide[:, N + shift:] == 7).all()


def test_a_single_row_of_any_stride(bwla):
    K, N = 96, 64
    x = torch.randn(K, 1, device="cuda").t()         # [1][K], row stride 1
    assert x.stride(0) == 1
    q = bwla.bwla_fp4_quantize_rows(x, 1)
    want = bwla.bwla_fp4_quantize_rows(x.clone(memory_format=torch.contiguous_format), 1)
    assert torch.equal(bwla.bwla_fp4_expand_rows(*q, 1), bwla.bwla_fp4_expand_rows(*want, 1))       # (scale bytes of rows beyond the last may differ)
    w = bwla.bwla_fp4_quantize_rows(torch.randn(N, K, device="cuda"), 1)
    out = torch.empty(N, 1, dtype=torch.bfloat16, device="cuda").t()
    assert torch.equal(bwla.bwla_fp4_gemm_codes(*q, *w, 1, out=out), bwla.bwla_fp4_gemm_codes(*want, *w, 1))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2,M", [(64, 64, 3), (64, 64, 500), (86, 128, 9), (64, 128, 400)])
def test_rotation_of_rows_off_16_bytes(bwla, fmt, n1, n2, M):
    rng = np.random.default_rng([n1, n2, M, 8])
    K = n1 * n2
    big = dev(rng.standard_normal((M, K + 3))).bfloat16()
    x = big[:, 1:K + 1]
    P1, P2 = haar(rng, n1), haar(rng, n2)
    check_rotated(bwla, x, P1, P2, fmt, bwla.bwla_rotate_quant_fp4(x, dev(P1), dev(P2), FORMATS[fmt]))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_other_streams(bwla, fmt):
    """Calls on two streams at once, with workspaces of their own."""
    K, N = 4096, 1024
    w = bwla.bwla_fp4_quantize_rows(torch.randn(N, K, device="cuda"), FORMATS[fmt])
    P1, P2 = dev(haar(np.random.default_rng(0), 64)), dev(haar(np.random.default_rng(1), 64))
    layer = bwla.bwla_fp4_layer_create(P1, P2, FORMATS[fmt], *w)
    xs = [torch.randn(M, K, device="cuda").bfloat16() for M in (5, 300)]
    want = [bwla.bwla_fp4_layer_linear(layer, x) for x in xs]
    wss = [bwla.new_fp4_layer_workspace(layer, x.shape[0]) for x in xs]
    outs = [torch.empty_like(y) for y in want]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, x, o, ws in zip(streams, xs, outs, wss):
            with torch.cuda.stream(s):
                bwla.bwla_fp4_layer_linear(layer, x, out=o, workspace=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(o, y) for o, y in zip(outs, want))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2", [(64, 64), (86, 128), (64, 88)])
def test_rotated_weights_without_a_synchronisation(bwla, fmt, n1, n2):
    """Weights that the kernel before makes (rotation and quantiser), read by the product at once."""
    g = torch.Generator(device="cuda").manual_seed(2)
    K, N, M = n1 * n2, 384, 16
    P1, P2 = dev(haar(np.random.default_rng(0), n1)), dev(haar(np.random.default_rng(1), n2))
    Ws = [torch.randn(N, K, device="cuda", generator=g).bfloat16() for _ in range(4)]
    a = bwla.bwla_fp4_quantize_rows(torch.randn(M, K, device="cuda", generator=g), FORMATS[fmt])
    ws, ws2 = bwla.new_fp4_workspace(M, K, N), bwla._fp4_scratch(bwla.bwla_rotate_quant_fp4_workspace_bytes(N, K, n1, n2), "cuda")
    want = []
    for W in Ws:
        q = bwla.bwla_rotate_quant_fp4(W, P1, P2, FORMATS[fmt])
        torch.cuda.synchronize()
        want.append(bwla.bwla_fp4_gemm_codes(*a, *q, FORMATS[fmt], workspace=ws))
        torch.cuda.synchronize()
        del q
    torch.cuda.synchronize()
    for _ in range(5):
        got = [bwla.bwla_fp4_gemm_codes(*a, *bwla.bwla_rotate_quant_fp4(W, P1, P2, FORMATS[fmt], workspace=ws2), FORMATS[fmt], workspace=ws) for W in Ws]
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M", [1, 128, 129, 1000])
def test_products_without_outputs(bwla, fmt, M):
    """No weight rows: an [M][0] tensor, with a workspace and without."""
    K = 64
    a = bwla.bwla_fp4_quantize_rows(torch.randn(M, K, device="cuda"), FORMATS[fmt])
    w = bwla.bwla_fp4_quantize_rows(torch.empty(0, K, device="cuda"), FORMATS[fmt])
    for ws in (None, bwla.new_fp4_workspace(M, K, 0)):
        assert bwla.bwla_fp4_gemm_codes(*a, *w, FORMATS[fmt], workspace=ws).shape == (M, 0)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_scratch_of_many_tokens_serves_fewer(bwla, fmt):
    """One workspace, made for the largest batch, for products and layers of all smaller ones (of some of which tiles are cut by k)."""
    rng = np.random.default_rng(11)
    K, N, most = 11008, 4096, 4096
    w, sw, vw = operand(rng, N, K, fmt, integers=True)
    ws = bwla.new_fp4_workspace(most, K, N)
    for M in (1153, 1, 3500, 129, 2100):
        a, sa, va = operand(rng, M, K, fmt, integers=True)
        check_product(bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, FORMATS[fmt], workspace=ws), va, vw, exact=True)
        assert bwla.bwla_check_status(ws) == 0 and not ws[:256].any()
    n1, n2 = 64, 128
    w = bwla.bwla_fp4_quantize_rows(torch.randn(N, n1 * n2, device="cuda"), FORMATS[fmt])
    layer = bwla.bwla_fp4_layer_create(dev(haar(rng, n1)), dev(haar(rng, n2)), FORMATS[fmt], *w)
    ws = bwla.new_fp4_layer_workspace(layer, most)
    for M in (3584, 1, 3500, 4096, 33):
        x = torch.randn(M, n1 * n2, device="cuda").bfloat16()
        assert torch.equal(bwla.bwla_fp4_layer_linear(layer, x, workspace=ws), bwla.bwla_fp4_layer_linear(layer, x))
        assert bwla.bwla_check_status(ws) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M", [1, 40, 600])
@pytest.mark.parametrize("N,K", [(512, 1024), (1536, 2048)])
def test_weights_made_by_a_kernel_that_lets_others_start(bwla, fmt, M, N, K):
    """Weights' codes and scales that the kernel directly before writes, which lets the next one start at once (a product, whose outputs are
    taken as codes: any bytes are) or is PyTorch's.  Two sets in turn, so that bytes of the round before give other outputs."""
    rng = np.random.default_rng([M, N, K, 21])
    a, sa, va = operand(rng, M, K, fmt)
    makers = []
    for _ in range(2):      # bf16 [N][K/4] are the bytes of codes [N][K/2]
        t, st, _ = operand(rng, N, 512, fmt)
        u, su, _ = operand(rng, K // 4, 512, fmt)
        makers.append((t, st, None, u, su, None))
    scales = [operand(rng, N, K, fmt)[1] for _ in range(2)]
    bytes_ = torch.empty(N, K // 4, dtype=torch.bfloat16, device="cuda")
    codes, sw = bytes_.view(torch.uint8), torch.empty_like(scales[0])
    ws, ws2 = bwla.new_fp4_workspace(N, 512, K // 4), bwla.new_fp4_workspace(M, K, N)
    want, made = [], []
    for m, s in zip(makers, scales):
        bwla.bwla_fp4_gemm_codes(*m, FORMATS[fmt], out=bytes_, workspace=ws)
        torch.cuda.synchronize()
        want.append(bwla.bwla_fp4_gemm_codes(a, sa, None, codes, s, None, FORMATS[fmt], workspace=ws2))
        torch.cuda.synchronize()
        made.append(codes.clone())
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        sw.copy_(scales[i % 2])
        bwla.bwla_fp4_gemm_codes(*makers[i % 2], FORMATS[fmt], out=bytes_, workspace=ws)
        got.append(bwla.bwla_fp4_gemm_codes(a, sa, None, codes, sw, None, FORMATS[fmt], workspace=ws2))
    for i in range(20):
        codes.copy_(made[i % 2])
        sw.copy_(scales[i % 2])
        got.append(bwla.bwla_fp4_gemm_codes(a, sa, None, codes, sw, None, FORMATS[fmt], workspace=ws2))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i % 2]) for i, y in enumerate(got))
    assert bwla.bwla_check_status(ws) == 0 and bwla.bwla_check_status(ws2) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M", [1, 2, 3, 4])
def test_pushed_sums_on_two_streams(bwla, fmt, M):
    """Few tokens, K cut over clusters of every size: calls on two streams beside one another, again and again."""
    shapes = [(256, 5120), (1000, 2048), (5120, 5120), (300, 25600)]
    rng = np.random.default_rng([M, 31])
    ops = [(*operand(rng, M, K, fmt, integers=True), *operand(rng, N, K, fmt, integers=True)) for N, K in shapes]
    streams = [torch.cuda.Stream() for _ in range(2)]
    wss = [[bwla.new_fp4_workspace(M, K, N) for N, K in shapes] for _ in streams]
    torch.cuda.synchronize()
    outs = []
    for i in range(25):
        for s, ws in zip(streams, wss):
            with torch.cuda.stream(s):
                outs.append([bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, FORMATS[fmt], workspace=x) for (a, sa, _, w, sw, _), x in zip(ops, ws)])
    torch.cuda.synchronize()
    for (_, _, va, _, _, vw), first, *rest in zip(ops, *outs):
        check_product(first, va, vw, exact=True)
        assert all(torch.equal(first, y) for y in rest)
    assert all(bwla.bwla_check_status(x) == 0 for ws in wss for x in ws)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2", [(32, 64), (64, 80), (86, 128), (160, 160)])
@pytest.mark.parametrize("M", [1, 300])
def test_a_layer_is_used_at_once(bwla, fmt, n1, n2, M):
    """Quantised weights, prepared factors and the first call one behind the other, nothing synchronised between them, in memory that held
    another layer before."""
    K, N = n1 * n2, 256
    rng = np.random.default_rng([n1, n2, M, 41])
    sets = [(dev(haar(rng, n1)), dev(haar(rng, n2)), torch.randn(N, K, device="cuda")) for _ in range(3)]
    x = torch.randn(M, K, device="cuda").bfloat16()
    q = bwla.bwla_fp4_quantize_rows(sets[0][2], FORMATS[fmt])
    want = []
    for P1, P2, W in sets:
        layer = bwla.bwla_fp4_layer_create(P1, P2, FORMATS[fmt], *bwla.bwla_fp4_quantize_rows(W, FORMATS[fmt], *q))
        torch.cuda.synchronize()
        want.append(bwla.bwla_fp4_layer_linear(layer, x))
        torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for P1, P2, W in sets:
            layer = bwla.bwla_fp4_layer_create(P1, P2, FORMATS[fmt], *bwla.bwla_fp4_quantize_rows(W, FORMATS[fmt], *q))
            got.append(bwla.bwla_fp4_layer_linear(layer, x))
            bwla.bwla_fp4_layer_destroy(layer)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_expansion_at_the_ends_of_fp32(bwla, dtype):
    """Which values come back as infinities, and what bf16 cannot hold: the header's numbers.  MX has neither."""
    rng = np.random.default_rng(51)
    unit = 2.0 ** 117
    x = np.zeros((64, 64))
    tops = np.r_[np.linspace(1700, 2047, 60), 2015.999, 2016.0, 2016.001, 2047.9]
    x[:, :16] = tops[:, None] * rng.choice([-1, 1], (64, 16)) * np.r_[1, rng.uniform(0.8, 1, 15)]
    x[:, 16:32] = rng.uniform(-2015, 2015, (64, 16))             # (a block of the same row without such a value)
    x[:, 1], x[:, 2] = 1760.0, 1760.001
    x[:, 0] = tops
    top = np.ascontiguousarray(x * unit, np.float32)
    small = (rng.uniform(-1, 1, (64, 64)) * np.exp2(rng.integers(-127, -112, (64, 1)))).astype(np.float32)
    for fmt in ("nv", "mx"):
        for rows in (top, small):
            q = bwla.bwla_fp4_quantize_rows(dev(rows), FORMATS[fmt])
            got = bwla.bwla_fp4_expand_rows(*q, FORMATS[fmt], dtype=dtype).double().cpu()
            want = torch.from_numpy(fp4.expand(*fp4.quantize(rows.astype(np.float64), fmt), fmt))      # (exact: 64 bits have room)
            beyond = want.abs() >= 2.0 ** 128
            v = np.abs(rows.astype(np.float64)) / unit
            says = (v > 1760) & np.repeat(v.reshape(64, 4, 16).max(2) > 2016, 16, 1) if fmt == "nv" else np.zeros(v.shape, bool)
            assert np.array_equal(beyond.numpy(), says)
            assert torch.equal(torch.isinf(got), beyond) and torch.equal(got[~beyond], want.to(dtype).double()[~beyond])
            exact = got == want
            assert exact[~beyond].all() or (fmt == "nv" and dtype is torch.bfloat16 and rows is small and exact[q[2].cpu() >= 2.0 ** -123].all())
    assert (tops > 2016).sum() > 3


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2", [(86, 128), (108, 128), (112, 128)])
@pytest.mark.parametrize("M", [1, 130, 1024, 2500])
def test_rows_off_16_bytes_have_the_codes_of_aligned_ones(bwla, fmt, n1, n2, M):
    K, N = n1 * n2, 200
    rng = np.random.default_rng([n1, M, 61])
    P1, P2 = dev(haar(rng, n1)), dev(haar(rng, n2))
    x = torch.randn(M, K + 3, device="cuda").bfloat16()[:, 1:K + 1]
    layer = bwla.bwla_fp4_layer_create(P1, P2, FORMATS[fmt], *bwla.bwla_fp4_quantize_rows(torch.randn(N, K, device="cuda"), FORMATS[fmt]))
    ws = bwla.new_fp4_layer_workspace(layer, M)
    nb = K // fp4.BLOCK[fmt]
    for call in (lambda x: bwla.bwla_fp4_layer_rotate_quant(layer, x, workspace=ws), lambda x: bwla.bwla_rotate_quant_fp4(x, P1, P2, FORMATS[fmt])):
        got, want = call(x), call(x.contiguous())
        assert torch.equal(got[0], want[0])
        assert np.array_equal(fp4.untile(got[1].cpu().numpy(), M, nb), fp4.untile(want[1].cpu().numpy(), M, nb))
        assert got[2] is None or torch.equal(got[2], want[2])
    assert torch.equal(bwla.bwla_fp4_layer_linear(layer, x, workspace=ws), bwla.bwla_fp4_layer_linear(layer, x.contiguous(), workspace=ws))
    assert bwla.bwla_check_status(ws) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2,M", [(32, 64, 5000), (64, 64, 4096), (64, 80, 4100), (64, 88, 2300), (86, 128, 2500), (112, 128, 1801)])
def test_rotation_of_many_steps(bwla, fmt, n1, n2, M):
    """Many steps a CTA follow one another: rows from all of them, the last ones among them."""
    K = n1 * n2
    rng = np.random.default_rng([n1, n2, M, 71])
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn(M, K, device="cuda", generator=g).bfloat16()
    x[M // 2] = 0
    P1, P2 = haar(rng, n1), haar(rng, n2)
    at = np.unique(np.r_[rng.integers(0, M, 160), 0, M // 2, np.arange(M - 24, M)])
    nb = K // fp4.BLOCK[fmt]
    layer = bwla.bwla_fp4_layer_create(dev(P1), dev(P2), FORMATS[fmt], *bwla.bwla_fp4_quantize_rows(torch.randn(8, K, device="cuda", generator=g), FORMATS[fmt]))
    first = None
    for codes, scales, rows in (bwla.bwla_rotate_quant_fp4(x, dev(P1), dev(P2), FORMATS[fmt]), bwla.bwla_fp4_layer_rotate_quant(layer, x), bwla.bwla_fp4_layer_rotate_quant(layer, x)):
        byte = fp4.untile(scales.cpu().numpy(), M, nb)
        i = torch.from_numpy(at).cuda()
        check_rotated(bwla, x[i], P1, P2, fmt, (codes[i], dev(fp4.tile(byte[at])), None if rows is None else rows[i]))
        again, first = first, (codes, byte)
    assert torch.equal(again[0], first[0]) and np.array_equal(again[1], first[1]), "a call must repeat itself bit for bit"


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [(2500, 18944, 512), (4096, 25600, 288), (3333, 8195, 1056)])
def test_product_of_many_full_rounds(bwla, fmt, M, N, K):
    rng = np.random.default_rng([M, N, K, 81])
    a, sa, va = operand(rng, M, K, fmt, integers=True)
    w, sw, vw = operand(rng, N, K, fmt, integers=True)
    ws = bwla.new_fp4_workspace(M, K, N)
    out = bwla.bwla_fp4_gemm_codes(a, sa, None, w, sw, None, FORMATS[fmt], workspace=ws)
    assert bwla.bwla_check_status(ws) == 0
    check_product(out, va, vw, exact=True)


def test_threads_with_layers_of_their_own(bwla):
    """Two threads, each with a layer, a workspace and a stream."""
    import threading
    K, N = 64 * 64, 1024
    jobs = []
    for i, (fmt, M) in enumerate((("mx", 3), ("nv", 300))):
        rng = np.random.default_rng([i, 91])
        w = bwla.bwla_fp4_quantize_rows(torch.randn(N, K, device="cuda"), FORMATS[fmt])
        layer = bwla.bwla_fp4_layer_create(dev(haar(rng, 64)), dev(haar(rng, 64)), FORMATS[fmt], *w)
        xs = [torch.randn(M, K, device="cuda").bfloat16() for _ in range(3)]
        jobs.append((layer, bwla.new_fp4_layer_workspace(layer, M), torch.cuda.Stream(), xs, [bwla.bwla_fp4_layer_linear(layer, x) for x in xs], []))
    torch.cuda.synchronize()

    def work(layer, ws, stream, xs, want, bad):
        with torch.cuda.stream(stream):
            for _ in range(40):
                got = [bwla.bwla_fp4_layer_linear(layer, x, workspace=ws) for x in xs]
                stream.synchronize()
                bad.extend(1 for u, v in zip(got, want) if not torch.equal(u, v))
        bad.append(0)

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(j[5] == [0] for j in jobs) and all(bwla.bwla_check_status(j[1]) == 0 for j in jobs)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("n1,n2,M", [(64, 64, 9), (86, 128, 9), (86, 128, 1100), (64, 88, 40)])
def test_rows_off_16_bytes_in_a_graph(bwla, fmt, n1, n2, M):
    K, N = n1 * n2, 320
    rng = np.random.default_rng([n1, n2, M, 101])
    layer = bwla.bwla_fp4_layer_create(dev(haar(rng, n1)), dev(haar(rng, n2)), FORMATS[fmt], *bwla.bwla_fp4_quantize_rows(torch.randn(N, K, device="cuda"), FORMATS[fmt]))
    x = torch.randn(M, K + 5, device="cuda").bfloat16()[:, 3:K + 3]
    ws, out = bwla.new_fp4_layer_workspace(layer, M), torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bwla.bwla_fp4_layer_linear(layer, x, out=out, workspace=ws)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for _ in range(3):
                bwla.bwla_fp4_layer_linear(layer, x, out=out, workspace=ws)
        for _ in range(3):
            x.copy_(torch.randn(M, K, device="cuda").bfloat16())
            g.replay()
            got = out.clone()
            assert torch.equal(got, bwla.bwla_fp4_layer_linear(layer, x))
    side.synchronize()
    assert bwla.bwla_check_status(ws) == 0
