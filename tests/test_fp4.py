"""Microscaled 4-bit floating point without a GPU: the oracle against the formats' own numbers, sizes, refusals."""
import ctypes as C

import numpy as np
import pytest

from oracle import fp4


@pytest.fixture(scope="module")
def lib():
    from paper_2605_00422_b200 import bwla
    return bwla._lib


def test_oracle_rounds_as_the_formats_say():
    assert fp4.E4M3[-1] == 448 and fp4.E4M3[1] == 2.0 ** -9
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9, 1e9])
    assert fp4.E2M1[fp4.nearest(ties, fp4.E2M1)].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 6]
    up = np.nextafter(ties, np.inf)
    assert fp4.E2M1[fp4.nearest(up, fp4.E2M1)].tolist() == [.5, 1, 1.5, 2, 3, 4, 6, 6, 6]
    # the scale of a block: the largest value lands in [4, 8)
    for top in (1.0, 1.99, 2.0, 6.0, 7.9, 8.0, 3e38, 2.0 ** -149):
        e = int(fp4.mx_exponent(np.float64(top)))
        assert (4 <= top / 2.0 ** e < 8) or e == -127
    # the scale of a row: the smallest power of two that brings the largest block's scale into e4m3's range
    for top in (2688.0, 2688.0001, 2687.9, 1.0, 1e-30, 3e38):
        E = int(fp4.nv_exponent(np.float64(top)))
        assert top <= 2688 * 2.0 ** E and top > 2688 * 2.0 ** (E - 1)
    v, s, r = fp4.quantize(np.array([[0.0] * 16 + [2688.0] * 8 + [1.0] * 8]), "nv")
    assert r[0] == 1 and s[0].tolist() == [0, 448] and v[0, 16] == 6 and v[0, -1] == 0
    for fmt in ("mx", "nv"):
        x = np.random.default_rng(1).standard_normal((3, 96))
        x[1, 40] = np.nan
        v, s, r = fp4.quantize(x, fmt)
        y = fp4.expand(v, s, r, fmt)
        assert np.isnan(y[1, 32:64]).all() and np.isnan(y[1]).all() == (fmt == "nv") and np.isfinite(y[[0, 2]]).all()
        assert np.array_equal(fp4.unpack(fp4.pack(v)), v)
        b = fp4.scale_bytes(s, fmt)
        assert np.array_equal(fp4.untile(fp4.tile(b), 3, b.shape[1]), b)
        assert np.array_equal(fp4.scales_of(b, fmt), s, equal_nan=True)


@pytest.mark.parametrize("rows,K,format,want", [(1, 32, 0, 512), (128, 128, 0, 512), (129, 160, 0, 2048), (1, 64, 1, 512), (333, 11008, 1, 3 * 172 * 512),
                                                 (0, 32, 0, 0), (1, 48, 0, 0), (1, 0, 0, 0), (-1, 32, 0, 0), (1, 32, 2, 0), (1, 1 << 25, 0, 0)])
def test_scale_bytes(lib, rows, K, format, want):
    assert lib.bwla_fp4_scale_bytes(rows, K, format) == want


def test_refusals_before_anything_runs(lib):
    """Bad arguments are refused before the device is looked at; good ones end at the missing device (here) or are not made."""
    buf = (C.c_uint8 * 4096)()
    at = (C.addressof(buf) + 255) // 256 * 256
    p, odd = C.c_void_p(at), C.c_void_p(at + 8)
    bad = -1
    q = lambda **k: lib.bwla_fp4_quantize_rows(*[{**dict(x=p, dtype=0, M=1, K=32, ldx=32, format=0, codes=p, scales=p, rows=p), **k}[n]
                                                for n in ("x", "dtype", "M", "K", "ldx", "format", "codes", "scales", "rows")], None)
    for k in (dict(x=None), dict(dtype=3), dict(dtype=-1), dict(M=-1), dict(K=0), dict(K=33), dict(K=16), dict(K=1 << 25, ldx=1 << 25), dict(ldx=31), dict(format=2),
              dict(codes=None), dict(codes=odd), dict(scales=None), dict(scales=odd), dict(format=1, rows=None), dict(M=1 << 31)):
        assert q(**k) == bad, k
    assert q(M=0, x=None, codes=None) == 0
    e = lambda **k: lib.bwla_fp4_expand_rows(*[{**dict(codes=p, scales=p, rows=None, M=1, K=32, format=0, out=p, dtype=1, ldo=32), **k}[n]
                                              for n in ("codes", "scales", "rows", "M", "K", "format", "out", "dtype", "ldo")], None)
    for k in (dict(codes=None), dict(scales=None), dict(out=None), dict(dtype=2), dict(ldo=31), dict(K=24), dict(format=-1), dict(M=-1), dict(codes=odd)):
        assert e(**k) == bad, k
    assert e(M=0) == 0
    names = ("ac", "as_", "ar", "M", "K", "wc", "ws", "wr", "N", "format", "out", "ldo", "work", "bytes")
    good = dict(ac=p, as_=p, ar=None, M=1, K=32, wc=p, ws=p, wr=None, N=8, format=0, out=p, ldo=8, work=p, bytes=256)
    g = lambda **k: lib.bwla_fp4_gemm_codes(*[{**good, **k}[n] for n in names], None)
    for k in (dict(ac=None), dict(as_=None), dict(wc=None), dict(ws=None), dict(out=None), dict(ldo=7), dict(K=31), dict(M=-1), dict(N=-1), dict(format=5), dict(ac=odd),
              dict(wc=odd), dict(as_=odd), dict(ws=odd), dict(out=C.c_void_p(at + 1))):
        assert g(**k) == bad, k
    for k in (dict(work=None), dict(work=odd), dict(bytes=255)):
        assert g(**k) == -3, k
    assert g(M=0) == 0 and g(N=0) == 0
    assert lib.bwla_fp4_gemm_workspace_bytes(1, 32, 8) >= 256 and lib.bwla_fp4_gemm_workspace_bytes(1, 33, 8) == 0
    r = lambda **k: lib.bwla_rotate_quant_fp4(*[{**dict(x=p, M=1, K=64, ldx=64, P1=p, n1=8, P2=p, n2=8, format=0, codes=p, scales=p, rows=p, work=p, bytes=1 << 20), **k}[n]
                                               for n in ("x", "M", "K", "ldx", "P1", "n1", "P2", "n2", "format", "codes", "scales", "rows", "work", "bytes")], None)
    for k in (dict(x=None), dict(K=96), dict(n1=9), dict(ldx=63), dict(P1=None), dict(P2=odd), dict(codes=odd), dict(format=1, rows=None), dict(M=-1), dict(format=2)):
        assert r(**k) == bad, k
    assert r(work=None) == -3 and r(bytes=255) == -3 and r(M=0) == 0
    h = C.c_void_p()
    c = lambda **k: lib.bwla_fp4_layer_create(C.byref(h), *[{**dict(K=64, N=8, P1=p, n1=8, P2=p, n2=8, format=0, wc=p, ws=p, wr=None, prepared=p, bytes=1 << 20), **k}[n]
                                              for n in ("K", "N", "P1", "n1", "P2", "n2", "format", "wc", "ws", "wr", "prepared", "bytes")], None)
    for k in (dict(K=96), dict(N=0), dict(P1=None), dict(wc=None), dict(ws=odd), dict(format=9), dict(n2=4)):
        assert c(**k) == bad, k
    assert c(prepared=None) == -3 and c(bytes=16) == -3
    assert lib.bwla_fp4_layer_linear(None, p, 1, 64, p, 8, p, 256, None) == bad
    assert lib.bwla_fp4_layer_rotate_quant(None, p, 1, 64, p, p, p, p, 256, None) == bad
    assert lib.bwla_fp4_layer_workspace_bytes(None, 1) == 0 and lib.bwla_fp4_layer_prepared_bytes(65, 8, 8) == 0
    import torch
    if not torch.cuda.is_available():
        assert q() == e() == g() == r() == c() == -2          # BWLA_ERR_UNSUPPORTED: nothing ran


def test_binding_refuses_what_the_library_cannot_see():
    """Shapes and types: TypeError before a pointer is taken (tensors here are on the CPU, or of the wrong kind)."""
    import torch

    from paper_2605_00422_b200 import bwla
    x = torch.zeros(2, 64)
    for call in (lambda: bwla.bwla_fp4_quantize_rows(x, 0), lambda: bwla.bwla_fp4_expand_rows(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8), None, 0),
                 lambda: bwla.bwla_fp4_gemm_codes(x, x, None, x, x, None, 0, out=x, workspace=x), lambda: bwla.bwla_rotate_quant_fp4(x, x, x, 0, workspace=x),
                 lambda: bwla.bwla_fp4_quantize_rows(x.double(), 0)):
        with pytest.raises((TypeError, RuntimeError)):
            call()

    class Other:
        _h, N, K = 1, 64, 64
    with pytest.raises((AttributeError, TypeError)):
        bwla._calls.fp4_linear(Other(), x.bfloat16(), x.bfloat16(), x)


def test_factors_that_are_not_square_are_refused():
    """The library reads n1 x n1 and n2 x n2 values."""
    import torch

    from paper_2605_00422_b200 import bwla
    x, eye = torch.zeros(2, 64, dtype=torch.bfloat16), torch.eye(8)
    w = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for P1, P2, name in ((eye[:, :4].contiguous(), eye, "P1"), (eye, eye[:, :4].contiguous(), "P2"), (eye[0], eye, "P1")):
        for call in (lambda: bwla.bwla_rotate_quant_fp4(x, P1, P2, 0, workspace=w[0].view(-1)), lambda: bwla.bwla_fp4_layer_create(P1, P2, 0, *w)):
            with pytest.raises(TypeError, match=f"{name}: expected a square matrix"):
                call()


PLANS = r"""
#include "host_plans.h"
#include <cstdio>
#include <vector>
using namespace bwla;
// The pieces of fp4_pair_kernel: every k-block of every tile belongs to one piece, the pairs that it works out for a cut tile are those that
// have parts of it, nobody leaves two sums in one place, and counters fit the status words.
static bool pieces(const Fp4PairPlan& r, int tiles, int kblocks) {
    std::vector<std::vector<int>> owner(tiles, std::vector<int>(kblocks, -1));
    const int pairs = r.pairs, rest_tiles = tiles - r.whole * pairs;
    const int64_t rest = (int64_t)rest_tiles * kblocks;
    if (rest_tiles < 0) return false;
    for (int pair = 0; pair < pairs; ++pair) {
        const int s0 = r.cut ? (int)(rest * pair / pairs) : std::min(pair, rest_tiles) * kblocks;
        const int s1 = r.cut ? (int)(rest * (pair + 1) / pairs) : std::min(pair + 1, rest_tiles) * kblocks;
        const int first = s0 / kblocks, count = r.whole + (s1 > s0 ? (s1 + kblocks - 1) / kblocks - first : 0);
        int left[2] = {0, 0};
        for (int i = 0; i < count; ++i) {
            int tile, kb0 = 0, kb1 = kblocks, rt = 0;
            if (i < r.whole) tile = pair + i * pairs;
            else { rt = first + i - r.whole; tile = r.whole * pairs + rt; kb0 = std::max(s0 - rt * kblocks, 0); kb1 = std::min(s1 - rt * kblocks, kblocks); }
            if (tile >= tiles || kb0 >= kb1) return false;
            for (int kb = kb0; kb < kb1; ++kb) { if (owner[tile][kb] >= 0) return false; owner[tile][kb] = pair; }
            if (kb1 - kb0 < kblocks) {
                if (!r.cut) return false;
                const int64_t begin = (int64_t)rt * kblocks;
                const int from = (int)(((begin + 1) * pairs - 1) / rest), to = (int)(((begin + kblocks) * pairs - 1) / rest);
                if (++left[kb0 == 0] > 1 || pair < from || pair > to || (kb0 == 0) != (pair == from) || from * 2 + 1 >= 256 - 4 * 4 || to - from + 1 > 255) return false;
            }
        }
    }
    for (int t = r.whole * pairs; t < tiles; ++t)
        if (r.cut) {
            const int64_t begin = (int64_t)(t - r.whole * pairs) * kblocks;
            if (owner[t][0] != (int)(((begin + 1) * pairs - 1) / rest) || owner[t][kblocks - 1] != (int)(((begin + kblocks) * pairs - 1) / rest)) return false;
        }
    for (auto& t : owner) for (int o : t) if (o < 0) return false;
    return true;
}
int main() {
    int cut = 0, pairs = 0;
    for (int64_t M : {1, 129, 256, 257, 333, 512, 1000, 1024, 2048, 4096, 9000})
        for (int64_t N : {1, 77, 256, 1000, 2600, 4095, 5120, 8192, 25600})
            for (int64_t K : {32, 256, 288, 1024, 5120, 11008, 25600})
                for (int device : {74, 70, 3})
                    for (int may : {1, 0}) {
                        const Fp4PairPlan r = fp4_pair_plan(M, K, N, device, may);
                        const int tiles = (int)(((M + 255) / 256) * ((N + 255) / 256)), kblocks = (int)((K + 255) / 256);
                        if (r.pairs < 1 || r.pairs > device || (r.cut && !may) || !pieces(r, tiles, kblocks)) { std::printf("%d %d %d: %d\n", (int)M, (int)N, (int)K, device); return 0; }
                        cut += r.cut; pairs += fp4_in_pairs(M, K, N);
                        if (fp4_part_bytes(r) > (size_t)74 * 2 * kFp4PartBytes) return 0;
                        for (int nv : {0, 1}) {      // (tiles beside one another start in even columns of their scales: at multiples of 64 tokens)
                            const Fp4SplitPlan q = fp4_split_plan(M, K, N, nv);
                            if ((q.tok != 16 && q.tok != 32 && q.tok != 64 && q.tok != 128) || (q.tok < 64 && M > q.tok) || q.parts < 1 || q.parts > std::min(8, kblocks) ||
                                (q.deep && q.tok < 64)) { std::printf("split %d\n", q.tok); return 0; }
                        }
                        for (int tok : {16, 32, 64, 128}) {
                            const int parts = fp4_split_parts(M, K, N, tok);
                            if (parts < 1 || parts > 8 || parts > kblocks) { std::printf("parts %d\n", parts); return 0; }
                        }
                    }
    // A call for microscaled codes of rotated rows that keeps no room for fp32 outputs finds a kernel whatever x's alignment, and that kernel's places fit
    for (int n1 = 1; n1 <= 192; ++n1)
        for (int n2 = 8; n2 <= 256; n2 += 8) {
            RotGeom g;
            if (n1 * n2 % 32 || n1 * n2 > 25600 || !rot_geometry(n1, n2, &g)) continue;
            int groups = 1;
            const bool mma = rot_fp4_groups(g, &groups);
            RotRowsGeom rows;
            const bool many = rot_rows_geometry(n1, n2, 1, &rows);
            if (many && (!rot_rows_fp4(rows) || rows.total > kRotMaxSmem || rows.exps < 2 * rows.tps * (rows.K / 16) || rows.staged)) { std::printf("rows %d x %d\n", n1, n2); return 0; }
            if (!rot_fp4_unfused(g) && (!mma || !(many || rot_mma_always(g)))) { std::printf("unfused %d x %d\n", n1, n2); return 0; }
            if (g.group_off % 16 || g.group_bytes % 16 || rot_fp4_group_bytes(g) % 16 || rot_fp4_group_bytes(g) < g.n1 * rot_fp4_row(g) * 4 + 2 * (g.K >> 4)) return 0;
        }
    std::printf("ok %d %d\n", cut > 20, pairs > 20);
}
"""


def test_plans_cover_their_work(tmp_path):
    import os
    import subprocess
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_00422_b200", "csrc")
    (tmp_path / "plans.cpp").write_text(PLANS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", csrc, "-o", str(tmp_path / "plans"), str(tmp_path / "plans.cpp")], check=True)
    r = subprocess.run([str(tmp_path / "plans")], capture_output=True, text=True, timeout=120)
    assert r.stdout == "ok 1 1\n", (r.returncode, r.stdout)


def test_workspace_of_products_without_outputs():
    """N == 0 is a no-op for any number of tokens, its workspace the status words alone; in a process of its own, which a division by zero would end."""
    import os
    import subprocess
    import sys
    code = ("from paper_2605_00422_b200 import bwla\n"
            "print(*[bwla.bwla_fp4_gemm_workspace_bytes(M, K, 0) for M in (0, 1, 128, 129, 4096, 100000) for K in (64, 5120)])\n"
            "print(*[bwla._lib.bwla_fp4_gemm_codes(256, 256, None, M, 64, 256, 256, None, 0, 0, 256, 0, 256, 256, None) for M in (1, 129, 4096)])\n")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and r.stdout.split("\n")[:2] == [" ".join(["256"] * 12), "0 0 0"], (r.returncode, r.stdout, r.stderr)


SIZES = r"""
#include "host_plans.h"
#include <cstdio>
using namespace bwla;
// Scratch made for M tokens is enough for every smaller number of them, and never falls as M grows.
int main() {
    int cut = 0, kept = 0;
    for (int64_t N : {1, 77, 256, 1000, 4096, 5120, 8192, 11008, 25600})
        for (int64_t K : {32, 256, 2048, 5120, 8192, 11008, 25600, 65536}) {
            size_t most = 0, before = 0;
            for (int64_t M = 0; M <= 45000; M += M < 2500 ? 1 : 127) {
                const size_t need = fp4_in_pairs(M, K, N) ? fp4_part_bytes(fp4_pair_plan(M, K, N, kFp4Pairs, true)) : 0, room = fp4_part_bytes_up_to(M, K, N);
                most = std::max(most, need);
                if (room < most || room < before || room > (size_t)kFp4Pairs * 2 * kFp4PartBytes) { std::printf("%d %d %d: %zu of %zu\n", (int)M, (int)K, (int)N, room, most); return 0; }
                if (M <= 2048 && room != most) { std::printf("%d %d %d: %zu for %zu\n", (int)M, (int)K, (int)N, room, most); return 0; }
                before = room; cut += need > 0; kept += room > need;
            }
        }
    std::printf("ok %d %d\n", cut > 1000, kept > 1000);
}
"""


def test_scratch_of_many_tokens_serves_fewer(lib, tmp_path):
    import os
    import subprocess
    big = lib.bwla_fp4_gemm_workspace_bytes(4096, 11008, 4096)
    buf = (C.c_uint8 * 4096)()
    p = C.c_void_p((C.addressof(buf) + 255) // 256 * 256)
    import torch
    for M in (1, 128, 129, 1000, 1153, 2048, 3500, 4000, 4095, 4096):
        assert lib.bwla_fp4_gemm_workspace_bytes(M, 11008, 4096) <= big
        if not torch.cuda.is_available():      # (refused for the missing device, not for the workspace)
            assert lib.bwla_fp4_gemm_codes(p, p, None, M, 11008, p, p, None, 4096, 0, p, 4096, p, big, None) == -2
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_00422_b200", "csrc")
    (tmp_path / "sizes.cpp").write_text(SIZES)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", csrc, "-o", str(tmp_path / "sizes"), str(tmp_path / "sizes.cpp")], check=True)
    r = subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, timeout=300)
    assert r.stdout == "ok 1 1\n", (r.returncode, r.stdout)


def test_pointers_off_their_elements_are_refused(lib):
    """What the kernels read or write in whole elements has to lie on them."""
    buf = (C.c_uint8 * 4096)()
    at = (C.addressof(buf) + 255) // 256 * 256
    p, one, two = C.c_void_p(at), C.c_void_p(at + 1), C.c_void_p(at + 2)
    quantize = lambda x, dtype, rows: lib.bwla_fp4_quantize_rows(x, dtype, 1, 32, 32, 1, p, p, rows, None)
    expand = lambda out, dtype, rows: lib.bwla_fp4_expand_rows(p, p, rows, 1, 32, 1, out, dtype, 32, None)
    gemm = lambda a, w, out: lib.bwla_fp4_gemm_codes(p, p, a, 1, 32, p, p, w, 8, 1, out, 8, p, 256, None)
    rotate = lambda x, rows: lib.bwla_rotate_quant_fp4(x, 1, 64, 64, p, 8, p, 8, 1, p, p, rows, p, 1 << 20, None)
    h = C.c_void_p()
    create = lambda w: lib.bwla_fp4_layer_create(C.byref(h), 64, 8, p, 8, p, 8, 1, p, p, w, p, 1 << 20, None)
    for st in (quantize(one, 0, p), quantize(two, 0, p), quantize(one, 1, p), quantize(one, 2, p), quantize(p, 0, two), expand(one, 0, None), expand(two, 0, None),
               expand(one, 1, None), expand(p, 1, two), gemm(two, None, p), gemm(None, one, p), gemm(None, None, one), rotate(one, p), rotate(p, two), create(two)):
        assert st == -1
    import torch
    if not torch.cuda.is_available():          # on their elements they are taken: what is refused here is the missing device
        assert quantize(two, 1, p) == quantize(two, 2, p) == expand(two, 1, None) == gemm(None, None, two) == rotate(two, p) == create(None) == -2


@pytest.mark.parametrize("n1,n2", [(86, 128), (108, 128), (112, 128)])
def test_room_for_rows_off_16_bytes_is_bounded(lib, n1, n2):
    """Factors whose every aligned call writes codes at once keep no rotated values, only some rows to copy unaligned ones to."""
    K = n1 * n2
    size = lambda M: lib.bwla_rotate_quant_fp4_workspace_bytes(M, K, n1, n2)
    assert size(1) <= 256 + 2 * K + 256 and size(4096) == size(1 << 20) == 256 + 1024 * 2 * K
    assert size(0) == 256 and all(size(M) <= size(M + 1) for M in (0, 1, 5, 127, 1023, 1024))
