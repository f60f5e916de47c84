"""CPU checks of the layer's operators (layer norm, expert sort, dispatch and combine, microscaled 4-bit products): arguments
that the host refuses before anything is launched, sizes that it computes, the rule that picks a product's tile, and the
oracle's microscaled 4-bit quantizer against exact arithmetic."""

import ctypes
import os
import shutil
import subprocess
import sys
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "oracle"))
import ufp4_oracle as O  # noqa: E402

OK, INVALID, SHAPE, ALIGN, MISMATCH, UNSUPPORTED = 0, 1, 2, 3, 4, 5
F32, BF16 = U.OUT_F32, U.OUT_BF16
FAKE = 1 << 20  # never dereferenced: every call below fails validation or has nothing to do
R = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(U.library_path()):
        pytest.skip("libufp4.so not built")
    return U.lib()


def desc(rows=16, red=128, fmt=U.E2M1_MX32, rht_block=0, codes=FAKE, scales=FAKE, cld=None, sld=None, panels=None, layout=0):
    d = U.QDesc(codes=codes, scales=scales, code_panel_ld=cld or max(16, red // 32 * 2048),
                scale_panel_ld=sld or max(16, (red + 127) // 128 * 512), panels=panels or max(1, (rows + 127) // 128), rows=rows,
                red=red, format=fmt, rht_block=rht_block, layout=layout)
    for k in range(8):
        d.sign_words[k] = 0
    return d


# ------------------------------------------------------------------------------------------------
# sizes
# ------------------------------------------------------------------------------------------------

def test_microscaled_operand_bytes(lib):
    p, c, s = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    cb, sb = ctypes.c_size_t(), ctypes.c_size_t()
    # 129 rows: two panels; five 32-blocks: 5 x 128 x 16 bytes of codes, and scales in two groups of four blocks
    assert lib.ufp4_qtensor_bytes(4, 129, 160, R(p), R(c), R(s), R(cb), R(sb)) == OK
    assert (p.value, c.value, s.value, cb.value, sb.value) == (2, 10240, 1024, 20480, 2048)
    assert lib.ufp4_qtensor_bytes(4, 0, 0, R(p), R(c), R(s), None, None) == OK
    assert (p.value, c.value, s.value) == (1, 16, 16)
    assert lib.ufp4_qtensor_bytes(4, 16, 48, None, None, None, None, None) == SHAPE
    assert lib.ufp4_qtensor_bytes(5, 16, 32, None, None, None, None, None) == INVALID


def test_workspaces(lib):
    b = ctypes.c_size_t(7)
    norm, sort = lib.ufp4_layer_norm_bwd_workspace, lib.ufp4_moe_sort_workspace
    for dt in (F32, BF16):
        assert norm(dt, 0, 2048, R(b)) == OK and b.value == 0
        assert norm(dt, 1, 2048, R(b)) == OK and b.value == 2 * 2048 * 4
        # one partial row of both sums per workgroup, at most one workgroup a CU
        assert norm(dt, 1 << 20, 2048, R(b)) == OK and b.value == 256 * 2 * 2048 * 4
        assert norm(dt, 1 << 40, 1 << 30, R(b)) == OK and 0 < b.value <= 256 * 2 * 4 << 30
        assert norm(dt, 5, (1 << 30) + 1, R(b)) == UNSUPPORTED
        assert norm(dt, -1, 8, R(b)) == INVALID and norm(dt, 8, -1, R(b)) == INVALID and norm(dt, 8, 8, None) == INVALID
    assert norm(2, 8, 8, R(b)) == INVALID
    assert sort(0, 1, 1, R(b)) == OK and b.value == 0
    assert sort(7, 6, 64, R(b)) == OK and b.value == 0  # one workgroup
    assert sort(16384, 6, 64, R(b)) == OK and b.value == (24 + 1) * 64 * 4
    assert sort(-1, 1, 1, R(b)) == INVALID and sort(1, 0, 1, R(b)) == INVALID and sort(1, 1, 0, R(b)) == INVALID
    assert sort(1, 1, 1, None) == INVALID
    assert sort(1, 65, 1, R(b)) == UNSUPPORTED and sort(1, 1, 1025, R(b)) == UNSUPPORTED
    assert sort((1 << 31) // 8, 8, 4, R(b)) == UNSUPPORTED and sort((1 << 31) // 8 - 1, 8, 4, R(b)) == OK


# ------------------------------------------------------------------------------------------------
# refusals
# ------------------------------------------------------------------------------------------------

def test_layer_norm_refusals(lib):
    def call(dt=BF16, x=FAKE, rows=4, cols=8, ldx=8, wdt=F32, gamma=FAKE, beta=FAKE, eps=1e-5, y=FAKE, ldy=8, mean=FAKE, rstd=FAKE):
        return lib.ufp4_layer_norm(dt, x, rows, cols, ldx, wdt, gamma, beta, eps, y, ldy, mean, rstd, None)

    assert call(rows=0, x=None, y=None) == OK and call(cols=0, x=None, y=None, ldx=0, ldy=0) == OK
    assert call(dt=2) == INVALID and call(wdt=-1) == INVALID and call(rows=-1) == INVALID and call(cols=-1) == INVALID
    for eps in (-1e-9, float("nan"), float("inf")):
        assert call(eps=eps) == INVALID
    assert call(x=None) == INVALID and call(y=None) == INVALID
    assert call(ldx=7) == SHAPE and call(ldy=7) == SHAPE
    assert call(x=FAKE + 1) == ALIGN and call(y=FAKE + 1) == ALIGN and call(dt=F32, x=FAKE + 2) == ALIGN
    assert call(gamma=FAKE + 2) == ALIGN and call(beta=FAKE + 2) == ALIGN and call(wdt=BF16, gamma=FAKE + 1) == ALIGN
    assert call(mean=FAKE + 2) == ALIGN and call(rstd=FAKE + 2) == ALIGN
    assert call(cols=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31) == UNSUPPORTED


def test_layer_norm_bwd_refusals(lib):
    def call(dt=BF16, dy=FAKE, lddy=8, x=FAKE, rows=4, cols=8, ldx=8, wdt=F32, gamma=FAKE, mean=FAKE, rstd=FAKE, dx=FAKE, lddx=8,
             dg=FAKE, db=FAKE, ws=FAKE, n=1 << 20):
        return lib.ufp4_layer_norm_bwd(dt, dy, lddy, x, rows, cols, ldx, wdt, gamma, mean, rstd, dx, lddx, dg, db, ws, n, None)

    assert call(rows=0, dy=None, x=None, dx=None, mean=None, rstd=None, dg=None, db=None, ws=None) == OK
    assert call(cols=0, dy=None, x=None, dx=None) == OK
    assert call(dt=3) == INVALID and call(wdt=2) == INVALID and call(rows=-2) == INVALID and call(cols=-2) == INVALID
    for k in ("dy", "x", "dx", "mean", "rstd", "ws"):
        assert call(**{k: None}) == INVALID, k
    for k in ("lddy", "ldx", "lddx"):
        assert call(**{k: 7}) == SHAPE, k
    assert call(n=4 * 2 * 8 * 4 // 64 - 1) == SHAPE and call(dg=None, n=0) == SHAPE
    for k in ("dy", "x", "dx"):
        assert call(**{k: FAKE + 1}) == ALIGN, k
    for k in ("gamma", "mean", "rstd", "dg", "db"):
        assert call(**{k: FAKE + 2}) == ALIGN, k
    assert call(ws=FAKE + 8) == ALIGN
    big = dict(cols=(1 << 30) + 1, lddy=1 << 31, ldx=1 << 31, lddx=1 << 31)
    assert call(**big) == UNSUPPORTED


def test_sort_refusals(lib):
    def call(ids=FAKE, bits=64, tokens=4000, k=2, e=4, off=FAKE, rows=FAKE, src=FAKE, ws=FAKE, n=1 << 20):
        return lib.ufp4_moe_sort(ids, bits, tokens, k, e, off, rows, src, ws, n, None)

    assert call(bits=16) == INVALID and call(tokens=-1) == INVALID and call(k=0) == INVALID and call(e=0) == INVALID
    assert call(ids=None) == INVALID and call(off=None) == INVALID and call(rows=None) == INVALID and call(ws=None) == INVALID
    assert call(n=3 * 4 * 4 - 1) == SHAPE
    assert call(ids=FAKE + 4) == ALIGN and call(bits=32, ids=FAKE + 2) == ALIGN and call(off=FAKE + 4) == ALIGN
    assert call(rows=FAKE + 2) == ALIGN and call(src=FAKE + 2) == ALIGN and call(ws=FAKE + 2) == ALIGN
    assert call(k=65) == UNSUPPORTED and call(e=1025) == UNSUPPORTED and call(tokens=1 << 30) == UNSUPPORTED


def test_dispatch_and_combine_refusals(lib):
    def dispatch(dt=BF16, x=FAKE, tokens=3, cols=8, ldx=8, rows=FAKE, k=2, off=FAKE, e=4, w=FAKE, y=FAKE, yrows=6, ldy=8):
        return lib.ufp4_moe_dispatch(dt, x, tokens, cols, ldx, rows, k, off, e, w, y, yrows, ldy, None)

    def combine(dt=BF16, y=FAKE, yrows=6, cols=8, ldy=8, rows=FAKE, tokens=3, k=2, w=FAKE, out=FAKE, ldo=8):
        return lib.ufp4_moe_combine(dt, y, yrows, cols, ldy, rows, tokens, k, w, out, ldo, None)

    def bwd(dt=BF16, dout=FAKE, tokens=3, cols=8, lddo=8, y=FAKE, yrows=6, ldy=8, rows=FAKE, k=2, off=FAKE, e=4, w=FAKE, dy=FAKE,
            lddy=8, dw=FAKE):
        return lib.ufp4_moe_combine_bwd(dt, dout, tokens, cols, lddo, y, yrows, ldy, rows, k, off, e, w, dy, lddy, dw, None)

    assert dispatch(tokens=0, yrows=0, x=None, y=None, rows=None) == OK and combine(tokens=0, out=None, rows=None) == OK
    assert bwd(tokens=0, yrows=0, dout=None, y=None, dy=None, rows=None, dw=None) == OK
    for f in (dispatch, combine, bwd):
        assert f(dt=4) == INVALID and f(tokens=-1) == INVALID and f(cols=-1) == INVALID and f(k=0) == INVALID
        assert f(yrows=-1) == INVALID and f(rows=None) == INVALID
        assert f(rows=FAKE + 2) == ALIGN and f(w=FAKE + 2) == ALIGN and f(y=FAKE + 1) == ALIGN
        assert f(ldy=7) == SHAPE
        assert f(k=65, yrows=195) == UNSUPPORTED and f(tokens=1 << 24, yrows=1 << 25) == UNSUPPORTED
        assert f(tokens=1 << 30, yrows=1 << 31) == UNSUPPORTED
    for f in (dispatch, bwd):
        assert f(off=None) == INVALID and f(e=0) == INVALID and f(off=FAKE + 4) == ALIGN and f(yrows=5) == SHAPE
    assert dispatch(x=None) == INVALID and dispatch(y=None) == INVALID and dispatch(ldx=7) == SHAPE and dispatch(x=FAKE + 1) == ALIGN
    assert combine(out=None) == INVALID and combine(ldo=7) == SHAPE and combine(out=FAKE + 1) == ALIGN
    assert bwd(dout=None) == INVALID and bwd(dy=None) == INVALID and bwd(dw=None) == INVALID and bwd(lddo=7) == SHAPE
    assert bwd(lddy=7) == SHAPE and bwd(dw=FAKE + 2) == ALIGN and bwd(dy=FAKE + 1) == ALIGN


def test_microscaled_quantizer_refusals(lib):
    def call(x=FAKE, rows=64, cols=64, ld=64, transpose=0, rht=0, mask=0, rounding=0, out=None):
        return lib.ufp4_mxfp4_quantize(x, rows, cols, ld, transpose, rht, mask, rounding, 0, 0, R(out or desc(128, 128)), None)

    assert call(x=None) == INVALID and call(rows=-1) == INVALID and call(rounding=2) == INVALID
    assert call(cols=48, ld=48) == SHAPE and call(rows=48, transpose=1) == SHAPE and call(ld=56) == SHAPE
    assert call(x=FAKE + 2) == ALIGN and call(ld=65) == SHAPE
    assert call(out=desc(codes=FAKE + 8)) == ALIGN and call(out=desc(codes=None)) == INVALID
    assert call(out=desc(64, 64, cld=2048)) == SHAPE and call(out=desc(64, 64, sld=256)) == SHAPE
    assert call(rows=129, out=desc(64, 64, panels=1)) == SHAPE


def test_microscaled_product_refusals(lib):
    a, b = desc(8, 128), desc(24, 128)

    def call(x=a, w=b, y=FAKE, ldc=24, dt=BF16, f=lib.ufp4_mxfp4_gemm_fwd_y):
        return f(R(x), R(w), y, ldc, dt, None)

    for f in (lib.ufp4_mxfp4_gemm_fwd_y, lib.ufp4_mxfp4_gemm_bwd_dx, lib.ufp4_mxfp4_gemm_bwd_dw):
        assert call(x=desc(0, 128), y=None, f=f) == OK
        assert call(y=None, f=f) == INVALID and call(dt=2, f=f) == INVALID and call(ldc=23, f=f) == SHAPE
        assert call(w=desc(24, 96), f=f) == MISMATCH and call(w=desc(24, 128, rht_block=16), f=f) == MISMATCH
        assert call(w=desc(24, 128, fmt=U.UNIFORM_MX32, cld=4 * 3072), f=f) == MISMATCH
        assert call(w=desc(24, 128, fmt=3), f=f) == INVALID
    # the other products do not take this format
    assert lib.ufp4_gemm_fwd_y(R(a), R(b), FAKE, 24, BF16, None) == MISMATCH
    assert lib.ufp4_mx_gemm_fwd_y(R(a), R(b), FAKE, 24, BF16, None) == MISMATCH


def test_grouped_product_refusals(lib):
    x, w = desc(256, 128, layout=1), desc(512, 128)

    def fwd(x=x, w=w, off=FAKE, g=4, m=100, ldc=128):
        return lib.ufp4_mxfp4_gemm_fwd_y_grouped(R(x), R(w), off, g, m, FAKE, ldc, BF16, None)

    assert fwd(off=None) == INVALID and fwd(g=0) == INVALID and fwd(m=-1) == INVALID
    assert fwd(x=desc(256, 128)) == MISMATCH and fwd(ldc=127) == SHAPE
    assert fwd(w=desc(1025 * 128, 128), g=1025) == UNSUPPORTED

    def dx(dy=desc(256, 96, layout=1), wt=desc(64, 4 * 96), g=4):
        return lib.ufp4_mxfp4_gemm_bwd_dx_grouped(R(dy), R(wt), FAKE, g, 100, FAKE, 64, BF16, None)

    assert dx() == UNSUPPORTED and dx(wt=desc(64, 4 * 128)) == MISMATCH

    def dw(a=desc(64, 256, layout=2), b=desc(96, 256, layout=2), g=4, ldc=96):
        return lib.ufp4_mxfp4_gemm_bwd_dw_grouped(R(a), R(b), FAKE, g, FAKE, ldc, F32, None)

    assert dw(a=desc(64, 256)) == MISMATCH and dw(a=desc(64, 128, layout=2)) == MISMATCH and dw(ldc=95) == SHAPE
    assert dw(g=0) == INVALID and dw(g=1025) == UNSUPPORTED


def test_few_token_product_refusals(lib):
    def call(x=FAKE, rows=3, ldx=128, w=desc(24, 128), y=FAKE, ldc=24, dt=BF16):
        return lib.ufp4_mxfp4_linear(x, rows, ldx, R(w), y, ldc, dt, None)

    assert call(rows=0, x=None, y=None) == OK
    assert call(x=None) == INVALID and call(y=None) == INVALID and call(rows=-1) == INVALID and call(dt=2) == INVALID
    assert call(ldx=120) == SHAPE and call(ldc=23) == SHAPE and call(x=FAKE + 8) == ALIGN and call(ldx=132) == SHAPE
    assert call(rows=17) == UNSUPPORTED and call(w=desc(24, 128, rht_block=16)) == UNSUPPORTED
    assert call(w=desc(24, 128, layout=1)) == MISMATCH and call(w=desc(24, 128, fmt=U.UNIFORM_MX32, cld=4 * 3072)) == MISMATCH


def test_dequantize_refusals(lib):
    def call(q=desc(24, 128), out=FAKE, ldo=128):
        return lib.ufp4_mxfp4_dequantize(R(q), out, ldo, None)

    assert lib.ufp4_mxfp4_dequantize(None, FAKE, 128, None) == INVALID
    assert call(out=None) == INVALID and call(ldo=120) == SHAPE and call(out=FAKE + 8) == ALIGN and call(ldo=132) == SHAPE
    assert call(q=desc(24, 128, fmt=U.UNIFORM_MX32, cld=4 * 3072)) == MISMATCH and call(q=desc(24, 128, fmt=9)) == INVALID


# ------------------------------------------------------------------------------------------------
# the rule that picks a product's tile
# ------------------------------------------------------------------------------------------------

TILES = ("256", "128", "64", "64 in four teams")
# us of each tile: rows, columns, reduction (bf16 output)
TILE_TIMES = [
    (8192, 8192, 2048, (78, 89, 155, 266)), (8192, 4096, 1024, (31, 29.5, 46, 99)), (4096, 4096, 4096, (36.4, 42.0, 67.9, 100)),
    (2048, 2048, 2048, (16.3, 9.5, 11.3, 17.9)), (256, 8192, 2048, (15.8, 9.0, 7.5, 10.4)),
    (64, 2048, 8192, (38.3, 20.4, 14.8, 11.7)), (256, 256, 32768, (133, 67.3, 49.0, 33.6)),
    (1024, 8192, 2048, (17.9, 14.9, 21.4, 35.5)), (2048, 4096, 1024, (13.0, 9.7, 12.9, 26.3)), (512, 512, 512, (9.5, 6.8, 6.8, 7.4)),
    (4096, 2048, 8192, (51.9, 41.4, 68.0, 94.5)), (2048, 1408, 2048, (17.1, 9.2, 9.8, 14.6)),
]


@pytest.mark.parametrize("m,n,red,us", TILE_TIMES)
def test_the_tile_taken_is_among_the_fastest(lib, m, n, red, us):
    fn = ctypes.CDLL(U.library_path()).ufp4_plan_gemm_mxfp4
    k = fn(0, *map(ctypes.c_int64, (m, n, red)), ctypes.c_int32(1), ctypes.c_int64(m))
    assert us[k] <= 1.1 * min(us), TILES[k]


def test_a_smaller_tile_is_not_taken_past_its_grid(lib):
    """What the largest tile's grid holds launches whatever the rule would like better."""
    fn = ctypes.CDLL(U.library_path()).ufp4_plan_gemm_mxfp4
    for m, n in ((1 << 30, 256), (256, 1 << 30), (1 << 23, 1 << 15)):
        k = fn(0, *map(ctypes.c_int64, (m, n, 32)), ctypes.c_int32(1), ctypes.c_int64(m))
        side, threads = ((256, 512), (128, 256), (64, 256), (64, 1024))[k]
        assert -(-m // side) * -(-n // side) * threads < 1 << 32


# ------------------------------------------------------------------------------------------------
# the oracle's quantizer against exact arithmetic
# ------------------------------------------------------------------------------------------------

LEVELS = [Fraction(v) for v in ("0", "1/2", "1", "3/2", "2", "3", "4", "6")]


def _nearest(v):
    """(index, sign) of the level nearest to v, ties to the even index, cut at 6."""
    a = min(abs(v), Fraction(6))
    best = min(range(8), key=lambda i: (abs(a - LEVELS[i]), i & 1))
    return best if v >= 0 else -best


def test_microscaled_oracle_against_exact_arithmetic():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 96)) * np.exp2(rng.integers(-40, 40, (6, 96)) * (rng.random((6, 96)) < 0.3))
    x[0, :32] = 0
    x[1, :32] = np.arange(32) / 4 - 4  # ties of every kind
    x[2, :32] = 2.0**-133  # below the smallest scale's levels
    x[3, :32] = 3e38
    x = x.astype(np.float32)
    bits = (x.view(np.uint32) + 0x8000) & 0xFFFF0000
    x = bits.view(np.float32)
    codes, e8 = O.quantize_rows_mxfp4(x, O.RTNE, False)
    for r in range(6):
        for b in range(3):
            blk = [Fraction(float(v)) for v in x[r, 32 * b : 32 * b + 32]]
            top = max(abs(v) for v in blk)
            e = -127
            while top >= Fraction(2) ** (e + 3):
                e += 1
            assert int(e8[r, b]) == e + 127
            assert [int(c) for c in codes[r, 32 * b : 32 * b + 32]] == [_nearest(v / Fraction(2) ** e) for v in blk]


def test_microscaled_oracle_stochastic_rounding_stays_between_neighbours():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((64, 64)).astype(np.float32)
    codes, e8 = O.quantize_rows_mxfp4(x, O.SR, False, seed=3)
    scale = np.exp2(np.repeat(e8.astype(np.int64) - 127, 32, axis=-1).astype(np.float64))
    v = np.clip(x / scale, -6, 6)
    lv = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    q = np.sign(codes) * lv[np.abs(codes)]
    assert np.allclose(O.dequantize_mxfp4(codes, e8), q * scale, rtol=0, atol=0)
    lo = lv[np.searchsorted(lv, np.abs(v), side="right") - 1]
    hi = lv[np.minimum(np.searchsorted(lv, np.abs(v), side="left"), 7)]
    assert ((np.abs(q) == lo) | (np.abs(q) == hi)).all()
    # unbiased: the mean error of 4096 roundings, each of variance up to 1 (a step of 2 halves at most)
    assert abs(float((q - v).mean())) < 5 * 0.5 / 64


# ------------------------------------------------------------------------------------------------
# the binding's host module
# ------------------------------------------------------------------------------------------------

def test_host_module_refuses_before_the_library(lib):
    """Tensors that the calls cannot take: ValueError, and TypeError for what is no tensor; nothing is launched."""
    h, null = U._host(), 0  # the stream
    x, rows, off = torch.zeros(2, 32, dtype=torch.bfloat16), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    v, a = torch.zeros(2), ctypes.addressof
    d, other = desc(2, 32), desc(2, 64)
    calls = [
        lambda t: h.layer_norm(t, None, None, 1e-5, None, null), lambda t: h.layer_norm_bwd(x, t, None, v, v, True, None, null),
        lambda t: h.moe_sort(t, 4, null), lambda t: h.moe_dispatch(t, rows, off, None, None, null),
        lambda t: h.moe_combine(t, rows, None, None, null), lambda t: h.moe_combine_bwd(x, t, rows, off, None, None, null),
        lambda t: h.mxfp4_quantize(t, False, False, 0, 0, 0, 0, a(d), False, null), lambda t: h.mxfp4_linear(t, a(d), BF16, None, 16, null),
    ]
    for call in calls:
        with pytest.raises(ValueError, match="CUDA"):
            call(x)
        with pytest.raises(TypeError, match="tensor"):
            call(3)
    codes = torch.zeros(1, 2048, dtype=torch.uint8)
    with pytest.raises(ValueError, match="out_dtype"):
        h.mxfp4_gemm_fwd_y(codes, a(d), a(d), -1, None, null)
    for bad in (torch.zeros(2, 3), torch.zeros(2, 2, dtype=torch.float64), torch.zeros(2, 2).t()[:, :1]):
        with pytest.raises(ValueError, match="out"):
            h.mxfp4_gemm_fwd_y(codes, a(d), a(d), BF16, bad, null)
    with pytest.raises(ValueError, match="bf16"):
        h.mxfp4_dequantize(codes, a(d), torch.zeros(2, 32), null)
    with pytest.raises(U.UFP4Error) as e:  # a status of the library: its number and the call's name
        h.mxfp4_gemm_fwd_y(codes, a(d), a(other), F32, torch.zeros(2, 2), null)
    assert e.value.status == MISMATCH and "ufp4_mxfp4_gemm_fwd_y" in str(e.value)
    with pytest.raises(TypeError, match="arguments"):
        h.layer_norm(x)


def test_host_module_refuses_grouped_calls_before_the_library(lib):
    """The same of the grouped calls and of the two-operand quantizer, and a status of the library with the call's name."""
    h, null, a = U._host(), 0, ctypes.addressof
    x, off, codes = torch.zeros(2, 32, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64), torch.zeros(1, 2048, dtype=torch.uint8)
    d, e = desc(2, 32), desc(4, 32)
    for bad, error in ((x, ValueError), (3, TypeError)):
        with pytest.raises(error):
            h.mxfp4_quantize_dual(bad, False, False, 0, 0, 0, 0, 0, 0, a(d), False, a(e), False, null)
        with pytest.raises(error):
            h.mxfp4_quantize_grouped(bad, off, 32, True, False, 0, 0, 0, 0, a(d), False, null)

    def y(offsets, out=None, code=BF16, rows=7):
        return h.mxfp4_gemm_fwd_y_grouped(codes, a(d), a(e), offsets, rows, code, out, null)

    def dx(offsets, out=None, code=BF16):
        return h.mxfp4_gemm_bwd_dx_grouped(codes, a(d), a(e), offsets, 7, code, out, null)

    def dw(offsets, out=None, code=BF16):
        return h.mxfp4_gemm_bwd_dw_grouped(codes, a(d), a(e), offsets, code, out, null)

    for call, shape in ((y, (7, 2)), (dx, (7, 4)), (dw, (2, 2, 4))):
        for offsets in (off.int(), off[None], off[:1], torch.zeros(6, dtype=torch.int64)[::2]):
            with pytest.raises(ValueError, match="offsets"):
                call(offsets)
        with pytest.raises(TypeError, match="offsets"):
            call(None)
        with pytest.raises(ValueError, match="out_dtype"):
            call(off, code=-1)
        wrong = torch.zeros(*shape[:-1], shape[-1] + 1)
        for out in (wrong, wrong[..., 0], torch.zeros(shape, dtype=torch.float64), torch.zeros(*shape[:-1], 2 * shape[-1])[..., ::2]):
            with pytest.raises(ValueError, match="out"):
                call(off, out)
        with pytest.raises(TypeError, match="arguments"):
            getattr(h, "mxfp4_gemm_bwd_dw_grouped")(codes, a(d))
    with pytest.raises(ValueError, match="apart"):
        dw(off, torch.zeros(2, 3, 4)[:, :2])
    with pytest.raises(U.UFP4Error, match="ufp4_mxfp4_gemm_bwd_dw_grouped"):  # plain operands
        dw(off)
    with pytest.raises(RuntimeError):
        y(off, rows=-1)


STAND_IN = """
int PyGILState_Check(void);
static int calls, held;
static int called(void) { ++calls; held += PyGILState_Check(); return 0; }
int call_count(void) { return calls; }
int held_count(void) { return held; }
"""
STAND_IN_RUN = """
import ctypes, sys
import torch
sys.path.insert(0, sys.argv[2])
s = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)  # found before the library
from paper_2606_20381_amd import _host as h, ufp4 as U
codes, off = torch.zeros(1, 2048, dtype=torch.uint8), torch.zeros(3, dtype=torch.int64)
d = U.QDesc(codes=1 << 20, scales=1 << 20, code_panel_ld=2048, scale_panel_ld=512, panels=1, rows=2, red=32, format=U.E2M1_MX32)
a = ctypes.addressof(d)
for out in (None, torch.zeros(2, 2)):
    for f in (h.mxfp4_gemm_fwd_y, h.mxfp4_gemm_bwd_dx, h.mxfp4_gemm_bwd_dw):
        assert f(codes, a, a, U.OUT_F32, out, 0).shape == (2, 2)
h.mxfp4_dequantize(codes, a, None, 0)
h.mxfp4_gemm_fwd_y_grouped(codes, a, a, off, 7, U.OUT_BF16, None, 0)
h.mxfp4_gemm_bwd_dx_grouped(codes, a, a, off, 7, U.OUT_BF16, None, 0)
h.mxfp4_gemm_bwd_dw_grouped(codes, a, a, off, U.OUT_F32, None, 0)
print("calls", s.call_count(), "held", s.held_count())
"""


def test_host_module_calls_the_library_without_the_interpreter_lock(lib, tmp_path):
    """A launch can wait (a full queue, work that another Python thread has still to issue), so other threads run meanwhile. The library's
    functions are replaced by ones that note whether the caller holds the lock."""
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    names = ["ufp4_mxfp4_dequantize"] + [f"ufp4_mxfp4_gemm_{p}{g}" for p in ("fwd_y", "bwd_dx", "bwd_dw") for g in ("", "_grouped")]
    src, so = tmp_path / "standin.c", tmp_path / "standin.so"
    src.write_text(STAND_IN + "".join(f"int {n}() {{ return called(); }}\n" for n in names))
    subprocess.run([cc, "-shared", "-fPIC", "-o", str(so), str(src)], check=True)
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", STAND_IN_RUN, str(so), root], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split() == ["calls", "10", "held", "0"]


def test_operands_off_the_gpu_are_refused(lib):
    """A descriptor holds addresses only: operands in host memory are refused before a kernel could read them."""
    q, x = U.empty_qtensor(32, 32, U.E2M1_MX32, device="cpu"), torch.zeros(32, 32, dtype=torch.bfloat16)
    off = torch.zeros(2, dtype=torch.int64)
    calls = [lambda f=f: f(q, q) for f in (U.mxfp4_gemm_fwd_y, U.mxfp4_gemm_bwd_dx, U.mxfp4_gemm_bwd_dw)]
    calls += [lambda f=f: f(q, q, off, 32) for f in (U.mxfp4_gemm_fwd_y_grouped, U.mxfp4_gemm_bwd_dx_grouped)]
    calls += [lambda: U.mxfp4_gemm_bwd_dw_grouped(q, q, off), lambda: U.mxfp4_dequantize(q), lambda: U.mxfp4_linear(x, q),
              lambda: U.mxfp4_quantize(x, out=q), lambda: U.mxfp4_quantize_dual(x, out_rows=q), lambda: U.mxfp4_quantize_dual(x, out_cols=q),
              lambda: U.mxfp4_quantize_grouped(x, off, 32, transpose=True, out=q)]
    for call in calls:
        with pytest.raises(ValueError, match="CUDA device"):
            call()
    for call in (lambda: U.mxfp4_linear(3, q), lambda: U.mxfp4_quantize(3, out=q)):
        with pytest.raises(TypeError, match="tensor"):
            call()


# ------------------------------------------------------------------------------------------------
# the build
# ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("torch_is", ["there", "missing", "of another kind"])
def test_the_library_is_built_without_the_host_module(monkeypatch, tmp_path, torch_is):
    """The C interface needs no torch: a missing one, or headers that the host module does not compile with, leave a library."""
    from paper_2606_20381_amd import build as B

    for name, path in (("LIB", "lib.so"), ("HOST", "host.so"), ("BUILD", "objects")):
        monkeypatch.setattr(B, name, str(tmp_path / path))
    find = B.importlib.util.find_spec
    if torch_is == "missing":
        monkeypatch.setattr(B.importlib.util, "find_spec", lambda name: None if name == "torch" else find(name))

    def run(cmd, verbose):
        if torch_is == "of another kind" and any(a.endswith("ufp4_host.cpp") for a in cmd):
            raise RuntimeError("host module")
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(B, "_run", run)
    if torch_is == "of another kind":
        with pytest.raises(RuntimeError, match="host module"):
            B.build()
    else:
        assert B.build() == B.LIB
    assert os.path.exists(B.LIB) and os.path.exists(B.HOST) == (torch_is == "there")
