"""CPU checks of the grouped bf16 products, the 8-bit checkpoints and the activation: what the host refuses before anything is launched,
calls that have nothing to do, and sizes that it computes."""

import ctypes
import os

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

OK, INVALID, SHAPE, ALIGN, UNSUPPORTED = 0, 1, 2, 3, 5
F32, BF16 = U.OUT_F32, U.OUT_BF16
FAKE = 1 << 20  # never dereferenced: every call below fails validation or has nothing to do
R = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(U.library_path()):
        pytest.skip("libufp4.so not built")
    return U.lib()


@pytest.mark.parametrize("name", ["fwd_y", "bwd_dx", "bwd_dw"])
def test_product_refusals(lib, name):
    f = getattr(lib, f"ufp4_bf16_gemm_{name}_grouped")

    def call(a=FAKE, tokens=4, ka=8, lda=8, b=FAKE, nb=16, ldb=16, off=FAKE, G=2, c=FAKE, ldc=16, dt=F32, ws=FAKE, n=1 << 20):
        # fwd_y: x [4, 8], w [2 * 16, 8]; bwd_dx: dy [4, 8], w [2 * 8, 16]; bwd_dw: dy [4, 8], x [4, 16]
        return f(a, tokens, ka, lda, b, nb, ldb, off, G, c, ldc, dt, ws, n, None)

    if name == "bwd_dw":
        assert call(tokens=0, a=None, b=None, c=None) == INVALID  # dw of no tokens is zero: it needs dw
    else:
        assert call(tokens=0, a=None, c=None) == OK
    assert call(nb=0, b=None, c=None, ldb=0, ldc=0) == OK
    for k in ("a", "b", "c", "off"):
        assert call(**{k: None}) == INVALID, k
    for k in ("tokens", "ka", "nb"):
        assert call(**{k: -1}) == INVALID, k
    assert call(G=0) == INVALID and call(G=-1) == INVALID and call(dt=2) == INVALID and call(dt=-1) == INVALID
    assert call(lda=7) == SHAPE and call(ldb=7) == SHAPE and call(ldc=7) == SHAPE
    assert call(a=FAKE + 1) == ALIGN and call(b=FAKE + 1) == ALIGN and call(c=FAKE + 2) == ALIGN and call(off=FAKE + 4) == ALIGN
    assert call(dt=BF16, c=FAKE + 1) == ALIGN
    big = 1 << 31
    assert call(G=1025) == UNSUPPORTED and call(tokens=big) == UNSUPPORTED
    assert call(ka=(1 << 30) + 1, lda=big, ldb=big, ldc=big) == UNSUPPORTED
    assert call(nb=(1 << 30) + 1, lda=big, ldb=big, ldc=big) == UNSUPPORTED
    assert call(lda=1 << 41) == UNSUPPORTED and call(ldb=1 << 41) == UNSUPPORTED and call(ldc=1 << 41) == UNSUPPORTED
    # a product of many tiles needs its workspace
    many = dict(tokens=100_000, ka=4096, nb=4096, lda=4096, ldb=4096, ldc=4096)
    assert call(**many, ws=None) == INVALID and call(**many, n=511) == SHAPE and call(**many, ws=FAKE + 2) == ALIGN
    # tiles: outputs of 2^31 x 2^30
    assert call(tokens=big - 1, nb=1 << 30, ka=1 << 30, lda=big, ldb=big, ldc=big) == UNSUPPORTED


def test_product_workspace(lib):
    b, f = ctypes.c_size_t(7), lib.ufp4_bf16_gemm_grouped_workspace
    for p in range(3):
        assert f(p, 0, 0, 0, 1, R(b)) == OK and b.value == 0
        assert f(p, 4, 128, 128, 2, R(b)) == OK and b.value == 0
        assert f(p, 100_000, 4096, 4096, 64, R(b)) == OK and b.value == 512
        for bad in ((-1, 8, 8, 1), (8, -1, 8, 1), (8, 8, -1, 1), (8, 8, 8, 0)):
            assert f(p, *bad, R(b)) == INVALID
        assert f(p, 8, 8, 8, 1, None) == INVALID
        for big in ((1 << 31, 8, 8, 1), (8, (1 << 30) + 1, 8, 1), (8, 8, (1 << 30) + 1, 1), (8, 8, 8, 1025), ((1 << 31) - 1, 1 << 30, 1 << 30, 1)):
            assert f(p, *big, R(b)) == UNSUPPORTED
    assert f(3, 8, 8, 8, 1, R(b)) == INVALID and f(-1, 8, 8, 8, 1, R(b)) == INVALID


def test_product_from_a_checkpoint_refusals(lib):
    def call(dy=FAKE, tokens=4, N=8, lddy=8, codes=FAKE, cld=64, scales=FAKE, sld=2, K=40, off=FAKE, G=2, dw=FAKE, ldc=40, dt=F32, ws=FAKE, n=1 << 20):
        return lib.ufp4_bf16_gemm_bwd_dw_grouped_ckpt8(dy, tokens, N, lddy, codes, cld, scales, sld, K, off, G, dw, ldc, dt, ws, n, None)

    assert call(N=0, dy=None, dw=None) == OK and call(K=0, codes=None, scales=None, dw=None) == OK
    for k in ("dy", "codes", "scales", "off", "dw"):
        assert call(**{k: None}) == INVALID, k
    assert call(tokens=-1) == INVALID and call(G=0) == INVALID and call(dt=9) == INVALID
    assert call(cld=48) == SHAPE and call(sld=1) == SHAPE and call(lddy=7) == SHAPE and call(ldc=39) == SHAPE
    assert call(codes=FAKE + 8) == ALIGN and call(cld=72) == ALIGN and call(dy=FAKE + 1) == ALIGN and call(off=FAKE + 4) == ALIGN
    assert call(G=1025) == UNSUPPORTED and call(tokens=1 << 31) == UNSUPPORTED


def test_checkpoint_sizes(lib):
    c, s = ctypes.c_int64(), ctypes.c_int64()
    for cols, parts, code_ld, scale_ld in ((0, 1, 0, 0), (1, 1, 32, 4), (32, 1, 32, 4), (33, 1, 64, 4), (129, 1, 160, 8), (1411, 2, 2880, 92),
                                            (64, 2, 128, 4)):
        assert lib.ufp4_ckpt8_ld(cols, parts, R(c), R(s)) == OK and (c.value, s.value) == (code_ld, scale_ld)
    assert lib.ufp4_ckpt8_ld(8, 1, None, None) == OK
    assert lib.ufp4_ckpt8_ld(-1, 1, R(c), R(s)) == INVALID and lib.ufp4_ckpt8_ld(8, 0, R(c), R(s)) == INVALID
    assert lib.ufp4_ckpt8_ld(8, 3, R(c), R(s)) == INVALID and lib.ufp4_ckpt8_ld((1 << 30) + 1, 1, R(c), R(s)) == UNSUPPORTED


@pytest.mark.parametrize("save", [True, False])
def test_checkpoint_refusals(lib, save):
    def call(dt=BF16, x=FAKE, rows=4, cols=40, ldx=40, codes=FAKE, cld=64, scales=FAKE, sld=2):
        if save:
            return lib.ufp4_ckpt8_save(dt, x, rows, cols, ldx, codes, cld, scales, sld, None)
        return lib.ufp4_ckpt8_load(dt, codes, cld, scales, sld, rows, cols, x, ldx, None)

    assert call(rows=0, x=None, codes=None, scales=None) == OK and call(cols=0, x=None, codes=None, scales=None) == OK
    for k in ("x", "codes", "scales"):
        assert call(**{k: None}) == INVALID, k
    assert call(dt=2) == INVALID and call(rows=-1) == INVALID and call(cols=-1) == INVALID
    assert call(ldx=39) == SHAPE and call(cld=48) == SHAPE and call(sld=1) == SHAPE
    assert call(x=FAKE + 1) == ALIGN and call(dt=F32, x=FAKE + 2) == ALIGN and call(codes=FAKE + 8) == ALIGN and call(cld=72) == ALIGN
    big = 1 << 40
    assert call(cols=(1 << 30) + 1, ldx=big, cld=big, sld=big) == UNSUPPORTED
    assert call(rows=1 << 37, cols=1) == UNSUPPORTED and call(rows=1 << 32, cols=1024, ldx=big, cld=big, sld=big) == UNSUPPORTED
    assert call(ldx=big + 1) == UNSUPPORTED


@pytest.mark.parametrize("kind,parts", [(0, 1), (1, 2)])
def test_activation_refusals(lib, kind, parts):
    def fwd(kind=kind, dt=BF16, u=FAKE, rows=4, cols=40, ldu=80, a=FAKE, lda=40, codes=FAKE, cld=128, scales=FAKE, sld=4):
        return lib.ufp4_activation(kind, dt, u, rows, cols, ldu, a, lda, codes, cld, scales, sld, None)

    def bwd(kind=kind, dt=BF16, da=FAKE, rows=4, cols=40, ldda=40, u=None, ldu=80, codes=FAKE, cld=128, scales=FAKE, sld=4, du=FAKE, lddu=80,
            a=FAKE, lda=40):
        return lib.ufp4_activation_bwd(kind, dt, da, rows, cols, ldda, u, ldu, codes, cld, scales, sld, du, lddu, a, lda, None)

    for call in (fwd, bwd):
        none = dict(codes=None, scales=None, a=None)
        assert call(rows=0, **none) == OK and call(cols=0, **none) == OK
        assert call(kind=2) == INVALID and call(kind=-1) == INVALID and call(dt=5) == INVALID
        assert call(rows=-1) == INVALID and call(cols=-1) == INVALID
        assert call(scales=None) == INVALID and call(codes=FAKE + 8) == ALIGN and call(cld=136) == ALIGN
        assert call(cld=parts * 64 - 16) == SHAPE and call(sld=parts * 2 - 1) == SHAPE
        assert call(lda=39) == SHAPE and call(a=FAKE + 1) == ALIGN and call(cols=(1 << 30) + 1) == UNSUPPORTED
    assert fwd(u=None) == INVALID and fwd(a=None) == INVALID and fwd(codes=None) == INVALID and fwd(ldu=parts * 40 - 1) == SHAPE
    assert fwd(u=FAKE + 1) == ALIGN and fwd(dt=F32, u=FAKE + 2) == ALIGN
    assert bwd(da=None) == INVALID and bwd(du=None) == INVALID and bwd(codes=None) == INVALID
    assert bwd(u=FAKE) == INVALID  # u and its checkpoint
    assert bwd(u=FAKE, codes=None, ldu=parts * 40 - 1) == SHAPE and bwd(u=FAKE + 1, codes=None) == ALIGN
    assert bwd(ldda=39) == SHAPE and bwd(lddu=parts * 40 - 1) == SHAPE and bwd(da=FAKE + 1) == ALIGN and bwd(du=FAKE + 1) == ALIGN


def test_binding_refuses_what_is_not_on_a_gpu(lib, monkeypatch):
    monkeypatch.setattr(U, "_stream", lambda: 0)
    x, w, off = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(32, 8, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    kept = U.Checkpoint8(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8), 8)
    for call in (lambda: U.bf16_gemm_fwd_y_grouped(x, w, off), lambda: U.bf16_gemm_bwd_dx_grouped(x, w, off),
                 lambda: U.bf16_gemm_bwd_dw_grouped(x, x, off), lambda: U.bf16_gemm_bwd_dw_grouped(x, kept, off),
                 lambda: U.checkpoint8_save(x), lambda: U.checkpoint8_load(kept), lambda: U.activation(x),
                 lambda: U.activation_bwd(x, x), lambda: U.activation_bwd(x, kept)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_binding_refuses_other_arguments(lib, monkeypatch):
    monkeypatch.setattr(U, "_stream", lambda: 0)
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    for call in (lambda: U.activation(x, "gelu"), lambda: U.activation_bwd(x, x, "relu"),
                 lambda: U.activation_bwd(x, U.Checkpoint8(codes, scales, 16, 2), "relu2"),
                 lambda: U.activation_bwd(x, U.Checkpoint8(codes, scales, 8), "swiglu"),
                 lambda: U.activation_bwd(x, U.Checkpoint8(codes, scales, 9), "relu2"),
                 lambda: U.bf16_gemm_bwd_dw_grouped(x, U.Checkpoint8(codes, scales, 16, 2), x),
                 lambda: U.checkpoint8_save(x, out=U.Checkpoint8(codes, scales, 16, 2)),
                 lambda: U.checkpoint8_save(x, out=U.Checkpoint8(codes, scales, 9))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: U.checkpoint8_save(3), lambda: U.activation_bwd(3, x), lambda: U.bf16_gemm_fwd_y_grouped(None, x, x)):
        with pytest.raises((TypeError, AttributeError)):
            call()


# (pass, rows, N, K, groups, us of the kernels 0 few rows, 2 tiles of 128, 3 tiles of 256 on an MI355X; None: not measured)
FWD, DX, DW = range(3)
MEASURED = [
    (FWD, 42, 1408, 2048, 64, (21.0, 35.3, None)), (FWD, 384, 1408, 2048, 64, (82.5, 99.0, None)), (FWD, 1536, 1408, 2048, 64, (143.6, 113.9, None)),
    (FWD, 2, 1312, 512, 8, (5.5, 8.3, None)), (FWD, 512, 1312, 512, 8, (17.6, 8.7, None)), (FWD, 2, 4096, 5120, 8, (15.8, 48.3, None)),
    (FWD, 256, 4096, 5120, 8, (148.4, 81.2, None)), (FWD, 1, 8192, 2048, 1, (7.6, 20.6, None)), (FWD, 64, 8192, 2048, 1, (15.3, 22.3, None)),
    (FWD, 256, 8192, 2048, 1, (52.5, 23.4, None)),
    (FWD, 2048, 2048, 2048, 1, (None, 24.7, 42.8)), (FWD, 4096, 4096, 1024, 1, (None, 39.1, 36.3)), (DX, 4096, 4096, 1024, 1, (None, 37.2, 76.1)),
    (DW, 4096, 4096, 1024, 1, (None, 39.2, 80.1)), (DX, 4096, 2048, 8192, 1, (None, 149.8, 116.1)), (DW, 4096, 2048, 8192, 1, (None, 130.3, 116.3)),
    (FWD, 2048, 8192, 2048, 1, (None, 68.2, 60.3)), (DX, 2048, 8192, 2048, 1, (None, 70.2, 141.2)), (DX, 4096, 4096, 2048, 8, (None, 104.8, 80.2)),
    (DW, 16384, 512, 1312, 16, (None, 62.0, 89.3)), (FWD, 24576, 1408, 2048, 64, (None, 201.7, 180.9)), (DX, 24576, 1408, 2048, 64, (None, 240.7, 174.6)),
    (DW, 24576, 1408, 2048, 64, (None, 313.0, 261.7)), (DW, 6144, 1408, 2048, 64, (None, 178.4, 156.3)), (FWD, 6144, 1408, 2048, 64, (None, 88.8, 106.2)),
    (FWD, 98304, 1408, 2048, 64, (None, 810.2, 556.0)), (DX, 98304, 1408, 2048, 64, (None, 819.7, 557.0)), (DW, 98304, 1408, 2048, 64, (None, 761.5, 623.0)),
]


@pytest.mark.parametrize("p,rows,N,K,G,us", MEASURED)
def test_rule_takes_a_fast_kernel(lib, p, rows, N, K, G, us):
    """The kernel that the rule picks is within 25% of the best measured one."""
    pick = lib.ufp4_plan_gemm_bf16(p, ctypes.c_int64(rows), ctypes.c_int64(N), ctypes.c_int64(K), G, 1)
    took = {0: us[0], 2: us[1], 3: us[2]}[pick]
    assert took is not None and took <= 1.25 * min(v for v in us if v is not None)


def test_rule_on_other_alignment_and_passes(lib):
    plan = lambda p, rows, N, K, G, whole: lib.ufp4_plan_gemm_bf16(p, *(ctypes.c_int64(v) for v in (rows, N, K)), G, whole)  # noqa: E731
    assert plan(FWD, 98304, 1408, 2048, 64, 0) == 1 and plan(FWD, 64, 1408, 2048, 1, 0) == 0  # the few-row kernel takes any alignment
    assert plan(DX, 1, 1408, 2048, 1, 1) == 2 and plan(DW, 1, 1408, 2048, 1, 1) == 2
    assert plan(FWD, 0, 0, 0, 1, 1) == 0 and plan(DW, 0, 0, 0, 1, 1) in (2, 3)
