"""Products of microscaled 4-bit operands against 64-bit products of the same operands' values.

Tolerance. The matrix instruction adds 64 (or 128) exact products to an fp32 sum; counting one truncation (2^-23 of the sum of
magnitudes) for each instruction and 64 for what an instruction may lose inside, an output is off by at most
(K / 64 + 64 + splits) 2^-23 sum |a b|. bf16 outputs add 2^-8 of their value.
"""

import ctypes

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _operand(rows, red, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, red, generator=g, device="cuda") * scale
    x = x * torch.exp2(torch.randint(-6, 7, (rows, 1), generator=g, device="cuda").float())
    return U.mxfp4_quantize(x.to(BF))


def _values(q):
    return U.mxfp4_dequantize(q).double()


def _within(got, a, b, red, dt):
    ref, size = a @ b.t(), a.abs() @ b.abs().t()
    bound = (red / 64 + 64 + 16) * 2.0**-23 * size + (2.0**-8 * ref.abs() if dt == BF else 0)
    err = (got.double() - ref).abs()
    assert bool((err <= bound).all()), f"{int((~(err <= bound)).sum())} off, worst {float((err - bound).max()):.3e}"


DENSE = [(1, 1, 32), (5, 7, 64), (64, 64, 96), (65, 63, 128), (128, 128, 160), (200, 130, 512), (129, 385, 1056), (256, 256, 2048),
         (300, 3, 4096), (2048, 2048, 256), (4096, 4128, 224), (3900, 4000, 96), (1, 5000, 32), (16, 300, 16384)]


@pytest.mark.parametrize("M,N,K", DENSE)
@pytest.mark.parametrize("dt", [BF, F32])
def test_dense(M, N, K, dt):
    a, b = _operand(M, K, M + K), _operand(N, K, N + 2 * K)
    out = torch.full((M, N + 3), -7.0, dtype=dt, device="cuda")
    va, vb = _values(a), _values(b)
    for fn in (U.mxfp4_gemm_fwd_y, U.mxfp4_gemm_bwd_dx, U.mxfp4_gemm_bwd_dw):
        out.fill_(-7.0)
        got = fn(a, b, out=out[:, :N])
        _within(got, va, vb, K, dt)
        assert (out[:, N:] == -7).all()
    assert torch.equal(got, U.mxfp4_gemm_bwd_dw(a, b, dt))  # repeats


@pytest.mark.parametrize("M,N,K", [(70, 90, 192), (2100, 2100, 320), (4200, 4100, 160), (8192, 8192, 1056), (9000, 8200, 1248),
                                   (16384, 8192, 1024)])
def test_exact_where_sums_are_small_integers(M, N, K):
    """Values in 0, +-1, +-2, +-3 at scale 1: every partial sum is a small integer, so the result is exact, and a wrong lane,
    block, scale or edge shows as a wrong integer."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randint(-3, 4, (M, K), generator=g, device="cuda").to(BF)
    w = torch.randint(-3, 4, (N, K), generator=g, device="cuda").to(BF)
    x[:, ::32], w[:, ::32] = 4, 4  # the block's top: scale 1
    got = U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x), U.mxfp4_quantize(w))
    assert torch.equal(got.double(), x.double() @ w.double().t())
    bf = U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x), U.mxfp4_quantize(w), BF)
    assert torch.equal(bf, got.to(BF))


def _plan(M, N, K, mode=0, G=1, a_rows=None):
    fn = ctypes.CDLL(U.library_path()).ufp4_plan_gemm_mxfp4
    fn.argtypes = [ctypes.c_int, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int64]
    return fn(mode, M, N, K, G, M if a_rows is None else a_rows)


@pytest.mark.parametrize("kernel,M,N,K", [(0, 4096, 4096, 4096), (0, 4090, 4000, 2080), (1, 2048, 2048, 2048), (1, 2040, 1990, 2080),
                                          (2, 256, 8192, 2048), (2, 250, 8130, 1952), (3, 64, 2048, 8192), (3, 70, 1000, 8224),
                                          (3, 130, 66, 5000 * 32)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_every_kernel(kernel, M, N, K, dt):
    """Each of the kernels at a size that its rule gives it, with whole and with partial tiles and stages."""
    assert _plan(M, N, K) == kernel
    a, b = _operand(M, K, M + K), _operand(N, K, N + 2 * K)
    _within(U.mxfp4_gemm_fwd_y(a, b, dt), _values(a), _values(b), K, dt)


@pytest.mark.parametrize("kernel,counts,N,K", [(0, [6000, 3, 0, 6000, 129], 1024, 1056), (1, [2000, 0, 1300, 7], 1024, 2048),
                                               (2, [100, 5, 0, 77], 1280, 256), (3, [30, 0, 64, 1], 128, 4096)])
def test_every_grouped_kernel(kernel, counts, N, K):
    G, total = len(counts), sum(counts)
    off, p128 = U.group_offsets(counts, block=128)
    _, p32 = U.group_offsets(counts, block=32)
    assert _plan(total, N, K, 1, G, p128) == kernel
    g = torch.Generator(device="cuda").manual_seed(total)
    x, dy = (torch.randn(total, n, generator=g, device="cuda").to(BF) for n in (K, N))
    w = torch.randn(G * N, K, generator=g, device="cuda").to(BF)
    wq = U.mxfp4_quantize(w)
    y = U.mxfp4_gemm_fwd_y_grouped(U.mxfp4_quantize_grouped(x, off, p128, transpose=False), wq, off, total, BF)
    xtq = U.mxfp4_quantize_grouped(x, off, p32, transpose=True)
    dytq = U.mxfp4_quantize_grouped(dy, off, p32, transpose=True)
    dw = U.mxfp4_gemm_bwd_dw_grouped(dytq, xtq, off)
    vx, vw, vxt, vdyt = _values(U.mxfp4_quantize(x)), _values(wq), _values(xtq), _values(dytq)
    pads = U.padded_offsets([0] + torch.tensor(counts).cumsum(0).tolist(), 32)
    for e, s in enumerate(_groups(counts, total)):
        _within(y[s], vx[s], vw[e * N : (e + 1) * N], K, BF)
        r = slice(pads[e], pads[e + 1])
        _within(dw[e], vdyt[:, r], vxt[:, r], pads[e + 1] - pads[e], F32)


def test_scales_of_every_block_count():
    """Blocks with very different scales, all tails of the groups of four."""
    for nkb in range(1, 14):
        g = torch.Generator(device="cuda").manual_seed(nkb)
        x = torch.randn(96, nkb, 32, generator=g, device="cuda")
        x = x * torch.exp2(torch.randint(-20, 20, (96, nkb, 1), generator=g, device="cuda").float())
        a = U.mxfp4_quantize(x.view(96, -1).to(BF))
        _within(U.mxfp4_gemm_fwd_y(a, a), _values(a), _values(a), nkb * 32, F32)


def test_nan_scale_reaches_its_rows():
    x = torch.randn(70, 64, device="cuda").to(BF)
    w = torch.randn(40, 64, device="cuda").to(BF)
    x[3, 5] = float("inf")
    y = U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x), U.mxfp4_quantize(w))
    assert torch.isnan(y[3]).all() and torch.isfinite(y[torch.arange(70) != 3]).all()
    y = U.mxfp4_linear(x[2:5].contiguous(), U.mxfp4_quantize(w))
    assert torch.isnan(y[1]).all() and torch.isfinite(y[::2]).all()


def test_rotation_cancels():
    """Both operands rotated: the product of the unrotated tensors, up to the quantization error of 4 bits."""
    g = torch.Generator(device="cuda").manual_seed(0)
    x, w = (torch.randn(256, 1024, generator=g, device="cuda").to(BF) for _ in range(2))
    ref = x.double() @ w.double().t()
    for m in (0, 0x6A09):
        y = U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x, rht=True, sign_mask=m), U.mxfp4_quantize(w, rht=True, sign_mask=m))
        # each operand's relative error is at most about 0.15 for normal values (largest step 2 against amax in 4..8)
        assert float((y.double() - ref).norm() / ref.norm()) < 0.3
        z = U.mxfp4_linear(x[:3], U.mxfp4_quantize(w, rht=True, sign_mask=m), torch.float32)
        q = U.mxfp4_quantize(x[:3].contiguous(), rht=True, sign_mask=m)
        assert torch.equal(z, U.mxfp4_gemm_fwd_y(q, U.mxfp4_quantize(w, rht=True, sign_mask=m)))


def _groups(counts, rows):
    at = 0
    for c in counts:
        yield slice(at, at + c)
        at += c


COUNTS = [[100], [0, 1, 64, 0, 128, 129, 3, 255, 256, 0], [1] * 67, [700, 0, 31]]


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("N,K", [(128, 32), (256, 160), (384, 544)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_grouped(counts, N, K, dt):
    G, total = len(counts), sum(counts)
    g = torch.Generator(device="cuda").manual_seed(total + N)
    x = torch.randn(total, K, generator=g, device="cuda").to(BF)
    dy = torch.randn(total, N, generator=g, device="cuda").to(BF)
    w = torch.randn(G * N, K, generator=g, device="cuda").to(BF)
    off, p128 = U.group_offsets(counts, block=128)
    _, p32 = U.group_offsets(counts, block=32)
    wq, wtq = U.mxfp4_quantize(w), U.mxfp4_quantize(w, transpose=True)
    xq = U.mxfp4_quantize_grouped(x, off, p128, transpose=False)
    dyq = U.mxfp4_quantize_grouped(dy, off, p128, transpose=False)
    xtq = U.mxfp4_quantize_grouped(x, off, p32, transpose=True)
    dytq = U.mxfp4_quantize_grouped(dy, off, p32, transpose=True)
    y = U.mxfp4_gemm_fwd_y_grouped(xq, wq, off, total, dt)
    dx = U.mxfp4_gemm_bwd_dx_grouped(dyq, wtq, off, total, dt)
    dw = U.mxfp4_gemm_bwd_dw_grouped(dytq, xtq, off, dt)
    vw, vwt, vdyt, vxt = _values(wq), _values(wtq), _values(dytq), _values(xtq)
    pads = U.padded_offsets([0] + torch.tensor(counts).cumsum(0).tolist(), 32)
    vx, vdy = _values(U.mxfp4_quantize(x)), _values(U.mxfp4_quantize(dy))
    for e, s in enumerate(_groups(counts, total)):
        _within(y[s], vx[s], vw[e * N : (e + 1) * N], K, dt)
        _within(dx[s], vdy[s], vwt[:, e * N : (e + 1) * N], N, dt)
        r = slice(pads[e], pads[e + 1])
        _within(dw[e], vdyt[:, r], vxt[:, r], pads[e + 1] - pads[e], dt)
        if counts[e] == 0:
            assert not dw[e].any()


def test_grouped_neighbours_with_extreme_scales():
    """A group's products take nothing from the blocks of its neighbours in the same four, whatever their scales."""
    counts = [32, 64, 32, 96]
    x = torch.randn(224, 64, device="cuda").to(BF)
    dy = torch.randn(224, 128, device="cuda").to(BF)
    x[32:96] *= 2.0**100
    dy[32:96] *= 2.0**100
    x[128:] = float("inf")
    off, p32 = U.group_offsets(counts, block=32)
    a = U.mxfp4_quantize_grouped(dy, off, p32, transpose=True)
    b = U.mxfp4_quantize_grouped(x, off, p32, transpose=True)
    dw = U.mxfp4_gemm_bwd_dw_grouped(a, b, off)
    va, vb = _values(a), _values(b)
    _within(dw[0], va[:, :32], vb[:, :32], 32, F32)
    _within(dw[2], va[:, 96:128], vb[:, 96:128], 32, F32)
    assert torch.isinf(dw[1]).any() and torch.isnan(dw[3]).all()


@pytest.mark.parametrize("tokens", [1, 2, 3, 5, 8, 15, 16, 17, 40])
@pytest.mark.parametrize("N,K", [(1, 32), (16, 64), (100, 224), (256, 4096), (2048, 1056), (8300, 160), (520, 16384),
                                 (33000, 288), (16500, 1024), (300, 33024)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_linear(tokens, N, K, dt):
    g = torch.Generator(device="cuda").manual_seed(tokens + N)
    x = torch.randn(tokens, K + 8, generator=g, device="cuda").to(BF)[:, :K]
    wq = _operand(N, K, N + K)
    out = torch.full((tokens, N + 2), -7.0, dtype=dt, device="cuda")
    got = U.mxfp4_linear(x, wq, out=out[:, :N])
    _within(got, _values(U.mxfp4_quantize(x)), _values(wq), K, dt)
    assert (out[:, N:] == -7).all() and torch.equal(got, U.mxfp4_linear(x, wq, dt))


def test_empty():
    e = U.mxfp4_quantize(torch.empty(0, 64, dtype=BF, device="cuda"))
    w = _operand(8, 64, 1)
    assert U.mxfp4_gemm_fwd_y(e, w).shape == (0, 8) and U.mxfp4_gemm_fwd_y(w, e).shape == (8, 0)
    assert U.mxfp4_linear(torch.empty(0, 64, dtype=BF, device="cuda"), w).shape == (0, 8)
    z = U.mxfp4_quantize(torch.empty(5, 0, dtype=BF, device="cuda"))
    assert not U.mxfp4_gemm_fwd_y(z, z).any()  # an empty sum
    assert not U.mxfp4_linear(torch.empty(2, 0, dtype=BF, device="cuda"), z).any()


def test_other_stream_and_graph():
    x = torch.randn(5, 512, device="cuda").to(BF)
    big = torch.randn(600, 512, device="cuda").to(BF)
    wq = _operand(256, 512, 3)
    want, wantb = U.mxfp4_linear(x, wq), U.mxfp4_linear(big, wq)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, yb = torch.zeros_like(want), torch.zeros_like(wantb)
    xq = U.empty_qtensor(600, 512, U.E2M1_MX32)
    with torch.cuda.stream(s):
        U.mxfp4_linear(x, wq, out=y)
        U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(big, out=xq), wq, out=yb)
    s.synchronize()
    assert torch.equal(y, want) and torch.equal(yb, wantb)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        U.mxfp4_linear(x, wq, out=y)
        U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(big, out=xq), wq, out=yb)
    for i in range(3):
        x.mul_(2)
        big.neg_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, U.mxfp4_linear(x, wq)) and torch.equal(yb, U.mxfp4_linear(big, wq))


def test_refusals():
    a, b = _operand(8, 64, 1), _operand(8, 96, 2)
    x = torch.randn(4, 64, device="cuda").to(BF)
    with pytest.raises(U.UFP4Error):
        U.mxfp4_gemm_fwd_y(a, b)  # reduction lengths
    with pytest.raises(U.UFP4Error):
        U.mxfp4_gemm_fwd_y(a, U.mx_quantize(x, rht=False))  # formats
    with pytest.raises(U.UFP4Error):
        U.mx_gemm_fwd_y(a, a)
    with pytest.raises(U.UFP4Error):
        U.gemm_fwd_y(a, a)
    with pytest.raises(U.UFP4Error):
        U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x, rht=True), a)  # rotations
    with pytest.raises(U.UFP4Error):
        U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x, rht=True, sign_mask=1), U.mxfp4_quantize(x, rht=True, sign_mask=2))
    with pytest.raises(ValueError):
        U.mxfp4_linear(x, b)
    with pytest.raises(ValueError):
        U.mxfp4_linear(x.float(), a)
    off, p32 = U.group_offsets([2, 2], block=32)
    t = U.mxfp4_quantize_grouped(x, off, p32, transpose=True)
    with pytest.raises(U.UFP4Error):
        U.mxfp4_gemm_fwd_y_grouped(t, a, off, 4)  # forms
    with pytest.raises(U.UFP4Error):
        U.mxfp4_linear(x, t) if t.red == 64 else U.mxfp4_gemm_bwd_dw_grouped(a, a, off)
    # bwd_dx: a group's blocks of W^T must begin with a group of four scales
    dy = torch.randn(4, 96, device="cuda").to(BF)
    dyq = U.mxfp4_quantize_grouped(dy, off, 256, transpose=False)
    with pytest.raises(U.UFP4Error):
        U.mxfp4_gemm_bwd_dx_grouped(dyq, U.mxfp4_quantize(torch.randn(192, 64, device="cuda").to(BF), transpose=True), off, 4)


def _small(rows, cols, seed, by_rows):
    """Small integers whose blocks along the rows (by_rows) or the columns have the scale 1."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(-3, 4, (rows, cols), generator=g, device="cuda").to(BF)
    if by_rows:
        x[:, ::32] = 4
    else:
        x[::32] = 4
    return x


@pytest.mark.parametrize("kernel,counts,N,K", [(1, [9000, 0, 1, 5000, 2390], 8192, 128), (0, [12000, 3, 4600], 8192, 1056)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_large_grouped_outputs(kernel, counts, N, K, dt):
    """Outputs of 256 MiB and more are stored by kernels of their own: exact products again."""
    G, total = len(counts), sum(counts)
    assert total * N * 2 >= 1 << 28
    off, p128 = U.group_offsets(counts, block=128)
    assert _plan(total, N, K, 1, G, p128) == kernel
    x, w = _small(total, K, 1, True), _small(G * N, K, 2, True)
    y = U.mxfp4_gemm_fwd_y_grouped(U.mxfp4_quantize_grouped(x, off, p128, transpose=False), U.mxfp4_quantize(w), off, total, dt)
    for e, s in enumerate(_groups(counts, total)):
        assert torch.equal(y[s], (x[s].double() @ w[e * N : (e + 1) * N].double().t()).to(dt))


@pytest.mark.parametrize("kernel,counts,N,K", [(1, [96, 0, 1, 128, 70], 4096, 3400), (0, [3500, 3, 3000], 4200, 5400)])
def test_large_weight_gradients(kernel, counts, N, K):
    G, total = len(counts), sum(counts)
    assert G * N * K * 4 >= 1 << 28
    off, p32 = U.group_offsets(counts, block=32)
    assert _plan(N, K, p32, 2, G, N) == kernel
    starts = [0] + torch.tensor(counts).cumsum(0).tolist()
    x, dy = _small(total, K, 1, False), _small(total, N, 2, False)
    for a in starts[:-1]:  # each group's blocks begin with its first token
        if a < total:
            x[a : a + 1], dy[a : a + 1] = 4, 4
    for e, s in enumerate(_groups(counts, total)):
        x[s][::32], dy[s][::32] = 4, 4
    q = [U.mxfp4_quantize_grouped(t, off, p32, transpose=True) for t in (dy, x)]
    dw = U.mxfp4_gemm_bwd_dw_grouped(*q, off)
    for e, s in enumerate(_groups(counts, total)):
        assert torch.equal(dw[e].double(), dy[s].double().t().contiguous() @ x[s].double())


@pytest.mark.parametrize("claim", [2**20, 2**31 - 1, 2**33, 2**40])
def test_offsets_that_claim_too_much(claim):
    """Groups past the tokens that there are, in numbers whose sums pass 32 bits: the first group's results stand, and nothing
    past the output is written."""
    N, K, G = 256, 160, 130
    x, dy = torch.randn(100, K, device="cuda").to(BF), torch.randn(100, N, device="cuda").to(BF)
    wq = U.mxfp4_quantize(torch.randn(G * N, K, device="cuda").to(BF))
    off = torch.tensor([0] + [100 + g * claim for g in range(G)], device="cuda")
    xq = U.mxfp4_quantize_grouped(x, off, 256, transpose=False)
    out = torch.full((130, N), -7.0, dtype=F32, device="cuda")
    U.mxfp4_gemm_fwd_y_grouped(xq, wq, off, 100, F32, out=out[:100])
    _within(out[:100], _values(U.mxfp4_quantize(x)), _values(wq)[:N], K, F32)
    assert (out[100:] == -7).all()
    xtq, dytq = (U.mxfp4_quantize_grouped(t, off, 160, transpose=True) for t in (x, dy))
    dw = U.mxfp4_gemm_bwd_dw_grouped(dytq, xtq, off)
    _within(dw[0], _values(dytq)[:, :128], _values(xtq)[:, :128], 128, F32)
    assert not dw[2:].any()


@pytest.mark.parametrize("n,k,dt", [(4133, 4099, F32), (6001, 6007, BF), (4096, 4104, F32)])
def test_weight_gradients_stored_past_the_caches(n, k, dt):
    """A dense weights' gradient of 64 MiB and more is stored by a kernel of its own: the same numbers, bit for bit, as the forward
    product of these operands, and nothing beside the rows of a wider output."""
    g = torch.Generator(device="cuda").manual_seed(n)
    a, b = (U.mxfp4_quantize(torch.randn(r, 416, generator=g, device="cuda").to(BF)) for r in (n, k))
    want = U.mxfp4_gemm_fwd_y(a, b, dt)
    assert 64 << 20 <= want.numel() * want.element_size() < 256 << 20
    assert torch.equal(U.mxfp4_gemm_bwd_dw(a, b, dt), want)
    wide = torch.full((n, k + 8), 7.0, device="cuda", dtype=dt)
    U.mxfp4_gemm_bwd_dw(a, b, dt, out=wide[:, :k])
    assert torch.equal(wide[:, :k], want) and (wide[:, k:] == 7.0).all()


@pytest.mark.parametrize("tokens", [1, 4, 16, 17, 40])
def test_linear_refuses_a_grouped_weight(tokens):
    """W as a grouped call lays it out, rows or reduction padded: refused whatever the number of tokens."""
    x = torch.randn(tokens, 64, device="cuda").to(BF)
    off, p128 = U.group_offsets([100, 60], block=128)
    rows = U.mxfp4_quantize_grouped(torch.randn(160, 64, device="cuda").to(BF), off, p128, transpose=False)
    off, p32 = U.group_offsets([20, 12], block=32)
    red = U.mxfp4_quantize_grouped(torch.randn(32, 24, device="cuda").to(BF), off, p32, transpose=True)
    assert rows.red == red.red == 64
    for w in (rows, red):
        with pytest.raises(U.UFP4Error) as e:
            U.mxfp4_linear(x, w)
        assert e.value.status == 4


def test_operands_of_another_device_are_refused():
    """One operand on the GPU, the one beside it in host memory."""
    a, x, off = _operand(32, 32, 1), torch.randn(32, 32, device="cuda").to(BF), torch.tensor([0, 32], device="cuda")
    b = U.empty_qtensor(32, 32, U.E2M1_MX32, device="cpu")
    for p, q in ((a, b), (b, a)):
        for f in (U.mxfp4_gemm_fwd_y, U.mxfp4_gemm_bwd_dx, U.mxfp4_gemm_bwd_dw):
            with pytest.raises(ValueError):
                f(p, q)
        for f in (U.mxfp4_gemm_fwd_y_grouped, U.mxfp4_gemm_bwd_dx_grouped):
            with pytest.raises(ValueError):
                f(p, q, off, 32)
        with pytest.raises(ValueError):
            U.mxfp4_gemm_bwd_dw_grouped(p, q, off)
    for call in (lambda: U.mxfp4_linear(x, b), lambda: U.mxfp4_linear(x.cpu(), a), lambda: U.mxfp4_quantize(x, out=b),
                 lambda: U.mxfp4_quantize_dual(x, out_rows=b), lambda: U.mxfp4_quantize_dual(x, out_rows=a, out_cols=b),
                 lambda: U.mxfp4_quantize_grouped(x, off, 32, transpose=True, out=b), lambda: U.mxfp4_dequantize(b)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("counts,N,K", [([8100, 0, 12001, 12600], 256, 256), ([33, 20000, 0, 12000], 200, 136), ([70, 32000, 1], 64, 256)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_weight_gradients_by_four_teams(counts, N, K, dt):
    """Few tiles of long reductions: groups that begin and end inside four blocks, empty ones, and one shorter than the teams' first
    stages, in small integers, so that the fp32 sums are exact."""
    G, total = len(counts), sum(counts)
    off, p32 = U.group_offsets(counts, block=32)
    assert _plan(N, K, p32, 2, G, N) == 3
    x, dy = _small(total, K, 1, False), _small(total, N, 2, False)
    for s in _groups(counts, total):
        x[s][::32], dy[s][::32] = 4, 4
    q = [U.mxfp4_quantize_grouped(t, off, p32, transpose=True) for t in (dy, x)]
    dw = U.mxfp4_gemm_bwd_dw_grouped(*q, off, dt)
    for e, s in enumerate(_groups(counts, total)):
        assert torch.equal(dw[e], (dy[s].double().t().contiguous() @ x[s].double()).to(dt))


@pytest.mark.parametrize("counts,N,K", [([100, 0, 150, 50], 8192, 256), ([1, 130], 8192, 248)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_input_gradients_by_four_teams(counts, N, K, dt):
    """Few tokens and a long N: the grouped input gradient (N its reduction, K its columns)."""
    G, total = len(counts), sum(counts)
    off, p128 = U.group_offsets(counts, block=128)
    assert _plan(total, K, N, 1, G, p128) == 3
    dy, w = _small(total, N, 1, True), _small(G * N, K, 2, False)
    dx = U.mxfp4_gemm_bwd_dx_grouped(U.mxfp4_quantize_grouped(dy, off, p128, transpose=False), U.mxfp4_quantize(w, transpose=True), off,
                                     total, dt)
    for e, s in enumerate(_groups(counts, total)):
        assert torch.equal(dx[s], (dy[s].double() @ w[e * N : (e + 1) * N].double()).to(dt))


def test_large_outputs_of_the_64_row_tiles():
    """256 MiB and more of many small weight gradients: stored plainly, as the 64-row tiles store everything."""
    counts, N, K = [64] * 256, 192, 2048
    total, G = sum(counts), len(counts)
    off, p32 = U.group_offsets(counts, block=32)
    assert _plan(N, K, p32, 2, G, N) == 2 and G * N * K * 4 >= 1 << 28
    x, dy = _small(total, K, 1, False), _small(total, N, 2, False)
    dw = U.mxfp4_gemm_bwd_dw_grouped(*(U.mxfp4_quantize_grouped(t, off, p32, transpose=True) for t in (dy, x)), off)
    for e, s in enumerate(_groups(counts, total)):
        assert torch.equal(dw[e].double(), dy[s].double().t().contiguous() @ x[s].double())
