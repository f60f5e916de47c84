"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances. A row's sum is at most 32 additions in a thread and 10 levels of a tree, so its relative error is at most
42 * 2^-24 of the sum of magnitudes: |dmu| rstd <= 42 * 2^-24 (|mu| rstd + 1), the variance is off by about the same
share and rstd by half of it, and a handful of roundings follow: |dh| <= K (1 + |mu| rstd + |h|) with K = 64 * 2^-24. Rows
longer than the registers hold add up to cols / 8192 more terms per thread. An output adds its own rounding, 2^-24 or 2^-9
of its value (bf16: half an ulp of 8 bits).
"""

import ctypes

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5
K = 64 * 2.0**-24


def _k(cols):
    return K + 2.0**-24 * cols / 4096


def _unit(dt):
    return 2.0**-8 if dt == BF else 2.0**-23


def _tensor(rows, cols, dt, seed, pad=0, offset=0, mean=0.25, std=1.0):
    """A [rows, cols] view with rows `cols + pad` apart, `offset` elements into its storage."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((offset + max(1, rows * (cols + pad)),), float("nan"), device="cuda").to(dt)
    v = buf[offset:].as_strided((rows, cols), (cols + pad, 1))
    v.copy_((torch.randn(rows, cols, generator=g, device="cuda") * std + mean).to(dt))
    return v


def _weights(cols, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return ((1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt),
            (0.3 * torch.randn(cols, generator=g, device="cuda")).to(dt))


def _forward64(x, gamma, beta, eps=EPS):
    x = x.double()
    mean = x.mean(1)
    rstd = 1 / torch.sqrt((x - mean[:, None]).square().mean(1) + eps)
    h = (x - mean[:, None]) * rstd[:, None]
    y = h
    if gamma is not None:
        y = y * gamma.double()
    if beta is not None:
        y = y + beta.double()
    return y, mean, rstd, h


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 8), (9, 63), (4, 65), (33, 255), (7, 513), (6, 1030), (7, 1411), (4, 2048), (6, 2049),
          (3, 4096), (5, 5120), (9, 6145), (2, 8193), (3, 16384), (2, 20000), (2, 33000), (2, 65537), (700, 33), (2600, 100), (5000, 1000)]


def _within(name, got, ref, bound):
    err = (got.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{name}: {int(bad.sum())} values off, worst {float((err - bound).max()):.3e} over the bound"


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dt", [BF, F32])
def test_forward(rows, cols, dt):
    x = _tensor(rows, cols, dt, rows * 131 + cols)
    gamma, beta = _weights(cols, F32, cols)
    y, mean, rstd = U.layer_norm(x, gamma, beta, eps=EPS)
    ry, rm, rr, h = _forward64(x, gamma, beta)
    k = _k(cols)
    away = (1 + rm.abs() * rr)[:, None]
    _within("mean", mean, rm, k * (rm.abs() + 1 / rr) + 2.0**-23 * rm.abs())
    _within("rstd", rstd, rr, k * (1 + rm.abs() * rr) * rr)
    _within("y", y, ry, k * (away + h.abs()) * gamma.double().abs() + 2.0**-23 * beta.double().abs() + _unit(dt) * ry.abs())


@pytest.mark.parametrize("wdt", [BF, F32])
@pytest.mark.parametrize("which", ["gamma", "beta", "both", "none"])
def test_forward_weights(wdt, which):
    x = _tensor(5, 300, BF, 3)
    gamma, beta = _weights(300, wdt, 9)
    gamma = gamma if which in ("gamma", "both") else None
    beta = beta if which in ("beta", "both") else None
    y = U.layer_norm(x, gamma, beta, eps=EPS)[0]
    ry, rm, rr, h = _forward64(x, gamma, beta)
    _within("y", y, ry, 8 * _k(300) * (4 + h.abs()) + _unit(BF) * ry.abs())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("pad,offset", [(0, 1), (3, 0), (5, 3), (8, 8)])
def test_strides_and_alignment(dt, pad, offset):
    """Any leading dimension and element-aligned base; what lies between the rows is neither used nor written."""
    rows, cols = 11, 517
    x, dy = _tensor(rows, cols, dt, 5, pad, offset), _tensor(rows, cols, dt, 6, pad, offset, 0.0)
    gamma, beta = _weights(cols, F32, 7)
    out = _tensor(rows, cols, dt, 8, pad, offset)
    y, mean, rstd = U.layer_norm(x, gamma, beta, out=out)
    dense = U.layer_norm(x.contiguous(), gamma, beta)
    assert torch.equal(y, dense[0]) and torch.equal(mean, dense[1]) and torch.equal(rstd, dense[2])
    got = U.layer_norm_bwd(dy, x, gamma, mean, rstd, out=out)
    want = U.layer_norm_bwd(dy.contiguous(), x.contiguous(), gamma, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    store = out.as_strided((rows, cols + pad), (cols + pad, 1)) if pad else None
    if pad:
        assert torch.isnan(store[: rows - 1, cols:]).all()


def _backward64(dy, x, gamma, mean, rstd):
    dy, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    g = dy if gamma is None else dy * gamma.double()
    dx = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0), h, g


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dt", [BF, F32])
def test_backward(rows, cols, dt):
    x, dy = _tensor(rows, cols, dt, rows * 17 + cols), _tensor(rows, cols, dt, rows * 19 + cols, mean=0.1)
    gamma, _ = _weights(cols, F32, cols)
    _, mean, rstd = U.layer_norm(x, gamma, None)
    dx, dgamma, dbeta = U.layer_norm_bwd(dy, x, gamma, mean, rstd)
    rx, rg, rb, h, g = _backward64(dy, x, gamma, mean, rstd)
    k, r = _k(cols), rstd.double()[:, None]
    size = g.abs() + g.abs().mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True)
    # h itself: one subtraction and one product of rounded numbers, relative to |x| + |mu|
    h_off = 2.0**-22 * (x.double().abs() + mean.double().abs()[:, None]) * r
    h_part = h_off * (g * h).abs().mean(1, keepdim=True) + h.abs() * (g.abs() * h_off).mean(1, keepdim=True)
    _within("dx", dx, rx, r * (k * size + 2 * h_part) + _unit(dt) * rx.abs())
    # a column: at most rows / 4 terms in a thread, then 512 partial rows in 32 additions and 16 more
    kw = 2.0**-24 * (rows / 4 + 64)
    _within("dgamma", dgamma, rg, kw * (dy.double() * h).abs().sum(0) + 2 * (dy.double().abs() * h_off).sum(0))
    _within("dbeta", dbeta, rb, kw * dy.double().abs().sum(0))


@pytest.mark.parametrize("rows,cols", [(3, 5), (4, 64), (2, 300)])
def test_backward_against_differences(rows, cols):
    """The kernel's gradients against central differences (step 1e-5, 64 bits) of L = sum(y v)."""
    x, v = _tensor(rows, cols, F32, 1), _tensor(rows, cols, F32, 2, mean=0.0)
    gamma, beta = _weights(cols, F32, 3)
    _, mean, rstd = U.layer_norm(x, gamma, beta, eps=EPS)
    dx, dgamma, dbeta = U.layer_norm_bwd(v, x, gamma, mean, rstd)
    s = 1e-5

    def loss(x, gamma, beta):
        return float((_forward64(x, gamma, beta)[0] * v.double()).sum())

    x, gamma, beta = x.double(), gamma.double(), beta.double()
    for grad, arg in ((dx, 0), (dgamma, 1), (dbeta, 2)):
        base = [x, gamma, beta]
        scale = float(grad.abs().max()) + 1.0
        for i in range(0, grad.numel(), max(1, grad.numel() // 23)):
            lo, hi = [t.clone() for t in base], [t.clone() for t in base]
            lo[arg].view(-1)[i] -= s
            hi[arg].view(-1)[i] += s
            want = (loss(*hi) - loss(*lo)) / (2 * s)
            # fp32 kernel: 1e-5 of the gradient's size; differences: third derivatives times s^2, 64-bit noise / s
            assert abs(float(grad.view(-1)[i]) - want) <= 2e-5 * scale


def test_large_mean_keeps_its_variance():
    """mu = 2^12, sigma = 1: E[x^2] - mu^2 in fp32 would lose everything; two sums over the row do not."""
    x = _tensor(3, 2048, F32, 4, mean=4096.0)
    y, mean, rstd = U.layer_norm(x, None, None)
    _, rm, rr, h = _forward64(x, None, None)
    assert ((rstd.double() - rr).abs() <= K * 4097 * rr).all() and ((mean.double() - rm).abs() <= K * rm).all()


@pytest.mark.parametrize("cols", [40, 3000, 40000])
def test_constant_rows_and_special_values(cols):
    x = _tensor(6, cols, BF, 4)
    clean = U.layer_norm(x, None, None)
    x[1] = 3.0  # a row without variance: h = 0
    x[2, cols // 2] = float("inf")
    x[3, cols - 1] = float("nan")
    y, mean, rstd = U.layer_norm(x, None, None)
    assert (y[1] == 0).all() and abs(float(rstd[1]) - EPS**-0.5) <= 1e-4 * EPS**-0.5
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all() and torch.isinf(mean[2]) and torch.isnan(mean[3])
    for i in (0, 4, 5):  # a row's special values stay in it
        assert torch.equal(y[i], clean[0][i])
    dy = _tensor(6, cols, BF, 5)
    dx, dgamma, dbeta = U.layer_norm_bwd(dy, x, None, mean, rstd)
    want = U.layer_norm_bwd(dy[4:], x[4:], None, mean[4:], rstd[4:])[0]
    assert torch.equal(dx[4:], want) and torch.isnan(dx[2]).all() and torch.isnan(dx[3]).all()
    assert torch.isnan(dgamma).all() and torch.isfinite(dbeta).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("cols", [1, 100, 2048, 50000])
def test_empty_in_place_and_repeats(dt, cols):
    x = torch.empty(0, cols, dtype=dt, device="cuda")
    y, mean, rstd = U.layer_norm(x)
    dx, dgamma, dbeta = U.layer_norm_bwd(x, x, None, mean, rstd)
    assert y.shape == (0, cols) and dx.shape == (0, cols) and not dgamma.any() and not dbeta.any()
    x, dy = _tensor(9, cols, dt, 1), _tensor(9, cols, dt, 2)
    y, mean, rstd = U.layer_norm(x)
    got = U.layer_norm_bwd(dy, x, None, mean, rstd)
    again = U.layer_norm_bwd(dy, x, None, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for target in (0, 1):  # dx over x, dx over dy
        a, b = x.clone(), dy.clone()
        over = U.layer_norm_bwd(b, a, None, mean, rstd, out=a if target == 0 else b)
        assert all(torch.equal(p, q) for p, q in zip(over, got))
    dx, none, _ = U.layer_norm_bwd(dy, x, None, mean, rstd, weights=False)
    assert none is None and torch.equal(dx, got[0])
    a = x.clone()
    assert torch.equal(U.layer_norm(a, out=a)[0], y)


def test_other_stream():
    x = _tensor(4000, 2048, BF, 1)
    want = U.layer_norm(x)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        z = x.float().mul(1.0).to(BF)  # produced on this stream, consumed on it
        got = U.layer_norm(z)[0]
    s.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    x = torch.zeros(4, 8, dtype=BF, device="cuda")
    st = torch.zeros(4, device="cuda")
    for bad in (x.half(), x[0], x.t(), x.cpu(), x[:1].expand(4, 8)):
        with pytest.raises(ValueError):
            U.layer_norm(bad)
    with pytest.raises(ValueError):
        U.layer_norm(x, torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        U.layer_norm(x, torch.ones(8, device="cuda"), torch.zeros(8, device="cuda", dtype=BF))
    with pytest.raises(ValueError):
        U.layer_norm(x, torch.ones(16, device="cuda")[::2])
    with pytest.raises(ValueError):
        U.layer_norm(x, out=torch.empty(4, 9, dtype=BF, device="cuda"))
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(U.UFP4Error):
            U.layer_norm(x, eps=eps)
    with pytest.raises(ValueError):
        U.layer_norm_bwd(x.float(), x, None, st, st)
    with pytest.raises(ValueError):
        U.layer_norm_bwd(x, x, None, st[:3], st)


@pytest.mark.parametrize("rows,cols,dt", [(30011, 2304, torch.bfloat16), (20000, 1411, torch.float32), (4100, 16392, torch.bfloat16)])
def test_large_tensors(rows, cols, dt):
    """Tensors that no cache holds are stored by kernels of their own: the same numbers as from pieces of them."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, generator=g, device="cuda").to(dt)
    dy = torch.randn(rows, cols, generator=g, device="cuda").to(dt)
    gamma, beta = torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda")
    assert 2 * x.numel() * x.element_size() >= 1 << 28 or 3 * x.numel() * x.element_size() >= 1 << 28
    y, mean, rstd = U.layer_norm(x, gamma, beta)
    dx = U.layer_norm_bwd(dy, x, gamma, mean, rstd)[0]
    for a in range(0, rows, 1000):
        s = slice(a, min(rows, a + 1000))
        assert all(torch.equal(p, q[s]) for p, q in zip(U.layer_norm(x[s], gamma, beta), (y, mean, rstd)))
        assert torch.equal(U.layer_norm_bwd(dy[s], x[s], gamma, mean[s], rstd[s], weights=False)[0], dx[s])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [300, 40000])
def test_rows_past_32_bit_offsets(dt, cols):
    """Leading dimensions that put the third row past 2^31 elements."""
    ld = (1 << 30) + 4099
    hold = [torch.empty(2 * ld + cols, dtype=dt, device="cuda") for _ in range(2)]
    x, y = (h.as_strided((3, cols), (ld, 1)) for h in hold)
    x.copy_(torch.randn(3, cols, device="cuda"))
    g, b = torch.randn(cols, device="cuda"), torch.randn(cols, device="cuda")
    want, mean, rstd = U.layer_norm(x.contiguous(), g, b)
    got, m, r = U.layer_norm(x, g, b, out=y)
    assert torch.equal(got, want) and torch.equal(m, mean) and torch.equal(r, rstd)
    dy = torch.randn(3, cols, device="cuda").to(dt)
    assert all(torch.equal(p, q) for p, q in zip(U.layer_norm_bwd(dy, x, g, mean, rstd, out=y),
                                                 U.layer_norm_bwd(dy, x.contiguous(), g, mean, rstd)))


def test_weight_gradient_of_very_long_rows():
    """Rows whose 2 * cols sums are more than a grid of one workgroup for each 64 of them holds. The statistics are given as 0 and 1, so
    a column's dgamma is one product and one fused product and sum (two roundings of at most 2^-24 of the magnitudes each), its dbeta
    one sum of two numbers."""
    cols = (1 << 27) + 40
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.empty(2, cols, device="cuda", dtype=BF).normal_(generator=g) for _ in range(2))
    mean, rstd = torch.zeros(2, device="cuda"), torch.ones(2, device="cuda")
    _, dgamma, dbeta = U.layer_norm_bwd(dy, x, None, mean, rstd)
    for a in range(0, cols, 1 << 24):
        s = slice(a, min(cols, a + (1 << 24)))
        d, v = dy[:, s].double(), x[:, s].double()
        assert ((dgamma[s] - (d * v).sum(0)).abs() <= 4 * 2.0**-24 * (d * v).abs().sum(0)).all()
        assert torch.equal(dbeta[s], d.sum(0).float())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows", [1, 5, 300])
def test_rows_without_columns(dt, rows):
    """The mean and the variance of no numbers are 0 / 0; a row's statistics are never what the memory held before."""
    for _ in range(4):  # memory that the outputs are likely to get
        torch.full((rows,), 7.0, device="cuda")
        y, mean, rstd = U.layer_norm(torch.empty(rows, 0, dtype=dt, device="cuda"))
        assert y.shape == (rows, 0) and mean.shape == rstd.shape == (rows,)
        assert torch.isnan(mean).all() and torch.isnan(rstd).all()
    dx, dgamma, dbeta = U.layer_norm_bwd(y, y, None, mean, rstd)
    assert dx.shape == (rows, 0) and dgamma.shape == dbeta.shape == (0,)


# a row's threads and pieces: 8 to 64 x 1, 64 x 2, 256 x 1 .. 3, 1024 x 1 .. 4, and past them the columns' own kernel; the last three
# tensors are stored nontemporally
MANY_ROWS = [(40000, 33, BF), (20000, 100, BF), (20000, 250, BF), (9000, 500, BF), (7000, 1000, BF), (8192, 2048, BF), (4099, 1411, F32),
             (2500, 4000, BF), (1500, 5120, BF), (1500, 7000, BF), (1500, 7000, F32), (700, 16384, F32), (700, 16384, BF), (300, 20000, BF),
             (300, 33000, F32), (4100, 16392, BF), (30011, 2304, BF), (20000, 1411, F32), (6000, 16384, BF)]


@pytest.mark.parametrize("rows,cols,dt", MANY_ROWS)
def test_weight_gradients_of_many_rows(rows, cols, dt):
    """dgamma and dbeta where every workgroup adds up several rows. A workgroup has at most ceil(rows / parts) rows: a thread adds every
    kRows-th of them and the kRows sums are added in turn (together at most that many additions and one more; rows that share a wave have
    16 waves' sums, and three shuffles); then the parts' sums, ceil(parts / 16) in each of 16 waves and 16 more."""
    need = ctypes.c_size_t()
    assert U.lib().ufp4_layer_norm_bwd_workspace(U.OUT_BF16 if dt == BF else U.OUT_F32, rows, cols, ctypes.byref(need)) == 0
    parts = need.value // (8 * cols)
    assert parts > 1 and rows > 2 * parts
    x, dy = _tensor(rows, cols, dt, rows + cols), _tensor(rows, cols, dt, rows + 2 * cols, mean=0.1)
    gamma, _ = _weights(cols, F32, cols)
    _, mean, rstd = U.layer_norm(x, gamma, None)
    _, dgamma, dbeta = U.layer_norm_bwd(dy, x, gamma, mean, rstd)
    sums = torch.zeros(5, cols, dtype=torch.float64, device="cuda")
    for a in range(0, rows, 4096):
        s = slice(a, min(rows, a + 4096))
        d, v, m, r = dy[s].double(), x[s].double(), mean[s].double()[:, None], rstd[s].double()[:, None]
        t = d * ((v - m) * r)
        # h itself: one subtraction and one product of rounded numbers, relative to |x| + |mu|
        off = 2.0**-22 * d.abs() * (v.abs() + m.abs()) * r
        sums += torch.stack([q.sum(0) for q in (t, t.abs(), off, d, d.abs())])
    k = 2.0**-24 * (-(-rows // parts) + 1 + 16 + 3 + -(-parts // 16) + 16)
    _within("dgamma", dgamma, sums[0], k * sums[1] + 2 * sums[2])
    _within("dbeta", dbeta, sums[3], k * sums[4])
