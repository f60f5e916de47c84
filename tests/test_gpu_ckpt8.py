"""Activations kept in 8 bits, and the activation with its gradient, against definitions in 64 bits.

Kept values are compared bit for bit with a search over the format's levels. Squared ReLU: one fp32 product (bf16: exact, so the result
is the product rounded once; fp32: rounded once), its gradient two. Gated SiLU: a few fp32 roundings (e^x within 2 of the last place, the
reciprocal within 1), at most 2^-20 of the terms' magnitudes, and the result's own rounding.
"""

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
LEVELS = [n * 2.0**-9 if n < 8 else (8 + n % 8) * 2.0 ** (n // 8 - 10) for n in range(127)]


def _kept(x):
    """x's values in 8 bits, 64-bit arithmetic: levels by search, a middle to the even code."""
    at = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    rows, cols = x.shape
    t = torch.zeros(rows, -(-cols // 32) * 32, dtype=torch.float64, device=x.device)
    t[:, :cols] = x
    t = t.view(rows, -1, 32)
    finite = t.isfinite()
    top = torch.where(finite, t, 0.0).abs().amax(2, keepdim=True)
    e = torch.full_like(top, -124.0)
    for n in range(-123, 121):  # the smallest that covers
        e = torch.where(top > 448.0 * 2.0 ** (n - 1), float(n), e)
    a = torch.where(finite, t, 0.0).abs() / torch.exp2(e)
    low = torch.searchsorted((at[1:] + at[:-1]) / 2, a.contiguous())
    mid = ((at[1:] + at[:-1]) / 2)[low.clamp(max=125)]
    n = low + ((low % 2 == 1) & (mid == a)).long()
    v = torch.sign(t) * at[n] * torch.exp2(e)
    v = v.clamp(-1.875 * 2.0**127, 1.875 * 2.0**127)  # the largest level that is an fp32 number
    return torch.where(finite, v, float("nan")).reshape(rows, -1)[:, :cols]


def _same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=7e77), torch.nan_to_num(b.double(), nan=7e77))


def _values(rows, cols, dtype, seed, hard=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    if hard:
        x *= torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g, device="cuda").float())
        for r in range(0, rows, 7):  # rows of tiny, huge, equal, and of few values
            x[r] *= (1e-38, 1e30, 0.0, 1e-44)[r // 7 % 4]
            if r + 1 < rows:
                x[r + 1] = 1.75 * 2.0 ** (r % 9)
            if r + 2 < rows:
                x[r + 2] = 1.7578125 * 2.0 ** (r % 9)  # one bf16 step above the largest level: the next scale
            if r + 3 < rows:
                x[r + 3, 1:] = 0.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 31), (1, 32), (1, 33), (5, 64), (300, 100), (64, 1411), (3, 5000), (1000, 8), (2, 70000),
                                       (70000, 33), (2048, 8192)])
def test_save_and_load(rows, cols, dtype):
    x = _values(rows, cols, dtype, rows + cols)
    c = U.checkpoint8_save(x)
    assert c.shape == (rows, cols) and c.codes.shape == (rows, -(-cols // 32) * 32) and c.scales.shape == (rows, -(-cols // 128) * 4)
    ref = _kept(x)
    for out in (F32, BF):
        got = U.checkpoint8_load(c, out)
        assert got.dtype == out and _same(got, ref)
    assert not c.codes[:, cols:].any()
    # every value within half a step of its level
    ok = (ref - x.double()).abs() <= 2.0**-4 * x.double().abs() + 2.0**-134
    top = x.double().abs().amax() * 2.0**-18  # and, of values far below their block's largest, half of the smallest step
    assert bool((ok | ((ref - x.double()).abs() <= top)).all())


def test_every_bf16_number_alone():
    """A block with one number and nothing else, for all 65536."""
    x = torch.zeros(65536, 32, dtype=torch.int16, device="cuda")
    x[:, 5] = torch.arange(65536, device="cuda").to(torch.int16)
    x = x.view(BF)
    assert _same(U.checkpoint8_load(U.checkpoint8_save(x)), _kept(x))


def test_every_level_and_middle():
    """All levels, the middles between them and the fp32 numbers beside those, in blocks whose scale is 1 and 2^-100."""
    at = torch.tensor(LEVELS, dtype=torch.float64)
    mid = ((at[1:] + at[:-1]) / 2).float()
    v = torch.cat([at.float(), mid, torch.nextafter(mid, torch.tensor(0.0)), torch.nextafter(mid, torch.tensor(1e9))])
    x = torch.zeros(2 * len(v), 32)
    x[:, 0] = 448.0
    x[: len(v), 9], x[len(v) :, 9] = v, -v
    for scale in (1.0, 2.0**-100):
        y = (x * scale).cuda()
        assert _same(U.checkpoint8_load(U.checkpoint8_save(y), F32), _kept(y))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_infinities_and_nan(dtype):
    x = _values(9, 96, dtype, 1, hard=False)
    x[0, 3], x[1, 40], x[2, 64], x[3, :32], x[4] = float("nan"), float("inf"), float("-inf"), float("inf"), float("nan")
    got = U.checkpoint8_load(U.checkpoint8_save(x), F32)
    assert _same(got, _kept(x))
    assert bool(got[1, 40].isnan()) and int(got[:3].isnan().sum()) == 3


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("pad,at", [(8, 8), (5, 3), (1, 1)])
def test_strides(dtype, pad, at):
    x = _values(130, 200, dtype, 2)
    wide = torch.full((131, 200 + pad), float("nan"), dtype=dtype, device="cuda")
    wide[:130, at : at + 200] = x
    c = U.checkpoint8_save(wide[:130, at : at + 200])
    assert _same(U.checkpoint8_load(c, F32), _kept(x))
    out = torch.full((131, 200 + pad), 5.0, dtype=dtype, device="cuda")
    U.checkpoint8_load(c, out=out[:130, at : at + 200])
    assert _same(out[:130, at : at + 200], _kept(x))
    out[:130, at : at + 200] = 5.0
    assert bool((out == 5.0).all())
    # into a checkpoint of wider rows
    into = U.Checkpoint8(torch.full((130, 256), 9, dtype=torch.uint8, device="cuda"), torch.full((130, 8), 9, dtype=torch.uint8, device="cuda"), 200)
    assert U.checkpoint8_save(x, out=into) is into
    assert _same(U.checkpoint8_load(into, F32), _kept(x))
    assert bool((into.codes[:, 224:] == 9).all()) and bool((into.scales[:, 7:] == 9).all())


def test_nothing_to_keep():
    for shape in ((0, 40), (3, 0), (0, 0)):
        c = U.checkpoint8_save(torch.empty(shape, device="cuda"))
        assert tuple(U.checkpoint8_load(c).shape) == shape


# ------------------------------------------------------------------------------------------------
# activation
# ------------------------------------------------------------------------------------------------

def _act64(u, kind):
    """(a, its slope in u's parts, magnitudes of the terms of the slopes)."""
    if kind == "relu2":
        r = torch.relu(u)
        return r * r, (2 * r,), (2 * r,)
    g, v = u.chunk(2, 1)
    s, q = torch.sigmoid(g), torch.sigmoid(-g)
    return g * s * v, (v * (s + g * s * q), g * s), (v.abs() * (s + (g * s * q).abs()), (g * s).abs())


def _near(got, ref, terms, dtype):
    half = 2.0**-8 if dtype == BF else 2.0**-24
    return bool(((got.double() - ref).abs() <= half * ref.abs() + 2.0**-20 * terms + 2.0**-126).all())


@pytest.mark.parametrize("kind", ["relu2", "swiglu"])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (2, 31), (42, 1408), (300, 33), (129, 1411), (2, 9000), (4096, 1024)])
def test_activation_and_gradient(rows, cols, dtype, kind):
    parts = 2 if kind == "swiglu" else 1
    g = torch.Generator(device="cuda").manual_seed(rows * cols)
    u = (3.0 * torch.randn(rows, parts * cols, generator=g, device="cuda")).to(dtype)
    da = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    a, none = U.activation(u, kind)
    assert none is None
    ref, slopes, sizes = _act64(u.double(), kind)
    assert _near(a, ref, ref.abs(), dtype)
    a2, kept = U.activation(u, kind, save=True)
    assert torch.equal(a, a2) and kept.shape == tuple(u.shape) and kept.parts == parts
    values = torch.cat([_kept(p) for p in u.chunk(parts, 1)], 1)
    assert _same(U.checkpoint8_load(kept, F32), values) and _same(U.checkpoint8_load(kept), values)
    for saved, at in ((u, u.double()), (kept, values)):
        ref, slopes, sizes = _act64(at, kind)
        du, again = U.activation_bwd(da, saved, kind)
        assert du.dtype == dtype and du.shape == u.shape and _near(again, ref, ref.abs(), dtype)
        for p in range(parts):
            d = da.double()
            assert _near(du[:, p * cols : (p + 1) * cols], slopes[p] * d, sizes[p] * d.abs(), dtype)
        du2, none = U.activation_bwd(da, saved, kind, again=False)
        assert none is None and torch.equal(du, du2)
    if kind == "relu2":  # one rounding
        r = torch.relu(u.double())
        assert torch.equal(a, (r * r).to(dtype))


@pytest.mark.parametrize("kind", ["relu2", "swiglu"])
def test_gradient_by_differences(kind):
    """du against (f(u + h) - f(u - h)) / 2h in 64 bits."""
    parts = 2 if kind == "swiglu" else 1
    g = torch.Generator(device="cuda").manual_seed(9)
    u = 2.0 * torch.randn(64, parts * 96, generator=g, device="cuda")
    da = torch.randn(64, 96, generator=g, device="cuda")
    du, _ = U.activation_bwd(da, u, kind)
    h = 1e-5
    for p in range(parts):
        step = torch.zeros_like(u, dtype=torch.float64)
        step[:, p * 96 : (p + 1) * 96] = h
        slope = (_act64(u.double() + step, kind)[0] - _act64(u.double() - step, kind)[0]) / (2 * h)
        err = (du[:, p * 96 : (p + 1) * 96].double() - slope * da.double()).abs()
        assert float(err.max()) < 1e-4  # h^2 f''' / 6, h at the kink, and 2^-20 of values below 30


@pytest.mark.parametrize("kind", ["relu2", "swiglu"])
def test_activation_at_the_ends(kind):
    v = [0.0, -0.0, 1e-40, -1e-40, 88.0, -88.0, 89.0, -89.0, 104.0, -104.0, 1e10, -1e10, 3e38, float("inf"), float("nan")]
    g = torch.tensor([v], device="cuda")
    u = g if kind == "relu2" else torch.cat([g, torch.ones_like(g)], 1)
    a, _ = U.activation(u, kind)
    ref = _act64(u.double(), kind)[0].float()
    got = a[0].tolist()
    for x, y, r in zip(v, got, ref[0].tolist()):
        if r != r:
            assert y != y, x
        elif abs(r) == float("inf"):
            assert y == r, x
        else:
            # e^-|g| is rounded to a multiple of 2^-149 there (off by up to 2^-150), its product with r again, and g times that is the result
            assert abs(y - r) <= 1e-5 * abs(r) + (1 + abs(x)) * 2.0**-149, (x, y, r)
    du, _ = U.activation_bwd(torch.ones_like(g), u, kind)
    assert bool(du[0, :12].isfinite().all()) and bool(du[0, 14].isnan())


@pytest.mark.parametrize("kind", ["relu2", "swiglu"])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_activation_strides(kind, dtype):
    parts = 2 if kind == "swiglu" else 1
    g = torch.Generator(device="cuda").manual_seed(8)
    rows, cols = 70, 99

    def wide(n):
        t = torch.randn(rows + 1, n + 7, generator=g, device="cuda").to(dtype)
        return t[:rows, 3 : 3 + n]

    u, da = wide(parts * cols), wide(cols)
    out, dout = wide(cols), wide(parts * cols)
    a, kept = U.activation(u, kind, save=True, out=out)
    assert a.data_ptr() == out.data_ptr() and torch.equal(out, U.activation(u.contiguous(), kind)[0])
    du, _ = U.activation_bwd(da, kept, kind, out=dout)
    assert du.data_ptr() == dout.data_ptr() and torch.equal(dout, U.activation_bwd(da.contiguous(), kept, kind)[0])


def test_past_32_bits():
    """More than 2^32 bytes in and out."""
    rows, cols = 70_000, 32_768
    x = torch.zeros(rows, cols, dtype=BF, device="cuda")
    x[-3:] = _values(3, cols, BF, 4)
    c = U.checkpoint8_save(x)
    assert _same(U.checkpoint8_load(c)[-3:], _kept(x[-3:]))
    a, kept = U.activation(x, "relu2", save=True)
    assert torch.equal(a[-3:], (torch.relu(x[-3:].double()) ** 2).to(BF)) and torch.equal(kept.codes[-3:], c.codes[-3:])
    du, again = U.activation_bwd(x, kept, "relu2")
    at = torch.relu(_kept(x[-3:]))
    assert _same(again[-3:], (at * at).to(BF)) and _same(du[-3:], (2 * at * x[-3:].double()).to(BF))


def test_streams_and_graph():
    g = torch.Generator(device="cuda").manual_seed(3)
    u = torch.randn(300, 2 * 130, generator=g, device="cuda").to(BF)
    da = torch.randn(300, 130, generator=g, device="cuda").to(BF)

    def step():
        a, kept = U.activation(u, "swiglu", save=True)
        return a, *U.activation_bwd(da, kept, "swiglu"), U.checkpoint8_load(kept)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = step()
    side.synchronize()
    for x, y in zip(outs, step()):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for _ in range(3):
        u.copy_(torch.randn(300, 260, generator=g, device="cuda").to(BF))
        da.neg_()
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for x, y in zip(captured, eager):
            assert torch.equal(x, y)
