"""Tokens sorted by expert, dispatched, combined, and the gradients, against plain computations.

The sort is exact. dispatch without weights is a copy. The others sum k products in fp32: at most (k + 1) * 2^-24 of the
sum of magnitudes, plus the output's rounding (bf16: 2^-9 of its value, taken as 2^-8); the dot products of combine_bwd add
cols terms, at most 32 per thread in a row segment and one more segment's worth per 8192 columns, then 9 levels.
"""

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _order64(ids, experts):
    """The stable order on the CPU."""
    flat = ids.reshape(-1).cpu().tolist()
    slots = sorted((e, i) for i, e in enumerate(flat) if 0 <= e < experts)
    rows, source, offsets = [-1] * len(flat), [-1] * len(flat), [0] * (experts + 1)
    for place, (e, i) in enumerate(slots):
        rows[i], source[place] = place, i
        offsets[e + 1] += 1
    for e in range(experts):
        offsets[e + 1] += offsets[e]
    return offsets, rows, source


def _ids(tokens, k, experts, seed, kind="random", dtype=torch.int32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "one":  # every token to the last expert
        ids = torch.full((tokens, k), experts - 1, device="cuda")
    elif kind == "none":
        ids = torch.full((tokens, k), -1, device="cuda")
    else:
        ids = torch.randint(0, experts, (tokens, k), generator=g, device="cuda")
        if kind == "holes":
            bad = torch.tensor([-1, experts, -(2**31), 2**31 - 1], device="cuda")
            pick = bad[torch.randint(0, 4, (tokens, k), generator=g, device="cuda")]
            ids = torch.where(torch.rand(tokens, k, generator=g, device="cuda") < 0.2, pick, ids)
    return ids.to(dtype)


@pytest.mark.parametrize("tokens,k,experts", [(0, 2, 4), (1, 1, 1), (1, 6, 64), (7, 6, 64), (64, 1, 3), (100, 8, 1024),
                                              (4096, 1, 2), (4097, 1, 5), (1365, 3, 7), (16384, 6, 64), (9001, 8, 1000),
                                              (60001, 5, 31), (131072, 2, 128)])
@pytest.mark.parametrize("kind", ["random", "holes"])
def test_sort(tokens, k, experts, kind):
    ids = _ids(tokens, k, experts, tokens + k, kind)
    offsets, rows, source = U.moe_sort(ids, experts)
    want = _order64(ids, experts)
    assert offsets.tolist() == want[0]
    assert rows.shape == (tokens, k) and rows.reshape(-1).tolist() == want[1]
    assert source.tolist() == want[2]


@pytest.mark.parametrize("kind", ["one", "none"])
@pytest.mark.parametrize("tokens", [5, 5000, 200000])
def test_sort_one_expert_or_none(tokens, kind):
    ids = _ids(tokens, 2, 16, 1, kind, torch.int64)
    offsets, rows, source = U.moe_sort(ids, 16)
    n = 2 * tokens
    at = torch.arange(n, device="cuda", dtype=torch.int32)
    if kind == "one":
        assert offsets.tolist() == [0] * 16 + [n] and torch.equal(rows.view(-1), at) and torch.equal(source, at)
    else:
        assert offsets.tolist() == [0] * 17 and (rows == -1).all() and (source == -1).all()


def test_sort_int64_ids_past_32_bits():
    ids = torch.tensor([[3, 2**32], [2**40 + 1, 0]], device="cuda")  # low words that would be experts
    offsets, rows, source = U.moe_sort(ids, 4)
    assert offsets.tolist() == [0, 1, 1, 1, 2] and rows.tolist() == [[1, -1], [-1, 0]] and source.tolist() == [3, 0, -1, -1]


CASES = [(1, 1, 1, 1), (1, 6, 64, 2048), (7, 2, 8, 63), (5, 3, 4, 517), (33, 4, 16, 1411), (64, 8, 32, 2048), (11, 2, 4, 8200),
         (3, 64, 128, 100), (300, 6, 64, 5120), (40, 2, 8, 20001)]


def _case(tokens, k, experts, cols, dt, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed + tokens * 7 + cols)
    ids = _ids(tokens, k, experts, seed + 3, "holes")
    offsets, rows, _ = U.moe_sort(ids, experts)

    def make(n):
        buf = torch.full((max(1, n), cols + pad), float("nan"), device="cuda")
        buf[:n, :cols] = torch.randn(n, cols, generator=g, device="cuda")
        return buf.to(dt)[:n, :cols]

    w = torch.rand(tokens, k, generator=g, device="cuda") - 0.3
    return rows, offsets, make(tokens), make(tokens * k), w


def _unit(dt):
    return 2.0**-8 if dt == BF else 2.0**-23


def _scatter64(x, rows, w):
    out = torch.zeros(rows.numel(), x.shape[1], dtype=torch.float64, device="cuda")
    for t in range(rows.shape[0]):
        for j in range(rows.shape[1]):
            if rows[t, j] >= 0:
                out[rows[t, j]] = x[t].double() * (1.0 if w is None else w[t, j].double())
    return out


def _gather64(y, rows, w):
    keep = (rows >= 0)[:, :, None]
    each = torch.where(keep, y.double()[rows.long().clamp(min=0)], 0.0)
    return each if w is None else each * w.double()[:, :, None]


@pytest.mark.parametrize("tokens,k,experts,cols", CASES)
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("weighted", [False, True])
def test_dispatch_combine(tokens, k, experts, cols, dt, weighted):
    rows, offsets, x, y, w = _case(tokens, k, experts, cols, dt)
    w = w if weighted else None
    out = torch.full((tokens * k, cols), float("nan"), device="cuda").to(dt)
    got = U.moe_dispatch(x, rows, offsets, w, out=out)
    want = _scatter64(x, rows.cpu(), w)
    if not weighted:
        assert torch.equal(got.double(), want)
    assert ((got.double() - want).abs() <= _unit(dt) * want.abs()).all()
    each = _gather64(y, rows, w)
    ref, size = each.sum(1), each.abs().sum(1)
    got = U.moe_combine(y, rows, w)
    assert ((got.double() - ref).abs() <= (k + 1) * 2.0**-24 * size + _unit(dt) * ref.abs()).all()


@pytest.mark.parametrize("tokens,k,experts,cols", CASES)
@pytest.mark.parametrize("dt", [BF, F32])
def test_combine_bwd(tokens, k, experts, cols, dt):
    rows, offsets, dout, y, w = _case(tokens, k, experts, cols, dt, 5)
    out = torch.full(y.shape, float("nan"), device="cuda").to(dt)
    dy, dw = U.moe_combine_bwd(dout, y, rows, offsets, w, out=out)
    want = _scatter64(dout, rows.cpu(), w)
    assert ((dy.double() - want).abs() <= _unit(dt) * want.abs()).all()
    terms = _gather64(y, rows, None) * dout.double()[:, None, :]
    bound = (48 + cols / 256) * 2.0**-24 * terms.abs().sum(2)
    assert ((dw.double() - terms.sum(2)).abs() <= bound).all()
    assert (dw[rows < 0] == 0).all()
    # the same call without weights, and over y itself
    dy1, dw1 = U.moe_combine_bwd(dout, y, rows, offsets)
    assert torch.equal(dy1, U.moe_dispatch(dout, rows, offsets)) and torch.equal(dw1, dw)
    over = y.clone()
    dy2, dw2 = U.moe_combine_bwd(dout, over, rows, offsets, w, out=over)
    assert torch.equal(dy2, dy) and torch.equal(dw2, dw)


def test_gradients_are_adjoint_and_match_differences():
    """<dispatch(x), g> = <x, combine(g)> to fp32, and dw against differences of 64-bit losses."""
    rows, offsets, x, y, w = _case(9, 3, 5, 40, F32, 2)
    g = torch.randn(27, 40, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    a = (U.moe_dispatch(x, rows, offsets, w).double() * g.double()).sum()
    b = (x.double() * U.moe_combine(g, rows, w).double()).sum()
    assert abs(float(a - b)) <= 1e-5 * float(x.double().norm() * g.double().norm())
    dout = x
    dy, dw = U.moe_combine_bwd(dout, y, rows, offsets, w)

    def loss(y, w):
        return float((_gather64(y, rows, w).sum(1) * dout.double()).sum())

    y64, w64, s = y.double(), w.double(), 1e-4
    for i in range(27):
        hi, lo = w64.clone(), w64.clone()
        hi.view(-1)[i] += s
        lo.view(-1)[i] -= s
        assert abs(float(dw.view(-1)[i]) - (loss(y64, hi) - loss(y64, lo)) / (2 * s)) <= 1e-4
    for i in range(0, 27 * 40, 71):
        hi, lo = y64.clone(), y64.clone()
        hi.view(-1)[i] += s
        lo.view(-1)[i] -= s
        assert abs(float(dy.view(-1)[i]) - (loss(hi, w64) - loss(lo, w64)) / (2 * s)) <= 1e-5


@pytest.mark.parametrize("dt", [BF, F32])
def test_strides_and_rows_out_of_range(dt):
    rows, offsets, x, y, w = _case(13, 2, 4, 301, dt, 1, pad=5)
    xc, yc = x.contiguous(), y.contiguous()
    assert torch.equal(U.moe_dispatch(x, rows, offsets, w), U.moe_dispatch(xc, rows, offsets, w))
    assert torch.equal(U.moe_combine(y, rows, w), U.moe_combine(yc, rows, w))
    a, b = U.moe_combine_bwd(x, y, rows, offsets, w), U.moe_combine_bwd(xc, yc, rows, offsets, w)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # rows that lie outside y count as dropped
    far = rows.clone()
    far[3, 0], far[4, 1] = 26, 2**31 - 1
    gone = rows.clone()
    gone[3, 0] = gone[4, 1] = -1
    assert torch.equal(U.moe_combine(y, far, w), U.moe_combine(y, gone, w))


def test_special_values_stay_in_their_token():
    rows, offsets, x, y, w = _case(20, 2, 4, 70, BF, 3)
    keep = int((rows.min(1).values >= 0).nonzero()[0])
    clean = U.moe_combine(y, rows, w)
    y2 = y.clone()
    y2[rows[keep, 0].long()] = float("nan")
    y2[int(offsets[-1]):] = float("inf")  # rows that no slot takes are not read
    got = U.moe_combine(y2, rows, w)
    assert torch.isnan(got[keep]).all()
    rest = torch.arange(20, device="cuda") != keep
    assert torch.equal(got[rest], clean[rest])


def test_empty():
    rows = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    offsets = torch.zeros(5, dtype=torch.int64, device="cuda")
    x = torch.empty(0, 16, dtype=BF, device="cuda")
    assert U.moe_dispatch(x, rows, offsets).shape == (0, 16) and U.moe_combine(x, rows).shape == (0, 16)
    dy, dw = U.moe_combine_bwd(x, x, rows, offsets)
    assert dy.shape == (0, 16) and dw.shape == (0, 2)
    rows = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")  # nothing kept
    y = torch.full((6, 16), float("nan"), dtype=BF, device="cuda")
    assert (U.moe_combine(y, rows) == 0).all()
    assert (U.moe_dispatch(torch.ones(3, 16, dtype=BF, device="cuda"), rows, offsets) == 0).all()
    dy, dw = U.moe_combine_bwd(torch.ones(3, 16, dtype=BF, device="cuda"), y, rows, offsets)
    assert (dy == 0).all() and (dw == 0).all()


def test_refusals():
    x = torch.zeros(4, 8, dtype=BF, device="cuda")
    rows = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    for bad in (rows.float(), rows[0], rows.t()):
        with pytest.raises(ValueError):
            U.moe_sort(bad, 2)
    for n in (0, 1025):
        with pytest.raises(U.UFP4Error):
            U.moe_sort(rows, max(n, 0) or 0) if n else U.moe_sort(rows, 0)
    with pytest.raises(U.UFP4Error):
        U.moe_sort(torch.zeros(1, 65, dtype=torch.int32, device="cuda"), 4)
    with pytest.raises(ValueError):
        U.moe_dispatch(x[:3], rows, off)
    with pytest.raises(ValueError):
        U.moe_dispatch(x, rows.long(), off)
    with pytest.raises(ValueError):
        U.moe_dispatch(x, rows, off.int())
    with pytest.raises(ValueError):
        U.moe_dispatch(x, rows, off, torch.ones(4, 3, device="cuda"))
    with pytest.raises(ValueError):
        U.moe_dispatch(x, rows, off, torch.ones(4, 2, device="cuda", dtype=BF))
    with pytest.raises(ValueError):
        U.moe_combine(x.half(), rows)
    with pytest.raises(U.UFP4Error):
        U.moe_combine_bwd(x, x, rows, off)  # y must hold tokens * k rows


@pytest.mark.parametrize("tokens,k,cols,dt", [(9000, 7, 2200, torch.bfloat16), (8000, 3, 3001, torch.float32)])
def test_large_tensors(tokens, k, cols, dt):
    """Tensors that no cache holds are read and stored by kernels of their own."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(dt)
    assert tokens * k * cols * x.element_size() >= 1 << 28
    ids = torch.topk(torch.rand(tokens, 16, generator=g, device="cuda"), k, dim=1).indices
    ids[torch.rand(tokens, k, generator=g, device="cuda") < 0.03] = -1
    w = torch.rand(tokens, k, generator=g, device="cuda")
    off, rows, source = U.moe_sort(ids, 16)
    used = int(off[-1])
    y = U.moe_dispatch(x, rows, off)
    assert torch.equal(y[:used], x[source[:used].long() // k]) and not y[used:].any()
    out, small = U.moe_combine(y, rows, w), 1000
    dy, dw = U.moe_combine_bwd(x, y, rows, off, w)
    for a in range(0, tokens, small):  # fewer tokens at a time: the other kernels, on the rows that these tokens have
        s = slice(a, min(tokens, a + small))
        at = rows[s].reshape(-1)
        part = torch.where(at[:, None] >= 0, y[at.clamp(min=0).long()], torch.zeros((), dtype=dt, device="cuda"))
        place = torch.arange(at.numel(), device="cuda", dtype=torch.int32)
        local = torch.where(at >= 0, place, torch.full_like(place, -1)).view(-1, k)
        assert torch.equal(U.moe_combine(part, local, w[s]), out[s])
        n = torch.tensor([0, at.numel()], device="cuda")
        pdy, pdw = U.moe_combine_bwd(x[s], part, local, n, w[s])
        have = at >= 0
        assert torch.equal(pdw, dw[s]) and torch.equal(pdy[have], dy[at[have].long()])
    assert not dy[used:].any()


def test_rows_past_32_bit_offsets():
    """Leading dimensions that put rows past 2^31 elements."""
    ld, cols = (1 << 29) + 4099, 700
    ids = torch.tensor([[0, 2], [1, 0], [2, -1]], device="cuda")
    off, rows, _ = U.moe_sort(ids, 3)
    x = torch.randn(3, cols, device="cuda").to(torch.bfloat16)
    w = torch.rand(3, 2, device="cuda")
    hold = torch.empty(5 * ld + cols, dtype=torch.bfloat16, device="cuda")
    y = hold.as_strided((6, cols), (ld, 1))
    U.moe_dispatch(x, rows, off, w, out=y)
    near = U.moe_dispatch(x, rows, off, w)
    assert torch.equal(y, near) and torch.equal(U.moe_combine(y, rows, w), U.moe_combine(near, rows, w))
    want = U.moe_combine_bwd(x, near, rows, off, w)
    dy, dw = U.moe_combine_bwd(x, y, rows, off, w, out=y)
    assert torch.equal(dy, want[0]) and torch.equal(dw, want[1])


@pytest.mark.parametrize("cols", [40, 500, 512, 700, 1024, 1030, 2041, 2056])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("k", [1, 3, 5, 8])
def test_many_tokens_of_every_width(cols, dt, k):
    """Tokens past those that take a workgroup per slot: rows of one, two and four pieces a lane, and of several segments."""
    tokens = 2500
    rows, offsets, x, y, w = _case(tokens, k, 16, cols, dt, cols)
    assert tokens * k > 2048
    used, flat = int(offsets[-1]), rows.reshape(-1).long()
    have = flat >= 0
    want = torch.zeros(tokens * k, cols, dtype=torch.float64, device="cuda")
    want[flat[have]] = (x.double()[:, None, :] * w.double()[:, :, None]).reshape(-1, cols)[have]
    got = U.moe_dispatch(x, rows, offsets, w)
    assert ((got.double() - want).abs() <= _unit(dt) * want.abs()).all() and not got[used:].any()
    each = _gather64(y, rows, w)
    ref, size = each.sum(1), each.abs().sum(1)
    assert ((U.moe_combine(y, rows, w).double() - ref).abs() <= (k + 1) * 2.0**-24 * size + _unit(dt) * ref.abs()).all()
    dy, dw = U.moe_combine_bwd(x, y, rows, offsets, w)
    assert torch.equal(dy, got)
    terms = _gather64(y, rows, None) * x.double()[:, None, :]
    assert ((dw.double() - terms.sum(2)).abs() <= (48 + cols / 256) * 2.0**-24 * terms.abs().sum(2)).all()
    over = y.clone()
    again = U.moe_combine_bwd(x, over, rows, offsets, w, out=over)
    assert torch.equal(again[0], dy) and torch.equal(again[1], dw)
