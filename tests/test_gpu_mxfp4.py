"""Microscaled 4-bit quantizers against the CPU oracle (codes and scale bytes exact), their layout, and values at the edges."""

import numpy as np
import pytest
import torch

from oracle import ufp4_oracle as O
from paper_2606_20381_amd import ufp4 as U
from paper_2606_20381_amd.workloads import bf16_bits

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
MASK = 0x6A09


def _tensor(rows, cols, seed, pad=0, spread=False):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(rows, cols + pad, generator=g)
    if spread:  # every binade of bf16, zeros and whole zero blocks
        t *= torch.exp2(torch.randint(-126, 120, (rows, cols + pad), generator=g).float())
        t[torch.rand(rows, cols + pad, generator=g) < 0.1] = 0
        t[: rows // 3, : 32 * max(1, cols // 96)] = 0
    return t.to(BF).cuda()[:, :cols]


def _levels(q):
    """(signed E2M1 codes [rows, red], scale bytes) of a GPU operand; a negative zero counts as zero."""
    c = q.codes_rows().cpu().numpy()
    n = np.stack([c & 15, c >> 4], -1).reshape(q.rows, q.red).astype(np.int64)
    return np.where(n & 8, -(n & 7), n & 7), q.scales_rows().cpu().numpy()


def _check(q, a, rounding, rht, seed=0, stream=0, mask=MASK, row_ids=None, what=""):
    idx, e8 = O.quantize_rows_mxfp4(a, rounding, rht, mask, seed, stream, row_ids)
    gi, ge = _levels(q)
    assert np.array_equal(ge, e8), f"{what}: {np.argwhere(ge != e8)[:3]}"
    assert np.array_equal(gi, idx), f"{what}: {np.argwhere(gi != idx)[:3]}"


SHAPES = [(1, 32), (3, 64), (128, 96), (64, 128), (129, 160), (200, 288), (33, 1024), (300, 544)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("rounding", [U.RTNE, U.SR])
# (rotated blocks that span every binade are wider than what fp64 sums exactly; test_rotated_edges has the ends of the range)
@pytest.mark.parametrize("rht,spread", [(False, False), (True, False), (False, True)])
def test_rowwise(rows, cols, rht, rounding, spread):
    x = _tensor(rows, cols, rows + cols, pad=8, spread=spread)
    q = U.mxfp4_quantize(x, rht=rht, sign_mask=MASK, rounding=rounding, seed=2**40 + 5, stream_id=3)
    a = O.bf16_bits_to_f32(bf16_bits(x.cpu()))
    _check(q, a, rounding, rht, 2**40 + 5, 3)


@pytest.mark.parametrize("rows,cols", [(32, 1), (64, 3), (96, 128), (128, 64), (160, 129), (288, 200), (1024, 33), (544, 300)])
@pytest.mark.parametrize("rht", [False, True])
@pytest.mark.parametrize("rounding", [U.RTNE, U.SR])
def test_transposed(rows, cols, rht, rounding):
    pad = -cols % 8
    x = _tensor(rows, cols, rows * 3 + cols, pad=pad)
    q = U.mxfp4_quantize(x, transpose=True, rht=rht, sign_mask=MASK, rounding=rounding, seed=77, stream_id=1)
    a = np.ascontiguousarray(O.bf16_bits_to_f32(bf16_bits(x.cpu())).T)
    _check(q, a, rounding, rht, 77, 1)


def test_transposed_last_column_of_the_storage():
    """An odd column count whose last row ends the allocation: nothing past it is read into a code."""
    base = torch.randn(32 * 64 - 1).to(BF).cuda()
    x = base.as_strided((32, 63), (64, 1))
    q = U.mxfp4_quantize(x, transpose=True)
    _check(q, np.ascontiguousarray(O.bf16_bits_to_f32(bf16_bits(x.cpu())).T), U.RTNE, False)


@pytest.mark.parametrize("transpose", [False, True])
def test_every_bf16_value_at_every_scale(transpose):
    """Each finite bf16 pattern in blocks topped by each binade from the smallest subnormal to the largest number."""
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    fin = (bits & 0x7F80) != 0x7F80
    mags = np.unique(bits[fin] & 0x7FFF)
    rows = []
    for e in list(range(0, 255, 6)) + [1, 2, 3, 253, 254]:
        top = np.uint16((e << 7) | 0x35 if e else 1)
        below = mags[mags <= top][-31 * 40:]
        below = np.resize(below, (-(-len(below) // 31), 31))
        sign = (np.arange(below.size).reshape(below.shape) % 2).astype(np.uint16) << 15
        rows.append(np.concatenate([np.full((len(below), 1), top, np.uint16), below | sign], 1))
    b = np.concatenate(rows)
    x = torch.from_numpy(b.view(np.int16)).view(BF)
    x = x.t().contiguous() if transpose else x
    if transpose:
        x = torch.nn.functional.pad(x, (0, -x.shape[1] % 8))
    q = U.mxfp4_quantize(x.cuda()[:, : len(b)] if transpose else x.cuda(), transpose=transpose)
    _check(q, O.bf16_bits_to_f32(b), U.RTNE, False)
    back = U.mxfp4_dequantize(q).double().cpu().numpy()
    assert np.array_equal(back, O.dequantize_mxfp4(*O.quantize_rows_mxfp4(O.bf16_bits_to_f32(b), U.RTNE, False)))


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("rounding", [U.RTNE, U.SR])
def test_rotated_edges(transpose, rounding):
    """Rotated blocks past FLT_MAX and down to the subnormals: scales follow the exact sums."""
    g = np.random.default_rng(3)
    a = g.standard_normal((64, 64)).astype(np.float32)
    scale = np.ones((64, 1), np.float32)
    scale[:16] = 2.0**-126
    a = a * scale
    a[16:32] = np.float32(3.3e38) * np.sign(a[16:32])
    x = torch.from_numpy(a).to(BF)
    a = O.bf16_bits_to_f32(bf16_bits(x))
    src = x.t().contiguous().cuda() if transpose else x.cuda()
    q = U.mxfp4_quantize(src, transpose=transpose, rht=True, sign_mask=MASK, rounding=rounding, seed=9)
    # the sums in fp64 without an exponent limit, rounded to 24 bits (gradually below 2^-126)
    y = O.rht_exact_f64(a.reshape(64, 4, 16), MASK).reshape(64, 2, 32)
    small = np.abs(y) < 2.0**-126
    m, e = np.frexp(y)
    y = np.where(small, np.round(np.ldexp(y, 149)) * 2.0**-149, np.ldexp(np.round(np.ldexp(m, 24)), e - 24))
    E = np.maximum(np.frexp(np.abs(y).max(-1))[1] - 1 - 2, -127)
    assert (E[16:32] + 127).max() > 252  # past what bf16 holds
    gi, ge = _levels(q)
    assert np.array_equal(ge, (E + 127).astype(np.uint8))
    v = np.clip(np.ldexp(y, -E[..., None]), -6, 6).astype(np.float32)
    if rounding == U.RTNE:
        want = O.round_nearest_even(v, O.E2M1)
    else:
        u = O.sr_draws(np.arange(4)[None, :], np.arange(64)[:, None], 9, 0).reshape(64, 2, 32)
        want = O.round_stochastic(v, u, O.E2M1)
    assert np.array_equal(gi, want.reshape(64, 64))


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("rht", [False, True])
@pytest.mark.parametrize("rounding", [U.RTNE, U.SR])
def test_not_finite_blocks(transpose, rht, rounding):
    x = _tensor(64, 64, 1)
    x[5, 3], x[7, 40], x[20, 33] = float("inf"), float("nan"), float("-inf")
    clean = x.clone()
    clean[~torch.isfinite(x)] = 0
    q = U.mxfp4_quantize(x, transpose=transpose, rht=rht, sign_mask=MASK, rounding=rounding)
    c = U.mxfp4_quantize(clean, transpose=transpose, rht=rht, sign_mask=MASK, rounding=rounding)
    bad = ~torch.isfinite(x.t() if transpose else x).view(64, 2, 32).all(2)
    e, ec = q.scales_rows(), c.scales_rows()
    assert (e[bad] == 255).all() and torch.equal(e[~bad], ec[~bad])
    codes = q.codes_rows().view(64, 2, 16)
    assert (codes[bad] == 0).all() and torch.equal(codes[~bad], c.codes_rows().view(64, 2, 16)[~bad])
    d = U.mxfp4_dequantize(q).view(64, 2, 32)
    assert torch.isnan(d[bad]).all() and torch.isfinite(d[~bad]).all()


@pytest.mark.parametrize("transpose", [False, True])
def test_padding_is_zero(transpose):
    """Rows past the operand's in its last panel, and the scale bytes that fill up the last four blocks."""
    x = _tensor(160, 96, 4) if not transpose else _tensor(96, 160, 4)
    q = U.empty_qtensor(160, 96, U.E2M1_MX32)
    q.codes.fill_(0xEE)
    q.scales.fill_(0xEE)
    U.mxfp4_quantize(x, transpose=transpose, out=q)
    codes = q.codes.view(2, 3, 128, 16)
    assert (codes[1, :, 32:] == 0).all()
    scales = q.scales.view(2, 1, 2, 128, 2)
    assert (scales[1, :, :, 32:] == 0).all() and (scales[:, 0, 1, :, 1] == 0).all()  # block 3 of 3
    assert (scales[0, 0, 0] > 0).all() and (scales[0, 0, 1, :, 0] > 0).all()


@pytest.mark.parametrize("rows,cols", [(1, 32), (96, 160), (257, 544)])
def test_dequantize(rows, cols):
    x = _tensor(rows, cols, 2, spread=True)
    q = U.mxfp4_quantize(x)
    out = torch.full((rows, cols + 24), -7.0, dtype=BF, device="cuda")
    d = U.mxfp4_dequantize(q, out=out[:, :cols])
    want = O.dequantize_mxfp4(*O.quantize_rows_mxfp4(O.bf16_bits_to_f32(bf16_bits(x.cpu())), U.RTNE, False))
    assert np.array_equal(d.double().cpu().numpy(), want) and (out[:, cols:] == -7).all()
    assert torch.equal(U.mxfp4_dequantize(U.mxfp4_quantize(d)), d)  # values on the grid stay


@pytest.mark.parametrize("rows,cols", [(32, 32), (128, 128), (160, 224), (96, 1056), (544, 64), (384, 640)])
@pytest.mark.parametrize("rounding", [U.RTNE, U.SR])
@pytest.mark.parametrize("rht_r,rht_c", [(False, False), (True, False), (False, True), (True, True)])
def test_dual_equals_two_calls(rows, cols, rounding, rht_r, rht_c):
    x = _tensor(rows, cols, rows + 6, pad=16)
    x[3, 5] = float("inf")
    out = [U.empty_qtensor(rows, cols, U.E2M1_MX32), U.empty_qtensor(cols, rows, U.E2M1_MX32)]
    for q in out:
        q.codes.fill_(0xEE)
        q.scales.fill_(0xEE)
    a, b = U.mxfp4_quantize_dual(x, rht_rows=rht_r, sign_mask_rows=0x1234, rht_cols=rht_c, sign_mask_cols=MASK, rounding=rounding,
                                 seed=3, stream_rows=1, stream_cols=2, out_rows=out[0], out_cols=out[1])
    c = U.mxfp4_quantize(x, rht=rht_r, sign_mask=0x1234, rounding=rounding, seed=3, stream_id=1)
    d = U.mxfp4_quantize(x, transpose=True, rht=rht_c, sign_mask=MASK, rounding=rounding, seed=3, stream_id=2)
    for p, q in ((a, c), (b, d)):
        assert torch.equal(p.codes, q.codes) and torch.equal(p.scales, q.scales)  # with their padding
        assert (p.rht_block, p.sign_mask, p.rows, p.red) == (q.rht_block, q.sign_mask, q.rows, q.red)


COUNTS = [[5], [0, 1, 33, 0, 128, 129, 2, 0], [1] * 70, [300, 0, 0, 17], [0, 0, 0]]


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("rht", [False, True])
@pytest.mark.parametrize("rounding", [U.RTNE, U.SR])
@pytest.mark.parametrize("transpose", [False, True])
def test_grouped(counts, rht, rounding, transpose):
    total, cols = sum(counts), 96
    x = _tensor(total, cols, len(counts) + total) if total else torch.empty(0, cols, dtype=BF, device="cuda")
    block = 32 if transpose else 128
    off, padded = U.group_offsets(counts, block=block)
    spare = padded + 2 * block  # a longer bound: the rest is zero
    q = U.mxfp4_quantize_grouped(x, off, spare, transpose=transpose, rht=rht, sign_mask=MASK, rounding=rounding, seed=4)
    a = O.bf16_bits_to_f32(bf16_bits(x.cpu()))
    pads = U.padded_offsets([0] + list(np.cumsum(counts)), block)
    full, ids = np.zeros((spare, cols), np.float32), np.zeros(spare, np.int64)
    at = 0
    for g, c in enumerate(counts):
        full[pads[g] : pads[g] + c] = a[at : at + c]
        ids[pads[g] : pads[g] + c] = np.arange(at, at + c)
        at += c
    if transpose:
        idx, e8 = O.quantize_rows_mxfp4(np.ascontiguousarray(full.T), rounding, rht, MASK, 4, 0)
    else:
        idx, e8 = O.quantize_rows_mxfp4(full, rounding, rht, MASK, 4, 0, row_ids=ids)
    gi, ge = _levels(q)
    assert np.array_equal(ge, e8) and np.array_equal(gi, idx)
    assert q.layout == (U.LAYOUT_GROUPED_RED if transpose else U.LAYOUT_GROUPED_ROWS)


def test_large_leading_offsets():
    """A tensor whose last rows lie past 2^31 elements from its base."""
    rows, cols, ld = 160, 64, 1 << 24
    base = torch.empty((rows - 1) * ld + cols, dtype=BF, device="cuda")
    x = base.as_strided((rows, cols), (ld, 1))
    x.copy_(_tensor(rows, cols, 8))
    for transpose in (False, True):
        a = U.mxfp4_quantize(x, transpose=transpose)
        b = U.mxfp4_quantize(x.contiguous(), transpose=transpose)
        assert torch.equal(a.codes_rows(), b.codes_rows()) and torch.equal(a.scales_rows(), b.scales_rows())


def test_empty_and_refusals():
    for t in (False, True):
        q = U.mxfp4_quantize(torch.empty(0, 64, dtype=BF, device="cuda"), transpose=t)
        assert (q.rows, q.red) == ((64, 0) if t else (0, 64))
        assert U.mxfp4_dequantize(q).numel() == 0
    x = torch.zeros(40, 64, dtype=BF, device="cuda")
    with pytest.raises(U.UFP4Error):
        U.mxfp4_quantize(x, transpose=True)  # 40 rows are no whole blocks
    with pytest.raises(U.UFP4Error):
        U.mxfp4_quantize(x[:, :48])
    with pytest.raises(U.UFP4Error):
        U.mxfp4_quantize(x[:, 4:36])  # 8-byte alignment
    with pytest.raises(U.UFP4Error):
        U.mxfp4_quantize(x, rounding=2)
    with pytest.raises(U.UFP4Error):
        U.mxfp4_quantize(x, sign_mask=1 << 16)
    with pytest.raises(U.UFP4Error):
        U.mxfp4_quantize(x, out=U.empty_qtensor(40, 32, U.E2M1_MX32))
    with pytest.raises(ValueError):
        U.mxfp4_quantize(x.float())
    with pytest.raises(U.UFP4Error):
        U.mxfp4_dequantize(U.mx_quantize(x))
    q = U.mxfp4_quantize(x)
    with pytest.raises(ValueError):
        U.mxfp4_dequantize(q, out=torch.empty(40, 32, dtype=BF, device="cuda"))


def test_large_tensor_and_back():
    """Outputs that no cache holds are stored by a kernel of their own: the same values as from a part of the rows."""
    x = torch.randn(16384 + 96, 8224, device="cuda").to(torch.bfloat16)
    got = U.mxfp4_dequantize(U.mxfp4_quantize(x))
    for a in range(0, x.shape[0], 4096):
        assert torch.equal(got[a : a + 4096], U.mxfp4_dequantize(U.mxfp4_quantize(x[a : a + 4096])))


@pytest.mark.parametrize("rounding", [U.RTNE, U.SR])
@pytest.mark.parametrize("form", ["rows", "transposed", "both", "groups"])
def test_padding_of_a_rotated_operand_is_zero(form, rounding):
    """The signs that turn the zeros of a rotated padding row into negative ones: its codes are zero all the same."""
    kw = dict(rounding=rounding, seed=3)
    x, mask = _tensor(160, 96, 4), 0xFFFF
    rows, cols = (U.empty_qtensor(r, c, U.E2M1_MX32) for r, c in ((256 if form == "groups" else 160, 96), (96, 160)))
    for q in (rows, cols):
        q.codes.fill_(0xEE)
        q.scales.fill_(0xEE)
    pads = {}  # of an operand: its blocks, and where its rows are none of x's
    if form in ("rows", "both"):
        pads[rows] = 3, [(1, slice(32, 128))]
    if form in ("transposed", "both"):
        pads[cols] = 5, [(0, slice(96, 128))]
    if form == "rows":
        U.mxfp4_quantize(x, rht=True, sign_mask=mask, out=rows, **kw)
    elif form == "transposed":
        U.mxfp4_quantize(x, transpose=True, rht=True, sign_mask=mask, out=cols, **kw)
    elif form == "both":
        U.mxfp4_quantize_dual(x, rht_rows=True, sign_mask_rows=mask, rht_cols=True, sign_mask_cols=mask, out_rows=rows, out_cols=cols, **kw)
    else:
        pads[rows] = 3, [(0, slice(100, 128)), (1, slice(60, 128))]
        off, padded = U.group_offsets([100, 60], block=128)
        assert padded == 256
        U.mxfp4_quantize_grouped(x, off, padded, transpose=False, rht=True, sign_mask=mask, out=rows, **kw)
    for q, (nkb, places) in pads.items():
        codes, scales = q.codes.view(q.panels, nkb, 128, 16), q.scales.view(q.panels, -1, 2, 128, 2)
        for p, r in places:
            assert not codes[p, :, r].any() and not scales[p, :, :, r].any()
        assert codes[0, :, :60].any(-1).all()  # and x's own are there
