"""Grouped products of bf16 rows (ufp4_bf16_gemm_*_grouped) against the same products in 64 bits.

Whole numbers: operands of -3 .. 3, so that every partial sum is below 2^24 and exact in fp32 in any order; fp32 results have to be
equal, bf16 ones the sum rounded once. Real numbers: the products of two bf16 numbers are exact in fp32; each of the R additions of a sum
is off by at most 2^-23 of the sum of magnitudes (2^-24 a rounding, as much again for what the matrix unit cuts when it aligns terms),
and the result's own rounding by 2^-24 or (bf16) 2^-8 of it.
"""

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
FILL = 12345.0  # what output rows outside the groups hold before and after


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _whole(g, *shape):
    return torch.randint(-3, 4, shape, generator=g, device="cuda").to(BF)


def _view(t, pad, at):
    """t's values at column `at` of a tensor `pad` columns wider, NaN around them."""
    if not pad:
        return t
    wide = torch.full((t.shape[0] + 1, t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[: t.shape[0], at : at + t.shape[1]] = t
    return wide[: t.shape[0], at : at + t.shape[1]]


def _spans(offsets, tokens):
    off = [min(max(int(v), 0), tokens) for v in offsets.tolist()]
    return [(a, max(a, b)) for a, b in zip(off[:-1], off[1:])]


def _reference(what, x, dy, w, offsets, tokens, N, K):
    """(result, sums of magnitudes) in 64 bits; rows in no group hold FILL."""
    outs = []
    for f in (lambda t: t.double(), lambda t: t.double().abs()):
        spans = _spans(offsets, tokens)
        if what in ("dw", "dw8"):
            r = torch.zeros(len(spans), N, K, dtype=torch.float64, device="cuda")
        else:
            r = torch.full((tokens, N if what == "fwd" else K), FILL, dtype=torch.float64, device="cuda")
        for e, (a, b) in enumerate(spans):
            if what == "fwd" and b > a:
                r[a:b] = f(x[a:b]) @ f(w[e * N : (e + 1) * N]).t()
            elif what == "dx" and b > a:
                r[a:b] = f(dy[a:b]) @ f(w[e * N : (e + 1) * N])
            elif what in ("dw", "dw8"):
                r[e] = f(dy[a:b]).t() @ f(x[a:b])
        outs.append(r)
    return outs


def _call(what, x, dy, w, offsets, out, dtype):
    if what == "fwd":
        return U.bf16_gemm_fwd_y_grouped(x, w, offsets, dtype, out=out)
    if what == "dx":
        return U.bf16_gemm_bwd_dx_grouped(dy, w, offsets, dtype, out=out)
    if what == "dw8":  # whole numbers to 15 are kept as they are
        return U.bf16_gemm_bwd_dw_grouped(dy, U.checkpoint8_save(x), offsets, dtype, out=out)
    return U.bf16_gemm_bwd_dw_grouped(dy, x, offsets, dtype, out=out)


def _out(what, tokens, N, K, G, dtype, pad=0):
    if what in ("dw", "dw8"):
        return torch.full((G, N, K + pad), FILL, dtype=dtype, device="cuda")[:, :, :K]
    cols = N if what == "fwd" else K
    return torch.full((tokens, cols + pad), FILL, dtype=dtype, device="cuda")[:, :cols]


COUNTS = [
    [1], [0], [0, 0, 5], [3, 0, 1, 0], [17, 128, 0, 1, 255, 16], [300], [129, 127, 257, 256, 1, 64], [31, 33, 32, 0, 95, 7],
    [2] * 70 + [0] * 3 + [40],
]
SIZES = [(1, 1), (8, 8), (7, 9), (64, 64), (129, 40), (40, 129), (256, 320), (257, 65), (520, 96), (96, 520), (131, 259)]


@pytest.mark.parametrize("what", ["fwd", "dx", "dw", "dw8"])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{max(c)}")
def test_whole_numbers(what, dtype, counts):
    g = _gen(len(counts) * 1000 + max(counts))
    offsets, _ = U.group_offsets(counts)
    G = len(counts)
    for tail in (0, 3):  # rows behind the last group
        tokens = sum(counts) + tail
        for n, (N, K) in enumerate(SIZES):
            x, dy, w = _whole(g, tokens, K), _whole(g, tokens, N), _whole(g, G * N, K)
            if tail:
                x[-tail:], dy[-tail:] = float("nan"), float("nan")
            ref, _ = _reference(what, x, dy, w, offsets, tokens, N, K)
            pad, at = ((0, 0), (8, 8), (5, 3))[n % 3]  # whole rows, rows of 16-byte pieces, rows that start anywhere
            got = _call(what, _view(x, pad, at), _view(dy, pad, at), _view(w, pad, at), offsets, _out(what, tokens, N, K, G, dtype, pad), dtype)
            assert torch.equal(got, ref.to(dtype)), (N, K, tail)


@pytest.mark.parametrize("what", ["fwd", "dx", "dw"])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("counts,N,K", [([700, 0, 1, 333], 384, 640), ([5, 4, 3, 2, 1], 1408, 2048), ([1000, 24], 515, 771),
                                        ([4096], 1024, 512), ([8], 4096, 24), ([0, 2500], 64, 4104)])
def test_real_numbers(what, dtype, counts, N, K):
    g = _gen(N)
    tokens, G = sum(counts), len(counts)
    offsets, _ = U.group_offsets(counts)
    x = (torch.randn(tokens, K, generator=g, device="cuda") + 0.25).to(BF)
    dy = (torch.randn(tokens, N, generator=g, device="cuda") * 1e-3).to(BF)
    w = (torch.randn(G * N, K, generator=g, device="cuda") * 0.02).to(BF)
    ref, size = _reference(what, x, dy, w, offsets, tokens, N, K)
    got = _call(what, x, dy, w, offsets, None, dtype)
    R = {"fwd": K, "dx": N, "dw": max(counts)}[what]
    tol = R * 2.0**-23 * size + (2.0**-8 if dtype == BF else 2.0**-24) * ref.abs()
    assert got.dtype == dtype and bool(((got.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("what", ["fwd", "dx", "dw", "dw8"])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("counts,N,K", [([4000, 10, 3500, 0, 900, 1], 2568, 2056), ([300] * 40, 1032, 776), ([1, 20000], 640, 1024),
                                        ([130] * 70 + [5000], 392, 1288), ([66, 65, 2, 700] * 25, 1160, 904)])
def test_more_tiles_than_workgroups(what, dtype, counts, N, K):
    """Tiles that workgroups take as they get done, long and short ones, in whole numbers; twice, since the order of taking is not fixed."""
    g = _gen(N + K)
    tokens, G = sum(counts) + 5, len(counts)
    offsets, _ = U.group_offsets(counts)
    x, dy, w = _whole(g, tokens, K), _whole(g, tokens, N), _whole(g, G * N, K)
    ref, _ = _reference(what, x, dy, w, offsets, tokens, N, K)
    for _ in range(2):
        assert torch.equal(_call(what, x, dy, w, offsets, _out(what, tokens, N, K, G, dtype), dtype), ref.to(dtype))


@pytest.mark.parametrize("what", ["fwd", "dx", "dw", "dw8"])
@pytest.mark.parametrize("N,K", [(264, 72), (33, 35)])
def test_offsets_that_lie(what, N, K):
    """Offsets past the rows, below zero or falling: cut to the rows; a group that ends before it starts has none."""
    g = _gen(3)
    tokens = 200
    x, dy, w = _whole(g, tokens, K), _whole(g, tokens, N), _whole(g, 4 * N, K)
    for off in ([-5, 20, 90, 150, 10**12], [0, 150, 150, 100, 200], [0, 0, 0, 0, 0], [300, 400, 500, 600, 700], [200, 120, 60, 10, 0]):
        offsets = torch.tensor(off, device="cuda")
        ref, _ = _reference(what, x, dy, w, offsets, tokens, N, K)
        got = _call(what, x, dy, w, offsets, _out(what, tokens, N, K, 4, F32), F32)
        if off[3] == 100:  # the last two groups claim the rows 100 .. 149 of the second again: any of them may have written those
            if what in ("fwd", "dx"):
                got[100:150] = ref[100:150]
        assert torch.equal(got.double(), ref), off


@pytest.mark.parametrize("what", ["fwd", "dx", "dw"])
def test_infinities_and_nan_stay_in_their_rows(what):
    g = _gen(4)
    counts, N, K = [70, 1, 59], 136, 72
    offsets, _ = U.group_offsets(counts)
    tokens = sum(counts)
    x, dy, w = _whole(g, tokens, K), _whole(g, tokens, N), _whole(g, 3 * N, K)
    clean, _ = _reference(what, x, dy, w, offsets, tokens, N, K)
    x[70], dy[70], w[N : 2 * N] = float("nan"), float("inf"), float("nan")  # the middle group's
    got = _call(what, x, dy, w, offsets, None, F32).double()
    if what == "dw":
        assert torch.equal(got[[0, 2]], clean[[0, 2]]) and bool(got[1].isnan().all())
    else:
        rest = [i for i in range(tokens) if i != 70]
        assert torch.equal(got[rest], clean[rest]) and bool(got[70].isnan().all())


@pytest.mark.parametrize("what", ["fwd", "dx", "dw"])
def test_nothing_to_do(what):
    offsets = torch.zeros(3, dtype=torch.int64, device="cuda")
    for tokens, N, K in ((0, 16, 24), (4, 0, 8), (4, 8, 0)):
        x, dy, w = (torch.ones(s, dtype=BF, device="cuda") for s in ((tokens, K), (tokens, N), (2 * N, K)))
        got = _call(what, x, dy, w, offsets, None, F32)
        assert tuple(got.shape) == {"fwd": (tokens, N), "dx": (tokens, K), "dw": (2, N, K)}[what]
        if what == "dw":
            assert not got.any()
    # a reduction of length zero is a sum of nothing
    some = torch.tensor([0, 1, 4], device="cuda")
    if what == "fwd":
        got = U.bf16_gemm_fwd_y_grouped(torch.ones(4, 0, dtype=BF, device="cuda"), torch.ones(16, 0, dtype=BF, device="cuda"), some)
        assert tuple(got.shape) == (4, 8) and not got.any()


@pytest.mark.parametrize("what", ["fwd", "dx", "dw", "dw8"])
def test_rows_past_32_bits(what):
    """Tensors of more than 2^32 bytes: the last group's rows lie behind them."""
    g = _gen(5)
    tokens, N, K = 2_200_000, 8, 1024
    if what == "dx":
        N, K = K, N
    x = torch.zeros(tokens, K, dtype=BF, device="cuda")
    dy = torch.zeros(tokens, N, dtype=BF, device="cuda")
    x[-300:], dy[-300:] = _whole(g, 300, K), _whole(g, 300, N)
    w = _whole(g, 2 * N, K)
    offsets = torch.tensor([tokens - 300, tokens - 129, tokens], device="cuda")
    got = _call(what, x, dy, w, offsets, None, F32)
    ref, _ = _reference(what, x[-300:], dy[-300:], w, offsets - (tokens - 300), 300, N, K)
    assert torch.equal(got.double() if what in ("dw", "dw8") else got[-300:].double(), ref)


@pytest.mark.parametrize("K", [40, 512, 1411])
@pytest.mark.parametrize("counts", [[33, 0, 100, 3], [513, 1024]])
def test_weight_gradient_from_a_checkpoint(K, counts):
    g = _gen(K)
    N, tokens = 264, sum(counts) + 2
    offsets, _ = U.group_offsets(counts)
    x = torch.randn(tokens, K, generator=g, device="cuda").to(BF)
    dy = (torch.randn(tokens, N, generator=g, device="cuda") * 1e-3).to(BF)
    x[-2:], dy[-2:] = float("nan"), float("nan")
    kept = U.checkpoint8_save(x)
    ref, size = _reference("dw", U.checkpoint8_load(kept), dy, None, offsets, tokens, N, K)
    for dtype in (F32, BF):
        got = U.bf16_gemm_bwd_dw_grouped(dy, kept, offsets, dtype)
        tol = max(counts) * 2.0**-23 * size + (2.0**-8 if dtype == BF else 2.0**-24) * ref.abs()
        assert bool(((got.double() - ref).abs() <= tol).all())
    # a checkpoint inside a wider one: rows further apart, columns from a block on
    if K > 64:
        for c in (32, 128):  # scales that lie anywhere, and in words of four
            part = U.Checkpoint8(kept.codes[:, c:], kept.scales[:, c // 32 : -(-K // 32)], K - c)
            got = U.bf16_gemm_bwd_dw_grouped(dy, part, offsets)
            tol = max(counts) * 2.0**-23 * size + 2.0**-24 * ref.abs()
            assert bool(((got.double() - ref[:, :, c:]).abs() <= tol[:, :, c:]).all())


def test_streams_and_graph():
    """The three products on another stream, and captured: replays with new contents equal eager calls."""
    g = _gen(6)
    counts, N, K = [130, 0, 77, 300], 264, 136
    offsets, _ = U.group_offsets(counts)
    tokens = sum(counts)
    x, dy, w = _whole(g, tokens, K), _whole(g, tokens, N), _whole(g, 4 * N, K)

    def step():
        kept = U.checkpoint8_save(x)
        return [_call(p, x, dy, w, offsets, None, F32) for p in ("fwd", "dx", "dw")] + [U.bf16_gemm_bwd_dw_grouped(dy, kept, offsets)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = step()
    side.synchronize()
    for p, o in zip(("fwd", "dx", "dw", "dw"), outs):
        assert torch.equal(o.double(), _reference(p, x, dy, w, offsets, tokens, N, K)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in range(3):
        h = _gen(100 + seed)
        x.copy_(_whole(h, tokens, K)), dy.copy_(_whole(h, tokens, N)), w.copy_(_whole(h, 4 * N, K))
        cut = torch.randint(0, tokens + 1, (3,), generator=h, device="cuda").sort().values
        offsets[1:4] = cut
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        for p, c, e in zip(("fwd", "dx", "dw", "dw"), captured, eager):
            assert torch.equal(c, e) and torch.equal(c.double(), _reference(p, x, dy, w, offsets, tokens, N, K)[0])


@pytest.mark.parametrize("counts,N,K", [([37, 0, 300, 5], 136, 72), ([9, 8], 33, 515), ([600, 500], 384, 1032)])
def test_adjoint(counts, N, K):
    """<dy, x w^T> = <dx, x> = <dw, w>, in whole numbers exactly."""
    g = _gen(7)
    tokens, G = sum(counts), len(counts)
    offsets, _ = U.group_offsets(counts)
    x, dy, w = _whole(g, tokens, K), _whole(g, tokens, N), _whole(g, G * N, K)
    y, dx, dw = (_call(p, x, dy, w, offsets, None, F32).double() for p in ("fwd", "dx", "dw"))
    a = (dy.double() * y).sum()
    assert a == (dx * x.double()).sum() and a == (dw.view(G * N, K) * w.double()).sum()
