"""Grouped bf16 products whose workgroups take their tiles as they get done, and whose results are stored nontemporally: what a training
micro-batch runs. Each case says which kernel it means, and the library's rules are held to that.

Operands are whole numbers of -3 .. 3 (a checkpoint in 8 bits keeps those as they are), every partial sum is below 2^24: fp32 results have to
equal the product in 64 bits, bf16 ones that rounded once.
"""

import ctypes

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
PASS = {"fwd": 0, "dx": 1, "dw": 2, "dw8": 2}
FILL = 12345.0


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _whole(g, *shape):
    return torch.randint(-3, 4, shape, generator=g, device="cuda", dtype=torch.int8).to(BF)


def _path(what, tokens, N, K, G, dtype):
    """(tile, whether workgroups take tiles from counters, whether results are stored nontemporally) of a product of whole pieces."""
    n = ctypes.c_size_t()
    assert U.lib().ufp4_bf16_gemm_grouped_workspace(PASS[what], tokens, N, K, G, ctypes.byref(n)) == 0
    sizes = (PASS[what], *(ctypes.c_int64(v) for v in (tokens, N, K)), G)
    tile = {2: 128, 3: 256}[U.lib().ufp4_plan_gemm_bf16(*sizes, 1)]
    return tile, n.value > 0, bool(U.lib().ufp4_plan_gemm_bf16_streams(*sizes, U.OUT_BF16 if dtype == BF else U.OUT_F32))


def _run(what, x, dy, w, offsets, dtype, out=None):
    if what == "fwd":
        return U.bf16_gemm_fwd_y_grouped(x, w, offsets, dtype, out=out)
    if what == "dx":
        return U.bf16_gemm_bwd_dx_grouped(dy, w, offsets, dtype, out=out)
    return U.bf16_gemm_bwd_dw_grouped(dy, U.checkpoint8_save(x) if what == "dw8" else x, offsets, dtype, out=out)


def _check(got, what, x, dy, w, offsets, N):
    """Every element, group by group; rows in no group hold FILL."""
    ends = offsets.tolist()
    for e, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
        we = None if w is None else w[e * N : (e + 1) * N].double()
        if what == "fwd":
            part, ref = got[a:b], x[a:b].double() @ we.t()
        elif what == "dx":
            part, ref = got[a:b], dy[a:b].double() @ we
        else:
            part, ref = got[e], dy[a:b].double().t() @ x[a:b].double()
        assert torch.equal(part, ref.to(got.dtype)), e
    if what in ("fwd", "dx"):
        assert bool((got[ends[-1] :] == FILL).all())


def _ragged(total, g):
    """Loads of `total` rows: long and short groups, some empty, sizes that no tile divides."""
    share = torch.rand(23, generator=g, device="cuda") ** 3
    counts = (share / share.sum() * total).int().tolist()
    return [0, 1] + counts + [255, 0, 257, 0]


# (rows, columns of the result, reduction, tile, nontemporal for bf16, for fp32): a reduction of few stages, of many, and of no whole ones
ROWS = [(70_000, 2056, 72, 256, True, True), (70_000, 2056, 264, 256, True, True), (70_000, 1928, 520, 256, True, True),
        (40_000, 2056, 264, 256, False, True), (272_000, 120, 264, 128, False, False), (272_000, 128, 72, 128, False, False)]


@pytest.mark.parametrize("what", ["fwd", "dx"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,wide,red,tile,stream_bf,stream_f32", ROWS)
def test_rows_products(what, dtype, rows, wide, red, tile, stream_bf, stream_f32):
    g = _gen(rows + wide + red)
    counts = _ragged(rows, g)
    offsets, _ = U.group_offsets(counts)
    tokens, G = sum(counts) + 3, len(counts)
    N, K = (wide, red) if what == "fwd" else (red, wide)
    assert _path(what, tokens, N, K, G, dtype) == (tile, True, stream_bf if dtype == BF else stream_f32)
    a, w = _whole(g, tokens, red), _whole(g, G * N, K)
    a[-3:] = float("nan")
    for _ in range(2):  # the order of taking is not fixed
        out = torch.full((tokens, wide), FILL, dtype=dtype, device="cuda")
        _check(_run(what, a, a, w, offsets, dtype, out), what, a, a, w, offsets, N)


@pytest.mark.parametrize("what", ["dw", "dw8"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,N,K,tile,stream_bf,stream_f32", [(24_000, 1416, 2056, 256, True, True), (24_000, 776, 1032, 256, False, True),
                                                                (9_000, 392, 520, 128, False, False)])
def test_weight_gradients(what, dtype, rows, N, K, tile, stream_bf, stream_f32):
    g = _gen(rows + N)
    counts = _ragged(rows, g)
    offsets, _ = U.group_offsets(counts)
    tokens, G = sum(counts) + 3, len(counts)
    assert _path(what, tokens, N, K, G, dtype) == (tile, True, stream_bf if dtype == BF else stream_f32)
    x, dy = _whole(g, tokens, K), _whole(g, tokens, N)
    x[-3:], dy[-3:] = float("nan"), float("nan")
    for _ in range(2):
        _check(_run(what, x, dy, None, offsets, dtype), what, x, dy, None, offsets, N)


# (what, rows, N, K): products that take a workspace, small enough to be run many times
COUNTED = [("fwd", 272_000, 120, 72), ("dx", 272_000, 72, 120), ("dw", 9_000, 392, 520), ("dw8", 9_000, 392, 520)]


def _job(what, rows, N, K, seed):
    g = _gen(seed)
    counts = _ragged(rows, g)
    offsets, _ = U.group_offsets(counts)
    tokens, G = offsets[-1].item(), len(counts)
    assert _path(what, tokens, N, K, G, F32)[1]
    return {"what": what, "x": None if what == "dx" else _whole(g, tokens, K), "dy": None if what == "fwd" else _whole(g, tokens, N),
            "w": _whole(g, G * N, K) if what in ("fwd", "dx") else None, "offsets": offsets, "N": N}


def _go(j):
    return _run(j["what"], j["x"], j["dy"], j["w"], j["offsets"], F32)


def _right(got, j):
    _check(got, j["what"], j["x"], j["dy"], j["w"], j["offsets"], j["N"])


def test_at_once_on_two_streams():
    """Calls in flight together, each with counters of its own."""
    jobs = [_job(*c, seed) for seed, c in enumerate(COUNTED)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for n in range(8):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[k].append(_go(jobs[(n + 2 * k) % 4]))
    torch.cuda.synchronize()
    for k in range(2):
        for n, got in enumerate(outs[k]):
            _right(got, jobs[(n + 2 * k) % 4])


def test_graphs_with_counters():
    """Captured, then replayed with new contents and loads, eager calls of the same kind in between; then two graphs at the same time."""
    graphs = []
    for first in (0, 2):
        jobs = [_job(*c, 10 + seed) for seed, c in enumerate(COUNTED[first : first + 2])]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for j in jobs:
                _go(j)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = [_go(j) for j in jobs]
        graphs.append((graph, jobs, got))

    def renew(jobs, seed):
        g = _gen(seed)
        for j in jobs:
            for n in ("x", "dy", "w"):
                if j[n] is not None:
                    j[n].copy_(_whole(g, *j[n].shape))
            last = j["offsets"][-1]
            cuts = (torch.rand(len(j["offsets"]) - 2, generator=g, device="cuda") * last).long().sort().values
            j["offsets"][1:-1] = cuts

    for seed in range(3):
        for graph, jobs, got in graphs:
            renew(jobs, 50 + seed)
            graph.replay()
            eager = [_go(j) for j in jobs]
            torch.cuda.synchronize()
            for j, c, e in zip(jobs, got, eager):
                assert torch.equal(c, e)
                _right(c, j)
    for seed in range(3):
        for _, jobs, got in graphs:
            renew(jobs, 90 + seed)
            for c in got:
                c.fill_(FILL)
        torch.cuda.synchronize()
        for graph, _, _ in graphs:
            with torch.cuda.stream(torch.cuda.Stream()):
                graph.replay()
        torch.cuda.synchronize()
        for _, jobs, got in graphs:
            for j, c in zip(jobs, got):
                _right(c, j)
