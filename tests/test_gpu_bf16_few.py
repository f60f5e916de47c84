"""Few rows a group on average, unevenly spread: whole numbers, so that every result is exact; and that a routing which gives all rows to one group
is no slower than one that reads every group's weights."""

import ctypes

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
FILL = 12345.0


def _whole(g, *shape):
    return torch.randint(-3, 4, shape, generator=g, device="cuda", dtype=torch.int8).to(BF)


def _few(tokens, N, K, G):
    return U.lib().ufp4_plan_gemm_bf16(0, *(ctypes.c_int64(v) for v in (tokens, N, K)), G, 1) == 0


def _spread(tokens, G, how):
    c = [0] * G
    if how == "first":
        c[0] = tokens
    elif how == "last":
        c[-1] = tokens
    elif how == "two":  # apart by more than 64 groups where there are so many
        c[G // 5] += tokens - tokens // 3
        c[G - 1 - G // 7] += tokens // 3
    elif how == "one each, then the rest":
        for i in range(min(G, tokens)):
            c[i] = 1
        c[G // 2] += tokens - sum(c)
    else:  # blocks of 15, 16, 17, 31, 32, 33, ... rows
        at, left = 0, tokens
        for n in (15, 16, 17, 0, 31, 32, 33, 1, 63, 64, 65) * G:
            if at == G or not left:
                break
            c[at] = min(n, left)
            left -= c[at]
            at += 1
        c[-1] += left
    return c


@pytest.mark.parametrize("how", ["first", "last", "two", "one each, then the rest", "blocks"])
@pytest.mark.parametrize("tokens,G", [(1, 1), (33, 1), (64, 1), (64, 2), (62, 3), (64, 5), (40, 130), (62, 201), (130, 17), (510, 64), (500, 128), (300, 101)])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_uneven_loads(tokens, G, how, dtype):
    g = torch.Generator(device="cuda").manual_seed(tokens + G)
    N, K = (72, 136) if G % 2 else (45, 67)
    counts = _spread(tokens, G, how)
    assert sum(counts) == tokens
    for tail in (0, 2):
        if tail and tokens == 64:  # past the few-row kernel's rows
            continue
        assert _few(tokens + tail, N, K, G)
        x, w = _whole(g, tokens + tail, K), _whole(g, G * N, K)
        if tail:
            x[-tail:] = float("nan")
        offsets, _ = U.group_offsets(counts)
        out = torch.full((tokens + tail, N), FILL, dtype=dtype, device="cuda")
        got = U.bf16_gemm_fwd_y_grouped(x, w, offsets, dtype, out=out)
        ref, at = torch.full((tokens + tail, N), FILL, dtype=torch.float64, device="cuda"), 0
        for e, n in enumerate(counts):
            ref[at : at + n] = x[at : at + n].double() @ w[e * N : (e + 1) * N].double().t()
            at += n
        assert torch.equal(got, ref.to(dtype)), (how, tail)


def _us(call):
    for _ in range(20):
        call()
    best = float("inf")
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(10):
            call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 100)
    return best


@pytest.mark.parametrize("tokens,G,N,K", [(512, 64, 1408, 2048), (1024, 128, 1408, 2048), (8192, 1024, 512, 512)])
def test_one_busy_group_is_no_slower(tokens, G, N, K):
    """All rows in one group read one G-th of the weights that even loads read. (With workgroups that took a group's rows one
    block after the other, it took 2.2 to 4 times as long here.)"""
    x, w = torch.randn(tokens, K, device="cuda").to(BF), torch.randn(G * N, K, device="cuda").to(BF)
    one, even = (U.group_offsets(c)[0] for c in (_spread(tokens, G, "last"), [tokens // G] * G))
    assert _us(lambda: U.bf16_gemm_fwd_y_grouped(x, w, one, BF)) <= 1.25 * _us(lambda: U.bf16_gemm_fwd_y_grouped(x, w, even, BF))
