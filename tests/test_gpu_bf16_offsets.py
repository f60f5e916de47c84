"""Grouped bf16 products whose offsets fall: y and dx as if no offset were below the ones before it, so that every row has one group at most,
whatever kernel takes the product; a weights' gradient sums every group's own rows. Operands are whole numbers, so that every result is
exact."""

import ctypes

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
FILL = 12345.0


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _whole(g, *shape):
    return torch.randint(-3, 4, shape, generator=g, device="cuda", dtype=torch.int8).to(BF)


def _owners(offsets, tokens):
    """The group of each row, -1 for none."""
    owner, cut = torch.full((tokens,), -1, dtype=torch.long), torch.tensor(offsets).clamp(0, tokens).cummax(0).values.tolist()
    for g in range(len(cut) - 1):
        owner[cut[g] : cut[g + 1]] = g
    return owner


def _lists(tokens, groups, seed):
    """Offsets that fall in several ways; most claim more tiles than the rows make."""
    g = torch.Generator().manual_seed(seed)
    wild = torch.randint(-tokens // 4, tokens + tokens // 4 + 1, (groups + 1,), generator=g).tolist()
    part = max(1, tokens - tokens // 5 - 1)
    again = [0 if i % 2 == 0 else part for i in range(groups)] + [tokens]  # the rows behind `part` are the last group's alone
    once = sorted(torch.randint(0, tokens + 1, (groups + 1,), generator=g).tolist())
    once[groups // 2] = 0  # rising but for one
    down = [tokens - i * tokens // groups for i in range(groups + 1)]
    late = [tokens // 3] * (groups // 2) + [tokens] + [0] * (groups // 2 + 1)
    return [wild, again, once, down, late[: groups + 1]]


# kernel of the forward pass and of the input's gradient as ufp4_plan_gemm_bf16 names them; odd widths: the one of any alignment
CASES = [(2, 5, 40, 72, 0, 2), (40, 70, 264, 136, 0, 2), (60, 130, 33, 35, 0, 1), (300, 40, 72, 40, 0, 2), (400, 100, 72, 40, 0, 2), (1000, 130, 33, 35, 1, 1), (1200, 20, 264, 136, 2, 2), (1200, 90, 131, 67, 1, 1),
         (8192, 8, 1408, 2048, 2, 3), (4096, 8, 4096, 2048, 3, 3)]


@pytest.mark.parametrize("tokens,G,N,K,kernel_fwd,kernel_dx", CASES)
def test_falling_offsets(tokens, G, N, K, kernel_fwd, kernel_dx):
    g = _gen(tokens + G)
    x, dy, w = _whole(g, tokens, K), _whole(g, tokens, N), _whole(g, G * N, K)
    wd = w.view(G, N, K).double()
    for p, kernel in ((0, kernel_fwd), (1, kernel_dx)):
        assert U.lib().ufp4_plan_gemm_bf16(p, *(ctypes.c_int64(v) for v in (tokens, N, K)), G, int(N % 8 == 0 and K % 8 == 0)) == kernel
    for off in _lists(tokens, G, tokens):
        assert len(off) == G + 1
        offsets, owner = torch.tensor(off, device="cuda"), _owners(off, tokens)
        for what in ("fwd", "dx"):
            a, wide = (x, N) if what == "fwd" else (dy, K)
            ref = torch.full((tokens, wide), FILL, dtype=torch.float64, device="cuda")
            for e in owner.unique().tolist():
                if e >= 0:
                    rows = (owner == e).nonzero()[:, 0].cuda()
                    ref[rows] = a[rows].double() @ (wd[e].t() if what == "fwd" else wd[e])
            out = torch.full((tokens, wide), FILL, dtype=F32, device="cuda")
            got = (U.bf16_gemm_fwd_y_grouped if what == "fwd" else U.bf16_gemm_bwd_dx_grouped)(a, w, offsets, F32, out=out)
            assert torch.equal(got.double(), ref), (what, off[:8])
        got = U.bf16_gemm_bwd_dw_grouped(dy, x, offsets)
        cut = [min(max(v, 0), tokens) for v in off]
        for e in range(G):
            rows = slice(cut[e], max(cut[e], cut[e + 1]))
            assert torch.equal(got[e].double(), dy[rows].double().t() @ x[rows].double()), ("dw", off[:8])


def test_a_row_of_one_late_group():
    """Two rows, of which the second is the last group's alone: more groups claim rows than there are rows."""
    g = _gen(1)
    x, w = _whole(g, 2, 64), _whole(g, 5 * 48, 64)
    got = U.bf16_gemm_fwd_y_grouped(x, w, torch.tensor([0, 1, 0, 1, 0, 2], device="cuda"))
    wd = w.view(5, 48, 64).double()
    assert torch.equal(got.double(), torch.stack([x[0].double() @ wd[0].t(), x[1].double() @ wd[4].t()]))
