"""Outputs of one row, whose row stride is of no account, and of groups of one row each, which lie as far apart as their rows."""

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _whole(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda").to(BF)


@pytest.mark.parametrize("cols", [48, 40])
def test_one_row(cols):
    x, w, off = _whole(1, 1, 64), _whole(2, 2 * cols, 64), torch.tensor([0, 0, 1], device="cuda")
    for out in (torch.zeros(cols, 1, device="cuda").t(), torch.zeros(3, cols, device="cuda").as_strided((1, cols), (7, 1))):
        assert U.bf16_gemm_fwd_y_grouped(x, w, off, out=out) is not None
        assert torch.equal(out.double(), x.double() @ w[cols:].double().t())
    dy, out = _whole(3, 1, cols), torch.zeros(64, 1, device="cuda").t()
    U.bf16_gemm_bwd_dx_grouped(dy, w, off, out=out)
    assert torch.equal(out.double(), dy.double() @ w[cols:].double())
    out = torch.zeros(64, 1, dtype=BF, device="cuda").t()
    U.checkpoint8_load(U.checkpoint8_save(x), out=out)
    assert torch.equal(out, x)


def test_groups_of_one_row():
    dy, x, off = _whole(4, 50, 1), _whole(5, 50, 72), torch.tensor([0, 20, 20, 50], device="cuda")
    wide = torch.full((3, 80), 7.0, device="cuda")
    U.bf16_gemm_bwd_dw_grouped(dy, x, off, out=wide[:, :72].unsqueeze(1))
    for e, (a, b) in enumerate(((0, 20), (20, 20), (20, 50))):
        assert torch.equal(wide[e, :72].double(), (dy[a:b].double().t() @ x[a:b].double())[0])
    assert bool((wide[:, 72:] == 7.0).all())


def test_one_token_in_4_bits():
    x, w = _whole(6, 1, 128), _whole(7, 256, 128)
    q = U.mxfp4_quantize(w)
    out = torch.zeros(256, 1, device="cuda").t()
    U.mxfp4_linear(x, q, torch.float32, out=out)
    assert torch.equal(out, U.mxfp4_linear(x, q, torch.float32))
    out = torch.zeros(256, 1, device="cuda").t()
    U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x), q, torch.float32, out=out)
    assert torch.equal(out, U.mxfp4_gemm_fwd_y(U.mxfp4_quantize(x), q, torch.float32))
