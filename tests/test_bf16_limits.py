"""Sizes at the documented limits of the grouped bf16 products: what the header allows is taken. On the host, and one of them on the GPU. And narrow
weights of many groups: the kernel that fits them."""

import ctypes
import os

import pytest
import torch

from paper_2606_20381_amd import ufp4 as U

OK, UNSUPPORTED = 0, 5


@pytest.fixture(autouse=True)
def built():
    if not os.path.exists(U.library_path()):
        pytest.skip("libufp4.so not built")


def _workspace(p, tokens, N, K, G):
    return U.lib().ufp4_bf16_gemm_grouped_workspace(p, tokens, N, K, G, ctypes.byref(ctypes.c_size_t()))


def _tiles(tokens, N, G):
    return (-(-tokens // 128) + G) * -(-N // 128)


@pytest.mark.parametrize("tokens,N,G", [(1, 1 << 28, 1), (64, 1 << 29, 1), (1, 1 << 18, 1024), (8192, 1 << 18, 1024), (7, 1 << 25, 30), (512, 1 << 22, 64)])
def test_few_rows_of_wide_weights(tokens, N, G):
    """Fewer than 2^23 tiles of 128 x 128: taken, with however few rows."""
    assert (_workspace(0, tokens, N, 8, G) == OK) == (_tiles(tokens, N, G) < 1 << 23)
    assert _workspace(0, tokens, 1 << 30, 8, 1024) == UNSUPPORTED


# (rows of a group, N, K, groups, us of tiles of 128 x 128 and of 256 x 256 on an MI355X)
NARROW = [(32, 64, 64, 1024, 95, 194), (128, 64, 64, 1024, 106, 219), (256, 64, 4096, 64, 45, 60), (64, 128, 256, 1024, 204, 205)]


@pytest.mark.parametrize("rows,N,K,G,small,large", NARROW)
def test_many_narrow_weight_gradients(rows, N, K, G, small, large):
    """As for fewer groups, the tile that covers less outside of the results."""
    assert small < large
    for groups in (G, G - 1):
        assert U.lib().ufp4_plan_gemm_bf16(2, *(ctypes.c_int64(v) for v in (rows * groups, N, K)), groups, 1) == 2
    for wide in ((98304, 1408, 2048, 64), (32768, 1416, 2056, 64), (65536, 136, 264, 1024)):  # tiles that hardly cover more
        assert U.lib().ufp4_plan_gemm_bf16(2, *(ctypes.c_int64(v) for v in wide[:3]), wide[3], 1) == 3


def test_activation_of_as_many_threads_as_a_grid_holds():
    """A lane takes 4 fp32 values of a block of 32: workgroups of 256 lanes that would make 2^32 of them are refused before the launch."""
    rows, cols, p = (1 << 29) - 1, 32, 1 << 20
    assert U.lib().ufp4_activation(0, U.OUT_F32, p, rows, cols, cols, p, cols, None, 0, None, 0, None) == UNSUPPORTED
    assert U.lib().ufp4_activation_bwd(0, U.OUT_F32, p, rows, cols, cols, p, cols, None, 0, None, 0, p, cols, None, 0, None) == UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,N,K,G", [(2, 1 << 28, 1, 1), (3, (1 << 27) + 40, 8, 3)])
def test_few_rows_of_wide_weights_run(tokens, N, K, G):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-3, 4, (tokens, K), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    w = torch.randint(-3, 4, (G * N, K), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    offsets = torch.tensor([0] * G + [tokens], device="cuda")
    got = U.bf16_gemm_fwd_y_grouped(x, w, offsets, torch.bfloat16)
    for n in range(0, N, 1 << 24):
        part = slice((G - 1) * N + n, (G - 1) * N + min(N, n + (1 << 24)))
        assert torch.equal(got[:, n : n + (1 << 24)], (x.float() @ w[part].float().t()).bfloat16()), n
