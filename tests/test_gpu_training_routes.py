"""Which kernels the calls of 8-bit float layers launch, and how many."""
import pytest
import torch

from paper_2512_18453_amd import nova
from tests.launches import launches

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def linear(M, N, K, dtype):
    Wq = torch.zeros(nova.nova_f8_bytes(N, K, 128), dtype=torch.uint8, device=DEV)
    x, y = torch.zeros((M, K), dtype=dtype, device=DEV), torch.empty((M, N), dtype=dtype, device=DEV)
    ws = torch.empty(nova.nova_f8_linear_workspace_bytes(M, N, K, dtype), dtype=torch.uint8, device=DEV)
    return [name for name, _, _ in launches(lambda: nova.nova_f8_linear(x, Wq, N, y=y, workspace=ws))]


# f8_rows_kernel<MT, NT, formats, way, band, x's type (-1: a layout)>; f8_tile_kernel<F8Tile<waves along rows, columns, panels of a wave>, formats, way, band>
@pytest.mark.parametrize("M,N,K,dtype,want", [
    (1, 1000, 4096, F32, ["f8_rows_kernel<1, 1, 0, 0, 1, 1, 0>"]),
    (1, 4096, 25088, F16, ["f8_rows_kernel<1, 1, 0, 0, 0, 1, 1>"]),
    (6, 4096, 4096, BF16, ["f8_rows_kernel<1, 1, 0, 0, 0, 1, 2>"]),
    (7, 4096, 4096, BF16, ["f8_quantize_rows_kernel<2, 0, 0>", "f8_rows_kernel<1, 1, 0, 0, 0, 1, -1>"]),
    (32, 4096, 4096, F16, ["f8_quantize_rows_kernel<1, 0, 0>", "f8_rows_kernel<2, 1, 0, 0, 0, 1, -1>"]),
    (64, 25088, 4096, F16, ["f8_quantize_rows_kernel<1, 0, 0>", "f8_rows_kernel<4, 2, 0, 0, 0, 1, -1>"]),
    (65, 25088, 400, F16, ["f8_quantize_rows_kernel<1, 0, 0>", "f8_tile_kernel<nova::F8Tile<2, 4, 4, 2>, 0, 0, 0, 1>"]),
    (4096, 8192, 8192, BF16, ["f8_quantize_rows_kernel<2, 0, 1>", "f8_tile_kernel<nova::F8Tile<4, 2, 4, 8>, 0, 0, 0, 1>"]),
    (517, 5001, 2055, F32, ["f8_quantize_rows_kernel<0, 0, 0>", "f8_tile_kernel<nova::F8Tile<4, 2, 2, 4>, 0, 0, 1, 1>"]),
    (4096, 8192, 2048, F32, ["f8_quantize_rows_kernel<0, 0, 1>", "f8_tile_kernel<nova::F8Tile<2, 2, 4, 4>, 0, 0, 1, 1>"]),
])
def test_linear(M, N, K, dtype, want):
    assert linear(M, N, K, dtype) == want


@pytest.mark.parametrize("M,dtype,want", [
    (32, F16, ["f8_quantize_backward_kernel<1, 1, 2>", "f8_rows_kernel<2, 2, 1, 0, 0, 1, -1>", "f8_tile_kernel<nova::F8Tile<4, 2, 2, 4>, 1, 0, 1, 0>"]),
    (100, BF16, ["f8_quantize_backward_kernel<2, 1, 8>", "f8_tile_kernel<nova::F8Tile<2, 4, 4, 2>, 1, 0, 0, 1>", "f8_tile_kernel<nova::F8Tile<4, 2, 2, 4>, 1, 0, 1, 0>"]),
])
def test_backward(M, dtype, want):
    N, K = 2048, 16384
    WqT = torch.zeros(nova.nova_f8_bytes(K, N, 128), dtype=torch.uint8, device=DEV)
    dy, x, dx = torch.zeros((M, N), dtype=dtype, device=DEV), torch.zeros((M, K), dtype=dtype, device=DEV), torch.empty((M, K), dtype=dtype, device=DEV)
    dw, db = torch.empty((N, K), device=DEV), torch.empty((N,), device=DEV)
    ws = torch.empty(nova.nova_f8_linear_backward_workspace_bytes(M, N, K, dtype), dtype=torch.uint8, device=DEV)
    assert [name for name, _, _ in launches(lambda: nova.nova_f8_linear_backward(dy, WqT, x, dx=dx, dw=dw, dbias=db, workspace=ws))] == want
