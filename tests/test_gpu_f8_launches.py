"""Products in 8-bit floating point of so many rows that they take two launches: 2^29 rows and some, 66 GB of layout."""
import pytest
import torch

from paper_2512_18453_amd import nova
from tests.launches import launches

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16 = torch.float32, torch.float16
LAUNCH = 2 ** 29                                                 # rows of 128 x 128 tiles, one across: 2^22 workgroups
PERIOD = 1000003


@pytest.fixture(autouse=True)
def give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def rows_of_one(M, dtype):
    base = torch.randn((PERIOD, 1), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(dtype)
    return base, base.repeat(-(-M // PERIOD), 1)[:M]


@pytest.mark.parametrize("dtype", [F16, F32])
def test_layer_of_two_launches(dtype):
    """Rows repeat with a period that divides nothing, so every row is compared; sums of one product are the same in every way of cutting."""
    M, N = LAUNCH + 17, 2
    base, x = rows_of_one(M, dtype)
    Wq = nova.nova_f8_quantize(torch.tensor([[1.5], [-0.3]], device=DEV), 128)
    y, want = torch.empty((M, N), dtype=dtype, device=DEV), nova.nova_f8_linear(base, Wq, N)
    workspace = torch.empty(nova.nova_f8_linear_workspace_bytes(M, N, 1, dtype), dtype=torch.uint8, device=DEV)

    def layer():
        nova.nova_f8_linear(x, Wq, N, y=y, workspace=workspace)
    names = [name for name, _, _ in launches(layer)]
    assert sum("f8_tile_kernel" in name for name in names) == 2, names
    layer()
    for row in range(0, M, PERIOD):
        assert torch.equal(y[row:row + PERIOD], want[:min(PERIOD, M - row)]), row


def test_product_of_two_launches_with_a_scale_for_128_rows():
    M, N = LAUNCH + 257, 2
    _, x = rows_of_one(M, F16)
    Bq = nova.nova_f8_quantize(torch.tensor([[1.5], [-0.3]], device=DEV), 1)
    out = nova.nova_f8_matmul(nova.nova_f8_quantize(x, 128), Bq, M, N, 1, block_a=128, block_b=1, dtype=F32)
    for first in (0, LAUNCH - 256, LAUNCH):
        some = x[first:first + 640]
        want = nova.nova_f8_matmul(nova.nova_f8_quantize(some, 128), Bq, len(some), N, 1, block_a=128, block_b=1, dtype=F32)
        assert torch.equal(out[first:first + 640], want), first
