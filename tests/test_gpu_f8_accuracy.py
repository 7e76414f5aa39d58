"""What the sums of products in 8-bit floating point lose: up to 64 rows nothing but binary32's roundings, whatever the results' type."""
import pytest
import torch

from paper_2512_18453_amd import nova
from tests import plain_training as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF_STEP = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}


def loud_and_quiet(rows, K, loud, quiet, seed):
    """In every eight neighbours one loud number, its sign another in the next eight, and seven quiet ones; rows differ by their sign and by a power of two."""
    k = torch.arange(K)
    v = torch.where(k % 8 == 3, loud, quiet).repeat(rows, 1)
    gen = torch.Generator().manual_seed(seed)
    return v * (2.0 ** torch.randint(0, 3, (rows, 1), generator=gen)) * (torch.randint(0, 2, (rows, 1), generator=gen) * 2 - 1)


def near(got, want, bound, dtype):
    over = ((got.double().cpu() - want).abs() - bound - HALF_STEP[dtype] * (want.abs() + bound)).max().item()
    assert over <= 0, over


@pytest.mark.parametrize("M,N,K", [(1, 40, 512), (5, 300, 256), (16, 40, 2048), (17, 40, 512), (32, 100, 1152), (33, 40, 512), (64, 130, 640)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_quiet_products_beside_loud_ones(M, N, K, dtype):
    """Loud products cancel; what is left are quiet ones of less than 2^-14 of them, which a sum that is held relative to the loudest of eight would lose whole: 0 where the
    sum is 7/32 K (times the row's and the column's power of two).  The bound, binary32's roundings of the loud ones, is a fifteenth of that."""
    x = loud_and_quiet(M, K, 112.0, 0.0625, 1)                   # (every number a code times its row's scale of 1/4, 1/2 or 1)
    alternate = 1 - 2 * (torch.arange(K) // 8 % 2).float()
    w = torch.where(torch.arange(K) % 8 == 3, 64.0 * alternate, 4.0).repeat(N, 1) * 2.0 ** -(torch.arange(N) % 3).float().unsqueeze(1)
    codes = w.to(torch.float8_e4m3fn)
    assert torch.equal(codes.float(), w)
    scales = torch.ones((-(-N // 128), K // 128))
    want, bound = plain.product(x.double(), w.double())
    assert (want.abs() > 10 * bound).all()
    near(nova.nova_f8_linear(x.to(dtype).to(DEV), nova.nova_f8_pack(codes.to(DEV), scales.to(DEV), 128), N), want, bound, dtype)
    Aq = nova.nova_f8_quantize(x.to(DEV), 1)
    near(nova.nova_f8_matmul(Aq, nova.nova_f8_pack(codes.to(DEV), scales.repeat_interleave(128, 0)[:N].contiguous().to(DEV), 1), M, N, K, block_b=1, dtype=dtype), want, bound, dtype)
    # the gradient of the input is the same product, by the layout of the transpose
    dx = nova.nova_f8_linear_backward(x.to(dtype).to(DEV), nova.nova_f8_pack(codes.T.contiguous().to(DEV), scales.T.contiguous().to(DEV), 128, transposed=True), None, K=N,
                                      format=nova.NOVA_F8_E4M3, need_dbias=False)[0]
    near(dx, want, bound, dtype)
