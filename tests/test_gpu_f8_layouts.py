"""Layouts of a transpose with a scale per row, which the weights' gradient sums along: every byte, padding included, against packing the plain form's codes."""
import pytest
import torch

from paper_2512_18453_amd import nova
from tests import plain_training as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


# up to 32 rows a thread takes two of them and three quarters of each panel are padding; 8 MB and more go past the caches
@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (2, 130), (5, 7), (16, 128), (17, 129), (31, 300), (32, 16), (33, 17), (128, 1), (129, 8), (130, 300), (300, 2055), (2051, 4101)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_every_byte_of_a_transposed_layout(shape, dtype):
    x = (torch.randn(shape, generator=torch.Generator().manual_seed(sum(shape))) * torch.logspace(-3, 3, shape[1])).to(dtype)
    x[shape[0] // 2] = 0
    for format in (nova.NOVA_F8_E4M3, nova.NOVA_F8_E5M2):
        codes, scales = plain.quantized(x.T, format, 1)
        Xq = torch.full((nova.nova_f8_bytes(*codes.shape, 1),), 0xAA, dtype=torch.uint8, device=DEV)
        nova.nova_f8_quantize(x.to(DEV), 1, format=format, transposed=True, Xq=Xq)
        assert torch.equal(nova.nova_f8_pack(codes.to(DEV), scales.to(DEV), 1), Xq)
