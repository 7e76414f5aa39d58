"""Layers with 4-bit weights at the ends of what the types hold: definition and tolerances as in test_gpu_q4.py."""
import pytest
import torch

from paper_2512_18453_amd import nova
from test_gpu_q4 import BF16, BWD, DEV, F16, F32, close, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [2, 40, 100])
def test_closed_places_meet_weights_that_are_no_numbers(M, group, dtype):
    # d = 0 behind a closed ReLU, and 0 times NaN or an infinity is NaN
    N, K = 70, 500
    gen, codes, scales, W = make(N, K, group, dtype)
    dy = torch.randn((M, N), device=DEV, generator=gen).to(dtype)
    y = torch.ones_like(dy)
    y[:, 7], y[:, 66] = 0.0, -1.0
    clean = nova.nova_q4_linear_backward(dy, nova.nova_q4_pack(codes, scales, group, BWD), K, group, y=y)
    scales[7, 1], scales[66, 2] = float("nan"), float("inf")
    got = nova.nova_q4_linear_backward(dy, nova.nova_q4_pack(codes, scales, group, BWD), K, group, y=y)
    bad = torch.zeros(K, dtype=torch.bool, device=DEV)
    bad[group:3 * group] = True
    assert bool(torch.isnan(got[:, bad]).all()) and torch.equal(got[:, ~bad], clean[:, ~bad])
