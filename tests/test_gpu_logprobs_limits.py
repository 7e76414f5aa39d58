"""Log probabilities: what rounding of the scale costs."""
import math

import pytest
import torch

from paper_2512_18453_amd import nova
from test_gpu_logprobs import DEV, F32, definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.9, 0.55, 1.0])
@pytest.mark.parametrize("V", [131071, 1000003])
def test_scale_is_not_rounded_twice(V, scale):
    # scale log2 e rounded to binary32 is off by up to 1.2 units of 2^-24 (0.86 at 0.9), the same for all entries of a row: with d the distance to the largest logit, E its mean
    # and W its variance, L would be off by E and the entropy by W times that.  What else is off is of either sign: every exponent is rounded by 2^-24 of itself at most, by different amounts
    # for different logits, of which there are as many as entries (E 2^-27 and W 2^-28 are left of it in the mean over the entries); the sums, the logarithm, its product and the result are each rounded by a unit at most, so that the mean
    # error of 64 rows stays within one and a half units of 1 + L (two of 1 + H).
    gen = torch.Generator(device=DEV).manual_seed(V)
    x = -(math.log(V) + 1.5 * torch.rand((64, V), device=DEV, generator=gen) - 0.75) / scale       # (together about as much as the largest)
    x[:, 11] = 0.0
    scale = torch.tensor(scale, dtype=F32).item()
    got = nova.nova_logprobs(x, scale=scale)
    want = definition(x, torch.full((64,), 11, device=DEV), None, scale, 0)
    L, H, p = want["L"].mean().item(), want["H"].mean().item(), want["lp"].exp()
    d = scale * x.double()
    E = -(p * d).sum(1).mean().item()
    W = (p * d * d).sum(1).mean().item() - E * E
    off_L, off_H = (got.stats[:, 1].double() - want["L"]).mean().item(), (got.entropy.double() - want["H"]).mean().item()
    print(f"  L {L:.3f} off {off_L * 2 ** 24:.2f} units, H {H:.3f} off {off_H * 2 ** 24:.2f}, E {E:.2f}, W {W:.2f}", flush=True)
    assert abs(off_L) <= 1.5 * 2.0 ** -24 * (1 + L) + E * 2.0 ** -27
    assert abs(off_H) <= 2 * 2.0 ** -24 * (1 + H) + W * 2.0 ** -28
