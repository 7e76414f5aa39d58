"""Log probabilities: what rounding of the scale costs, rows of logits and of masks at different strides, more rows than one launch takes."""
import math

import pytest
import torch

from paper_2512_18453_amd import nova
from test_gpu_logprobs import BF16, DEV, F16, F32, TINY, UNIT, check, definition, error, gradient, make, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.9, 0.55, 1.0])
@pytest.mark.parametrize("V", [131071, 1000003])
def test_scale_is_not_rounded_twice(V, scale):
    # scale log2 e rounded to binary32 is off by up to 1.2 units of 2^-24 (0.86 at 0.9), the same for all entries of a row: with d the distance to the largest
    # logit, E its mean and W its variance, L would be off by E and the entropy by W times that.  What else is off is of either sign: every exponent is rounded
    # by 2^-24 of itself at most, by different amounts for different logits, of which there are as many as entries (E 2^-27 and W 2^-28 are left of it in the
    # mean over the entries); the sums, the logarithm, its product and the result are each rounded by a unit at most, so that the mean error of 64 rows stays
    # within one and a half units of 1 + L (two of 1 + H).
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


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("R,V", [(4, 301), (2, 30001), (400, 2049), (1500, 70)])
def test_rows_of_logits_and_of_masks_at_different_strides(R, V, dtype):
    # what a row gives does not depend on where it and its mask begin
    gen, _, targets = make(R, V, dtype)
    a, h = torch.randn((R,), device=DEV, generator=gen), torch.randn((R,), device=DEV, generator=gen)
    for offset, mask_offset in ((0, 5), (1, 0), (3, 2), (7, 7)):
        x = torch.randn((R, V + 13), device=DEV, generator=gen).to(dtype)[:, offset:offset + V]
        mask = (torch.rand((R, V + 30), device=DEV, generator=gen) < 0.7)[:, mask_offset:mask_offset + V]
        got = nova.nova_logprobs(x, targets, mask=mask, scale=0.8, top=9)
        want = nova.nova_logprobs(x.contiguous(), targets, mask=mask.contiguous(), scale=0.8, top=9)
        for p, q in zip(got, want, strict=True):
            assert torch.equal(p, q)
        grid = torch.full((R, V + 17), 7.0, dtype=dtype, device=DEV)
        nova.nova_logprobs_backward(x, want.stats, targets, g_logprob=a, entropy=want.entropy, g_entropy=h, mask=mask, scale=0.8, dlogits=grid[:, 2:2 + V])
        back = nova.nova_logprobs_backward(x.contiguous(), want.stats, targets, g_logprob=a, entropy=want.entropy, g_entropy=h, mask=mask.contiguous(), scale=0.8)
        assert torch.equal(grid[:, 2:2 + V], back) and bool((grid[:, :2] == 7).all()) and bool((grid[:, 2 + V:] == 7).all())


@pytest.mark.parametrize("masks", ["none", "rows", "shared"])
@pytest.mark.parametrize("V", [1, 3])
def test_more_rows_than_one_launch(V, masks):
    # a launch takes 2^22 rows
    R = (1 << 22) + 3
    print(f"[case] {R} x {V}, masks: {masks}", flush=True)
    gen, x, targets = make(R, V, F16)
    mask = None
    if masks != "none":
        mask = torch.rand((R if masks == "rows" else 1, V), device=DEV, generator=gen) < 0.7
        mask[:, 0] = True
        if masks == "shared":
            targets[:] = 0
        else:
            mask.scatter_(1, targets.unsqueeze(1), True)
    f, want = check(x, targets, mask, 0.8, 2)
    a, h = torch.randn((R,), device=DEV, generator=gen), torch.randn((R,), device=DEV, generator=gen)
    got = nova.nova_logprobs_backward(x, f.stats, targets, g_logprob=a, entropy=f.entropy, g_entropy=h, mask=mask, scale=0.8)
    g, size = gradient(x, targets, mask, 0.8, a, h, want)
    bound = size * 2 * error(V, torch.where(want["lp"] > -60, want["lp"], 60.0), want["L"].unsqueeze(1)) + UNIT[F16] * g.abs() + TINY[F16]
    within(got, g, bound, "gradient")


@pytest.mark.parametrize("V", [100, 2049, 30001])
def test_small_scales_of_large_logits(V):
    # d = scale (x - M) has two roundings and ln p = d - L a third: two units of 2^-24 of |d| are what `error` has for them, so d is not rounded on the way
    for scale in (1e-3, 2.3e-4, 7e-3):
        gen = torch.Generator(device=DEV).manual_seed(V)
        x = 6e4 * torch.randn((400, V), device=DEV, generator=gen)
        targets = torch.randint(0, V, (400,), device=DEV, generator=gen)
        check(x, targets, None, torch.tensor(scale, dtype=F32).item(), 9)


def test_longest_row():
    # V = 2^31 - 1, as long as a row can be: 64 slices forward, 262144 workgroups a row backward
    V, step = 2 ** 31 - 1, 1 << 27
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.empty((1, V), dtype=BF16, device=DEV)
    for lo in range(0, V, step):
        x[0, lo:lo + step] = torch.randn((min(step, V - lo),), device=DEV, generator=gen)
    at = [0, V - 1, 1 << 30, (1 << 31) - 9, 77777777]
    x[0, at] = torch.tensor([30.0, 29.0, 28.0, 27.0, 26.0], device=DEV).to(BF16)
    targets = torch.tensor([V - 1], device=DEV)
    got = nova.nova_logprobs(x, targets, top=5)
    sums = torch.zeros(2, dtype=torch.float64, device=DEV)
    for lo in range(0, V, step):
        d = x[0, lo:lo + step].double() - 30.0
        sums += torch.stack([d.exp().sum(), (d.exp() * d).sum()])
    L, E = sums[0].log().item(), (sums[1] / sums[0]).item()
    assert got.top_ids[0].tolist() == at and got.stats[0, 0].item() == 30.0
    assert abs(got.stats[0, 1].item() - L) <= error(V, torch.zeros(()), torch.tensor(L)).item()
    assert abs(got.logprob.item() - (-1.0 - L)) <= error(V, torch.ones(()), torch.tensor(L)).item()
    assert abs(got.entropy.item() - (L - E)) <= error(V, torch.tensor(60.0), torch.tensor(L)).item() * (1 + L - E)
    a = torch.ones(1, device=DEV)
    dx = nova.nova_logprobs_backward(x, got.stats, targets, g_logprob=a, dlogits=x.clone())
    for lo in range(0, V, step):
        p = (x[0, lo:lo + step].double() - 30.0 - L).exp()
        want = -p
        if lo + step >= V:
            want[-1] += 1.0
        within(dx[0, lo:lo + step], want, UNIT[BF16] * want.abs() + 2.0 ** -17 * p + TINY[BF16], "gradient")
