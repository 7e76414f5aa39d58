"""Dropout: its mask bit for bit from the documented counters, its values and gradient, strides, sizes, masks that differ from replay to replay of a graph."""
import pytest
import torch

from paper_2512_18453_amd import nova
from tests import plain_training as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF_STEP = {F32: 0.0, F16: 2.0 ** -11, BF16: 2.0 ** -8}
SMALLEST = {F32: 0.0, F16: 2.0 ** -24, BF16: 2.0 ** -133}


def normal(*shape, seed=0, dtype=F32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def near(got, want, dtype):
    """want: binary32, as the documentation forms it; got: that rounded once (a product of binary32 and its rounding may be one step: 2^-24 more)."""
    err = (got.cpu().double() - want.double()).abs()
    assert bool((err <= (HALF_STEP[dtype] + (2.0 ** -24 if dtype != F32 else 0.0)) * want.double().abs() + SMALLEST[dtype]).all()), err.max().item()


SHAPES = [(1, 1), (1, 7), (3, 8), (5, 9), (2, 1000), (129, 33), (64, 4096), (1000, 1)]


@pytest.mark.parametrize("rows,columns", SHAPES)
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_forward_and_gradient(rows, columns, dtype, p):
    seed, offset = 0xFEDCBA9876543210 + columns, (1 << 40) + rows
    keep, factor = plain.kept(rows, columns, p, seed, offset), torch.tensor(1.0 / (1.0 - p) if p < 1 else 0.0, dtype=F32)
    x, r, dy = (normal(rows, columns, seed=s, dtype=dtype) for s in (1, 2, 3))
    x_on, r_on, dy_on = x.to(DEV), r.to(DEV), dy.to(DEV)
    branch = torch.where(keep, x.float() * factor, 0.0)
    near(nova.nova_dropout(x_on, p, seed, offset=offset), branch, dtype)
    near(nova.nova_dropout(x_on, p, seed, offset=offset, residual=r_on), branch + r.float(), dtype)
    opened = torch.where(keep, x.float().clamp(min=0.0) * factor, 0.0)
    y = nova.nova_dropout(x_on, p, seed, offset=offset, flags=nova.NOVA_FLAG_RELU)
    near(y, opened, dtype)
    near(nova.nova_dropout(x_on, p, seed, offset=offset, residual=r_on, flags=nova.NOVA_FLAG_RELU), opened + r.float(), dtype)
    back = torch.where(keep, dy.float() * factor, 0.0)
    near(nova.nova_dropout_backward(dy_on, p, seed, offset=offset), back, dtype)
    gated = nova.nova_dropout_backward(dy_on, p, seed, offset=offset, gate=x_on)
    near(gated, torch.where(x > 0, back, 0.0), dtype)
    assert torch.equal(nova.nova_dropout_backward(dy_on, p, seed, offset=offset, gate=y), gated)      # what the ReLU made opens the same places
    if p == 0.0:
        assert torch.equal(nova.nova_dropout(x_on, p, seed), x_on)


@pytest.mark.parametrize("p", [0.1, 0.3, 0.5, 2.0 ** -16, 2.0 ** -32, 2.0 ** -34, 1 - 2.0 ** -32, 1 - 2.0 ** -20])
def test_decisions_that_need_all_32_bits(p):
    """4 million elements, of which some 60 have the upper 16 bits of the threshold."""
    rows, columns, seed = 1024, 4096, 77
    u = plain.random_bits(rows, columns, seed, 5)
    threshold = int(p * 2.0 ** 32 + 0.5)
    assert 20 < int((u >> 16 == min(threshold >> 16, 65535)).sum()) < 140
    x = torch.ones((rows, columns), device=DEV)
    got = nova.nova_dropout(x, p, seed, offset=5).cpu() != 0
    assert torch.equal(got, torch.from_numpy(u.astype("int64") >= threshold))


def test_how_many_stay():
    """Of n elements the number kept is binomial: within six standard deviations of its mean."""
    n = 1 << 24
    for p in (0.05, 0.5, 0.9):
        y = nova.nova_dropout(torch.ones((1 << 12, 1 << 12), device=DEV), p, 123456789)
        kept = int((y != 0).sum())
        assert abs(kept - n * (1 - p)) <= 6 * (n * p * (1 - p)) ** 0.5
        assert bool(((y == 0) | (y == torch.tensor(1 / (1 - p), dtype=F32))).all())


def test_mask_is_of_row_and_column_alone():
    seed = 3
    whole = nova.nova_dropout(torch.ones((300, 1000), device=DEV), 0.4, seed)
    part = nova.nova_dropout(torch.ones((17, 333), device=DEV, dtype=BF16), 0.4, seed)
    assert torch.equal(part != 0, whole[:17, :333] != 0)
    for other in (dict(seed=4), dict(seed=seed + (1 << 32)), dict(seed=seed, offset=1), dict(seed=seed, offset=1 << 32)):
        assert not torch.equal(nova.nova_dropout(torch.ones((300, 1000), device=DEV), 0.4, **other) != 0, whole != 0)
    assert torch.equal(nova.nova_dropout(torch.ones((300, 1000), device=DEV), 0.4, seed, offset=-1) != 0, plain.kept(300, 1000, 0.4, seed, 2 ** 64 - 1).to(DEV))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("columns", [1, 8, 37, 1000])
def test_strides_and_places(dtype, columns):
    """Rows apart, at odd addresses, one row for all, results in the place of an input; nothing beside them is touched."""
    rows, p, seed = 9, 0.3, 11
    wide = normal(rows, 3 * (columns + 3), seed=1, dtype=dtype).to(DEV)
    x, r, out = (wide[:, i * (columns + 3) + 1:i * (columns + 3) + 1 + columns] for i in range(3))
    kept_beside = wide.clone()
    want = nova.nova_dropout(x.contiguous(), p, seed, residual=r.contiguous())
    assert torch.equal(nova.nova_dropout(x, p, seed, residual=r, y=out), want)
    kept_beside[:, 2 * (columns + 3) + 1:2 * (columns + 3) + 1 + columns] = want
    assert torch.equal(wide, kept_beside)
    one = nova.nova_dropout(x[:1].expand(rows, columns), p, seed)
    assert torch.equal(one, nova.nova_dropout(x[:1].repeat(rows, 1), p, seed))
    a, b = x.clone(memory_format=torch.contiguous_format), r.clone(memory_format=torch.contiguous_format)
    assert torch.equal(nova.nova_dropout(a, p, seed, residual=b, y=a), want)
    a = x.clone(memory_format=torch.contiguous_format)
    assert torch.equal(nova.nova_dropout(a, p, seed, residual=b, y=b), want)
    gated = nova.nova_dropout_backward(a, p, seed, gate=x)
    g = x.clone(memory_format=torch.contiguous_format)
    assert torch.equal(nova.nova_dropout_backward(a, p, seed, gate=g, dx=g), gated)


def test_dropped_values_do_not_matter():
    keep = plain.kept(64, 64, 0.5, 9, 0).to(DEV)
    x = torch.where(keep, 1.0, float("nan"))
    x[0] = torch.where(keep[0], 1.0, float("inf"))
    assert torch.equal(nova.nova_dropout(x, 0.5, 9), torch.where(keep, 2.0, 0.0))
    assert torch.equal(nova.nova_dropout_backward(x, 0.5, 9), torch.where(keep, 2.0, 0.0))
    assert bool(nova.nova_dropout(torch.full((64, 64), float("nan"), device=DEV), 0.5, 9, flags=nova.NOVA_FLAG_RELU)[keep].isnan().all())
    gate = torch.full((64, 64), float("nan"), device=DEV)
    assert not nova.nova_dropout_backward(torch.ones((64, 64), device=DEV), 0.5, 9, gate=gate).any()
    assert nova.nova_dropout(torch.empty((0, 8), device=DEV), 0.5, 9).shape == (0, 8) and nova.nova_dropout(torch.empty((8, 0), device=DEV), 0.5, 9).shape == (8, 0)


def test_gradient_against_differences():
    """Kept or not, the call is linear in x: differences of binary32 sums of small whole numbers are exact."""
    x = torch.randint(1, 100, (40, 72), device=DEV, dtype=F32, generator=torch.Generator(DEV).manual_seed(1))
    dy = torch.randint(-9, 9, (40, 72), device=DEV, dtype=F32, generator=torch.Generator(DEV).manual_seed(2))
    dx = nova.nova_dropout_backward(dy, 0.5, 21, gate=x)
    for i, j in ((0, 0), (3, 71), (39, 13), (17, 40)):
        step = x.clone()
        step[i, j] += 1
        change = nova.nova_dropout(step, 0.5, 21, flags=nova.NOVA_FLAG_RELU) - nova.nova_dropout(x, 0.5, 21, flags=nova.NOVA_FLAG_RELU)
        assert (change.double() * dy).sum() == dx[i, j]


def test_more_than_2_to_the_32_elements():
    rows, columns, seed = 65537, 65536 + 8, 5
    x = torch.ones((rows, columns), dtype=BF16, device=DEV)
    nova.nova_dropout(x, 0.5, seed, y=x)
    for first in (0, 32760, rows - 8):
        want = torch.from_numpy(plain.random_bits(8, columns, seed, 0, first_row=first).astype("int64") >= 1 << 31)
        assert torch.equal(x[first:first + 8].cpu() != 0, want)


def test_long_rows():
    columns = (1 << 31) - 1
    x = torch.ones((1, columns), dtype=BF16, device=DEV)
    nova.nova_dropout(x, 0.5, 5, y=x)
    assert abs(int((x[0, -(1 << 24):] != 0).sum()) - (1 << 23)) < 6 * (1 << 11)
    assert x[0, -1] in (0.0, 2.0) and bool((x[0, -9:] != 1).all())


def test_masks_of_a_replayed_graph():
    """The number on the device is read when the kernel runs: a replay draws the mask of its step, forward and backward the same one."""
    step = torch.zeros((1,), dtype=torch.int64, device=DEV)
    x, dy = normal(50, 100, seed=1).to(DEV), normal(50, 100, seed=2).to(DEV)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        nova.nova_dropout(x, 0.3, 17, offset=100, device_offset=step, y=y)
        nova.nova_dropout_backward(dy, 0.3, 17, offset=100, device_offset=step, dx=dx)
        step.add_(1)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, nova.nova_dropout(x, 0.3, 17, offset=100 + i)) and torch.equal(dx, nova.nova_dropout_backward(dy, 0.3, 17, offset=100 + i))
    step.fill_(-100)
    assert torch.equal(nova.nova_dropout(x, 0.3, 17, offset=100, device_offset=step), nova.nova_dropout(x, 0.3, 17))
