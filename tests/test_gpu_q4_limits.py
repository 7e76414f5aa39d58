"""Layers with 4-bit weights at the ends of what the types hold: definition and tolerances as in test_gpu_q4.py."""
import pytest
import torch

from launches import launches
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


# every kernel and height of tile, sums in one piece and cut, K that ends inside a panel, a panel that holds one group and several
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K,group", [(1, 130, 300, 128), (2, 40000, 130, 64), (4, 700, 2999, 32), (7, 300, 1000, 128), (16, 500, 2048, 64),
                                         (16, 60, 30000, 128), (30, 77, 515, 32), (33, 300, 5000, 128), (100, 200, 640, 64), (1010, 8150, 400, 128)])
def test_large_rows_under_small_scales(M, N, K, group, dtype):
    # the sum of a group over its codes is beyond binary32, the scaled one is not
    gen, codes, scales, W = make(N, K, group, dtype)
    scales *= 2.0 ** -30                                     # (exact)
    W *= 2.0 ** -30
    Wq = nova.nova_q4_pack(codes, scales, group)
    x = torch.randn((M, K), device=DEV, generator=gen).to(dtype)
    bias = torch.randn((N,), device=DEV, generator=gen).to(dtype)
    clean = nova.nova_q4_linear(x, Wq, N, group, bias=bias)
    rows = sorted({0, M // 2, M - 1})
    for r in rows:
        x[r] = (torch.sign(x[r].float()) * 2.0 ** 126 * (1 + torch.rand((K,), device=DEV, generator=gen))).clamp(-2.0 ** 127, 2.0 ** 127).to(dtype)
    x[M - 1, K // 2:] = 2.0 ** 126                           # (sums of one sign)
    codes[5, :] = 7
    W[5] = 7 * scales[5].double().repeat_interleave(group)[:K]
    Wq = nova.nova_q4_pack(codes, scales, group)
    ws = torch.full((nova.nova_q4_linear_workspace_bytes(M, N, K, group, dtype),), 0xFF, dtype=torch.uint8, device=DEV)
    got = nova.nova_q4_linear(x, Wq, N, group, bias=bias, workspace=ws)
    want, S = x[rows].double() @ W.T + bias.double(), x[rows].double().abs() @ W.abs().T + bias.double().abs()
    close(got[rows], want, S, K + 1)
    others = [r for r in range(M) if r not in rows]
    columns = torch.arange(N, device=DEV) != 5
    assert torch.equal(got[others][:, columns], clean[others][:, columns])      # rows beside them keep their bits
    relu = nova.nova_q4_linear(x, Wq, N, group, bias=bias, flags=nova.NOVA_FLAG_RELU)
    assert torch.equal(relu, torch.where(got < 0, 0.0, got))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("M", [1, 9, 40, 150])
def test_results_beyond_the_type_are_infinite(M, dtype):
    N, K, group = 48, 400, 32
    gen, codes, scales, W = make(N, K, group, dtype)
    codes = codes.abs().clamp(min=1, max=7)
    codes[1::2] *= -1
    x = (2.0 ** 126 * (1 + torch.rand((M, K), device=DEV, generator=gen))).clamp(max=2.0 ** 127).to(dtype)
    got = nova.nova_q4_linear(x, nova.nova_q4_pack(codes, torch.ones_like(scales), group), N, group)
    want = torch.full((M, N), float("inf"), device=DEV)
    want[:, 1::2] *= -1
    assert torch.equal(got.float(), want)


@pytest.mark.parametrize("M,dtype", [(1027, F16), (515, F32)])
def test_more_rows_than_one_launch(M, dtype):
    # the gradient of 2^24 inputs, the widest there is: 1024 (512) rows are 2^23 workgroups, all that a launch takes
    N, K, group = 3, 1 << 24, 32
    print(f"[case] backward {M} x {N} x {K}, {dtype}", flush=True)
    gen, codes, scales, W = make(N, K, group, dtype)
    Wb = nova.nova_q4_pack(codes, scales, group, BWD)
    dy, y = (torch.randn((M, N), device=DEV, generator=gen).to(dtype) for _ in range(2))
    dx = torch.empty((M, K), dtype=dtype, device=DEV)
    ws = torch.empty(nova.nova_q4_linear_workspace_bytes(M, N, K, group, dtype, BWD), dtype=torch.uint8, device=DEV)
    found = launches(lambda: nova.nova_q4_linear_backward(dy, Wb, K, group, y=y, dx=dx, workspace=ws))
    assert [blocks for _, blocks, _ in found] == [1 << 23, 1 << 18]
    nova.nova_q4_linear_backward(dy, Wb, K, group, y=y, dx=dx, workspace=ws)
    for r in (0, M - 4, M - 3, M - 2, M - 1):                # (the launch's last row, and the next one's)
        d = (dy[r:r + 1] * (y[r:r + 1] > 0)).double()
        close(dx[r:r + 1], d @ W, d.abs() @ W.abs(), N, 0.0 if dtype == F32 else 2.0 ** -15)


@pytest.mark.parametrize("M", [3, 40])
def test_weights_beyond_32_bits(M):
    # 9.4e9 weights: codes and layouts of more than 2^32 bytes
    N, K, group, dtype = (1 << 20) + 5, 9001, 128, F16
    gen = torch.Generator(device=DEV).manual_seed(M)
    codes = torch.randint(-8, 8, (N, K), dtype=torch.int8, device=DEV, generator=gen)
    scales = (torch.rand((N, -(-K // group)), device=DEV, generator=gen) * 0.1 + 0.002).to(dtype)

    def weights(rows, columns):
        return codes[rows][:, columns].double() * scales[rows][:, columns // group].double()
    every, some = slice(None), torch.tensor([0, 1, 524287, 524288, N - 2, N - 1], device=DEV)
    x = torch.randn((M, K), device=DEV, generator=gen).to(dtype)
    Wq = nova.nova_q4_pack(codes, scales, group)
    W = weights(some, torch.arange(K, device=DEV))
    close(nova.nova_q4_linear(x, Wq, N, group)[:, some], x.double() @ W.T, x.double().abs() @ W.abs().T, K)
    back = nova.nova_q4_unpack(Wq, N, K, group, dtype)
    assert torch.equal(back[0], codes) and torch.equal(back[1], scales)
    del Wq, back
    Wb = nova.nova_q4_pack(codes, scales, group, BWD)
    dy = torch.randn((M, N), device=DEV, generator=gen).to(dtype)
    some = torch.tensor([0, 127, 128, 4500, K - 1], device=DEV)
    W = weights(every, some)
    close(nova.nova_q4_linear_backward(dy, Wb, K, group)[:, some], dy.double() @ W, dy.double().abs() @ W.abs(), N, 2.0 ** -15)
