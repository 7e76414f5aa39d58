"""Layers with 4-bit weights against their definition in 64 bits: layouts read back, the product and the gradient of its input over types, groups, sizes that
are whole numbers of nothing, row strides, non-finite inputs, graph capture.

Tolerance, per element, of a sum of n products with S = sum |x W|: n roundings to binary32, each at most 2^-24 of a partial sum <= S and of either sign,
stay within (2 sqrt(n) + 16) 2^-23 S (four standard deviations, and room for a matrix unit that cuts off instead of rounding); the gradient's d * s is
held in 16 bits of mantissa in the 16-bit types: 2^-15 S; then one rounding to the type, with its smallest step."""
import numpy as np
import pytest
import torch

from paper_2512_18453_amd import nova

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
UNIT = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
TINY = {F32: 2.0 ** -149, F16: 2.0 ** -24, BF16: 2.0 ** -133}
FWD, BWD = nova.NOVA_Q4_FORWARD, nova.NOVA_Q4_BACKWARD


def make(N, K, group, dtype, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed + 7 * N + K)
    codes = torch.randint(-8, 8, (N, K), dtype=torch.int8, device=DEV, generator=gen)
    scales = (torch.rand((N, -(-K // group)), device=DEV, generator=gen) * 0.1 + 0.002).to(dtype)
    W = codes.double() * scales.double().repeat_interleave(group, 1)[:, :K]
    return gen, codes, scales, W


def close(got, want, S, n, extra=0.0):
    dtype = got.dtype
    bound = UNIT[dtype] * want.abs() + ((2 * n ** 0.5 + 16) * 2.0 ** -23 + extra) * S + TINY[dtype]
    worst = ((got.double() - want).abs() / bound).max().item()
    print(f"  {dtype}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


SHAPES = [(1, 1, 1, 32), (1, 1000, 4096, 64), (3, 17, 33, 32), (16, 16, 128, 128), (5, 130, 257, 128), (17, 100, 1000, 64), (32, 515, 640, 128),
          (33, 48, 2055, 32), (64, 257, 511, 64), (65, 300, 384, 128), (130, 70, 1537, 128), (200, 1030, 260, 32), (2, 20000, 96, 64), (1, 33, 9000, 128),
          (257, 513, 1024, 128), (512, 640, 520, 64)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (100, 333), (33, 640)])
def test_layouts_read_back(N, K, group, dtype):
    _, codes, scales, _ = make(N, K, group, dtype)
    for direction in (FWD, BWD):
        Wq = torch.full((nova.nova_q4_bytes(N, K, group, dtype, direction),), 0xFF, dtype=torch.uint8, device=DEV)
        nova.nova_q4_pack(codes, scales, group, direction, Wq)
        got = nova.nova_q4_unpack(Wq, N, K, group, dtype, direction)
        assert torch.equal(got[0], codes) and torch.equal(got[1], scales)
        # the layout that the header describes, panel by panel
        rows, red, grid = (N, K, codes) if direction == FWD else (K, N, codes.T)
        tiles, chunks = -(-rows // 16), -(-red // 128)
        padded = np.zeros((tiles * 16, chunks * 128), np.int64)
        padded[:rows, :red] = grid.cpu().numpy()
        p = padded.reshape(tiles, 16, chunks, 4, 4, 8).transpose(0, 2, 4, 1, 3, 5)          # tile, chunk, b, i, word, v
        shift = np.array([4 * (v // 2) + 16 * (v % 2) for v in range(8)])
        words = ((p & 15) << shift).sum(-1).astype(np.uint32).reshape(-1)
        assert np.array_equal(Wq.cpu().numpy()[:words.size * 4].view(np.uint32), words)
        G, s = -(-K // group), scales.float().cpu().numpy()
        if direction == FWD:
            want = np.zeros((tiles * 16, chunks * 128 // group), np.float32)
            want[:N, :G] = s
            want = want.reshape(tiles, 16, chunks, -1).transpose(0, 2, 1, 3).reshape(-1)
        else:
            want = np.zeros((G, chunks * 128), np.float32)
            want[:, :N] = s.T
            want = want.reshape(-1)
        tail = Wq[words.size * 4:words.size * 4 + want.size * scales.element_size()].clone().view(dtype).float().cpu().numpy()
        assert np.array_equal(tail, want)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_quantise(dtype):
    N, K, group = 37, 500, 64
    gen = torch.Generator(device=DEV).manual_seed(5)
    w = (torch.randn((N, K), device=DEV, generator=gen) * 0.05).to(dtype)
    w[3, 64:128] = 0.0                                      # a group of zeros
    w[4, :64] *= 1e-30 if dtype != F16 else 0.0             # tiny weights
    w[5, 70], w[6, 130], w[7, 499] = float("nan"), float("inf"), float("-inf")
    padded = torch.zeros((N, 8 * group), device=DEV)
    padded[:, :K] = w.float()
    blocks = padded.reshape(N, 8, group)
    largest = blocks.abs().amax(2)
    s = (largest / torch.full_like(largest, 7.0)).to(dtype)         # (a quotient by a number would be a product with its inverse here)
    s = torch.where(torch.isfinite(s), s, float("nan"))
    c = torch.round(blocks / s.float().unsqueeze(2)).clamp(-8, 7)
    c = torch.where((s > 0).unsqueeze(2), c, 0.0).reshape(N, -1)[:, :K].to(torch.int8)
    for direction in (FWD, BWD):
        codes, scales = nova.nova_q4_unpack(nova.nova_q4_quantize(w, group, direction), N, K, group, dtype, direction)
        assert torch.equal(torch.nan_to_num(scales, nan=-1.0), torch.nan_to_num(s, nan=-1.0)) and torch.equal(codes, c)
    assert torch.isnan(scales[5, 1]) and torch.isnan(scales[6, 2]) and torch.isnan(scales[7, 7]) and scales[3, 1] == 0


def test_codes_out_of_range_are_kept_within():
    codes = torch.tensor([[-128, -9, -8, 7, 8, 127]], dtype=torch.int8, device=DEV)
    Wq = nova.nova_q4_pack(codes, torch.ones((1, 1), device=DEV), 32)
    assert nova.nova_q4_unpack(Wq, 1, 6, 32, F32)[0].tolist() == [[-8, -8, -8, 7, 7, 7]]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("M,N,K,group", SHAPES)
def test_linear(M, N, K, group, dtype):
    print(f"[case] linear {M} x {N} x {K}, group {group}, {dtype}", flush=True)
    gen, codes, scales, W = make(N, K, group, dtype)
    Wq = nova.nova_q4_pack(codes, scales, group)
    x = torch.randn((M, K), device=DEV, generator=gen).to(dtype)
    bias = torch.randn((N,), device=DEV, generator=gen).to(dtype)
    want, S = x.double() @ W.T, x.double().abs() @ W.abs().T
    ws = torch.full((nova.nova_q4_linear_workspace_bytes(M, N, K, group, dtype),), 0xFF, dtype=torch.uint8, device=DEV)
    y = torch.full((M, N), float("nan"), dtype=dtype, device=DEV)
    got = nova.nova_q4_linear(x, Wq, N, group, y=y, workspace=ws)
    assert got is y
    close(got, want, S, K)
    again = nova.nova_q4_linear(x, Wq, N, group)
    assert torch.equal(got, again)                          # equal calls, equal bits, whatever the workspace held
    relu = nova.nova_q4_linear(x, Wq, N, group, bias=bias, flags=nova.NOVA_FLAG_RELU)
    want = want + bias.double()
    assert bool((relu >= 0).all())
    close(relu, want.clamp(min=0.0), S + bias.double().abs(), K + 1)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("M,N,K,group", SHAPES)
def test_backward(M, N, K, group, dtype):
    print(f"[case] backward {M} x {N} x {K}, group {group}, {dtype}", flush=True)
    gen, codes, scales, W = make(N, K, group, dtype)
    Wq = nova.nova_q4_pack(codes, scales, group, BWD)
    dy = torch.randn((M, N), device=DEV, generator=gen).to(dtype)
    y = torch.randn((M, N), device=DEV, generator=gen).to(dtype)
    y[:, 0] = 0.0
    extra = 0.0 if dtype == F32 else 2.0 ** -15
    ws = torch.full((nova.nova_q4_linear_workspace_bytes(M, N, K, group, dtype, BWD),), 0xFF, dtype=torch.uint8, device=DEV)
    dx = torch.full((M, K), float("nan"), dtype=dtype, device=DEV)
    got = nova.nova_q4_linear_backward(dy, Wq, K, group, dx=dx, workspace=ws)
    close(got, dy.double() @ W, dy.double().abs() @ W.abs(), N, extra)
    assert torch.equal(got, nova.nova_q4_linear_backward(dy, Wq, K, group))
    d = dy.double() * (y > 0)
    close(nova.nova_q4_linear_backward(dy, Wq, K, group, y=y), d @ W, d.abs() @ W.abs(), N, extra)


# few outputs of a long sum, on both sides of where a sum is cut into more pieces than a unit has waves
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("M,N,K,group", [(1, 10, 8192, 64), (4, 33, 25088, 128), (9, 70, 8193, 32), (16, 515, 12544, 128), (8, 17, 16385, 64),
                                         (6, 16, 60000, 128), (12, 2049, 8200, 64), (5, 2048, 16500, 128)])
def test_long_sums(M, N, K, group, dtype):
    print(f"[case] long sums {M} x {N} x {K}, group {group}, {dtype}", flush=True)
    gen, codes, scales, W = make(N, K, group, dtype)
    x = torch.randn((M, K), device=DEV, generator=gen).to(dtype)
    y = nova.nova_q4_linear(x, nova.nova_q4_pack(codes, scales, group), N, group)
    close(y, x.double() @ W.T, x.double().abs() @ W.abs().T, K)
    del W
    gen, codes, scales, W = make(K, N, group, dtype)            # the gradient's sum runs over the outputs
    dx = nova.nova_q4_linear_backward(x, nova.nova_q4_pack(codes, scales, group, BWD), N, group)
    extra = 0.0 if dtype == F32 else 2.0 ** -15
    close(dx, x.double() @ W, x.double().abs() @ W.abs(), K, extra)


def test_gradient_against_differences():
    # (the forward call itself, in binary32, in small steps: it is linear in x, so a central difference is exact up to the rounding of its two results)
    M, N, K, group = 3, 40, 150, 64
    gen, codes, scales, W = make(N, K, group, F32)
    Wq, Wb = nova.nova_q4_pack(codes, scales, group), nova.nova_q4_pack(codes, scales, group, BWD)
    x, v = (torch.randn((M, n), device=DEV, generator=gen) for n in (K, N))
    dx = nova.nova_q4_linear_backward(v, Wb, K, group).double()
    for k in range(0, K, 13):
        step = torch.zeros_like(x)
        step[:, k] = 0.5
        up, down = nova.nova_q4_linear(x + step, Wq, N, group).double(), nova.nova_q4_linear(x - step, Wq, N, group).double()
        slope = ((up - down) * v.double()).sum(1)
        size = ((x.double().abs() + 1) @ W.abs().T * v.double().abs()).sum(1)
        assert bool(((dx[:, k] - slope).abs() <= size * 2.0 ** -20).all()), k


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("M", [1, 7, 70])
def test_strided_rows_and_one_row_for_all(M, dtype):
    N, K, group = 77, 219, 64
    gen, codes, scales, W = make(N, K, group, dtype)
    Wq, Wb = nova.nova_q4_pack(codes, scales, group), nova.nova_q4_pack(codes, scales, group, BWD)
    wide = torch.randn((M, K + 14), device=DEV, generator=gen).to(dtype)
    grid = torch.full((M, N + 9), float("nan"), dtype=dtype, device=DEV)
    x, y = wide[:, 3:3 + K], grid[:, 5:5 + N]               # rows that begin anywhere
    nova.nova_q4_linear(x, Wq, N, group, y=y)
    assert torch.equal(y, nova.nova_q4_linear(x.contiguous(), Wq, N, group))
    assert bool(torch.isnan(grid[:, :5]).all()) and bool(torch.isnan(grid[:, 5 + N:]).all())
    one = x[:1].expand(M, K)
    assert torch.equal(nova.nova_q4_linear(one, Wq, N, group), nova.nova_q4_linear(one.contiguous(), Wq, N, group))
    wide = torch.randn((M, N + 14), device=DEV, generator=gen).to(dtype)
    grid = torch.full((M, K + 9), float("nan"), dtype=dtype, device=DEV)
    dy, dx = wide[:, 3:3 + N], grid[:, 1:1 + K]
    nova.nova_q4_linear_backward(dy, Wb, K, group, y=wide[:, 11:11 + N], dx=dx)
    assert torch.equal(dx, nova.nova_q4_linear_backward(dy.contiguous(), Wb, K, group, y=wide[:, 11:11 + N].contiguous()))
    assert bool(torch.isnan(grid[:, :1]).all()) and bool(torch.isnan(grid[:, 1 + K:]).all())
    ones = dy[:1].expand(M, N)
    assert torch.equal(nova.nova_q4_linear_backward(ones, Wb, K, group), nova.nova_q4_linear_backward(ones.contiguous(), Wb, K, group))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("M", [2, 40, 100])
def test_infinities_and_nan_stay_in_their_rows(M, dtype):
    N, K, group = 50, 300, 32
    gen, codes, scales, W = make(N, K, group, dtype)
    Wq, Wb = nova.nova_q4_pack(codes, scales, group), nova.nova_q4_pack(codes, scales, group, BWD)
    x = torch.randn((M, K), device=DEV, generator=gen).to(dtype)
    clean = nova.nova_q4_linear(x, Wq, N, group)
    x[0, 77], x[1, 299] = float("inf"), float("nan")
    got = nova.nova_q4_linear(x, Wq, N, group)
    sign = codes[:, 77].float()
    want = torch.where(sign == 0, float("nan"), sign * float("inf"))            # infinity times a code of zero is NaN
    assert torch.equal(torch.nan_to_num(got[0].float(), nan=9.0), torch.nan_to_num(want, nan=9.0))
    assert bool(torch.isnan(got[1]).all()) and torch.equal(got[2:], clean[2:])
    relu = nova.nova_q4_linear(x, Wq, N, group, flags=nova.NOVA_FLAG_RELU)
    assert bool(torch.isnan(relu[1]).all())
    dy = torch.randn((M, N), device=DEV, generator=gen).to(dtype)
    y = torch.ones_like(dy)
    y[0, 7], y[1, 49] = 0.0, float("nan")
    clean = nova.nova_q4_linear_backward(dy, Wb, K, group, y=y)
    dy[0, 7], dy[1, 49] = float("nan"), float("inf")         # places that the ReLU closed
    assert torch.equal(nova.nova_q4_linear_backward(dy, Wb, K, group, y=y), clean)
    got = nova.nova_q4_linear_backward(dy, Wb, K, group)
    sign = codes[49].float()
    want = torch.where(sign == 0, float("nan"), sign * float("inf"))
    assert bool(torch.isnan(got[0]).all()) and torch.equal(torch.nan_to_num(got[1].float(), nan=9.0), torch.nan_to_num(want, nan=9.0))
    assert torch.equal(got[2:], clean[2:])


def test_no_rows():
    _, codes, scales, _ = make(20, 40, 32, F16)
    Wq, Wb = nova.nova_q4_pack(codes, scales, 32), nova.nova_q4_pack(codes, scales, 32, BWD)
    assert nova.nova_q4_linear(torch.empty((0, 40), dtype=F16, device=DEV), Wq, 20, 32).shape == (0, 20)
    assert nova.nova_q4_linear_backward(torch.empty((0, 20), dtype=F16, device=DEV), Wb, 40, 32).shape == (0, 40)


@pytest.mark.parametrize("M,N,K", [(1, 1000, 4096), (32, 600, 5000), (300, 700, 1000)])
def test_graph_and_other_stream(M, N, K):
    gen, codes, scales, _ = make(N, K, 128, BF16)
    Wq, Wb = nova.nova_q4_pack(codes, scales, 128), nova.nova_q4_pack(codes, scales, 128, BWD)
    x = torch.randn((M, K), device=DEV, generator=gen).to(BF16)
    y, dx = torch.empty((M, N), dtype=BF16, device=DEV), torch.empty((M, K), dtype=BF16, device=DEV)
    wf, wb = (torch.empty(nova.nova_q4_linear_workspace_bytes(M, N, K, 128, BF16, d), dtype=torch.uint8, device=DEV) for d in (FWD, BWD))

    def both():
        nova.nova_q4_linear(x, Wq, N, 128, y=y, flags=nova.NOVA_FLAG_RELU, workspace=wf)
        nova.nova_q4_linear_backward(y, Wb, K, 128, y=y, dx=dx, workspace=wb)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    stream = torch.cuda.Stream()
    for rep in range(3):
        x.copy_(torch.randn((M, K), device=DEV, generator=gen).to(BF16))
        both()
        want = y.clone(), dx.clone()
        for t in (y, dx):
            t.fill_(float("nan"))
        for t in (wf, wb):
            t.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1]), rep
        with torch.cuda.stream(stream):
            again = nova.nova_q4_linear(x, Wq, N, 128, flags=nova.NOVA_FLAG_RELU)
        stream.synchronize()
        assert torch.equal(again, want[0])


def test_offsets_beyond_32_bits():
    # rows 2^30 elements apart: the third begins 2^32 bytes into the buffer
    M, N, K, group, far = 3, 300, 500, 128, 1 << 30
    gen, codes, scales, W = make(N, K, group, F16)
    Wq, Wb = nova.nova_q4_pack(codes, scales, group), nova.nova_q4_pack(codes, scales, group, BWD)
    space = [torch.empty(2 * far + 512, dtype=F16, device=DEV) for _ in range(2)]
    x, y = space[0].as_strided((M, K), (far, 1)), space[1].as_strided((M, N), (far, 1))
    x.copy_(torch.randn((M, K), device=DEV, generator=gen))
    nova.nova_q4_linear(x, Wq, N, group, y=y)
    assert torch.equal(y, nova.nova_q4_linear(x.contiguous(), Wq, N, group)) and bool((y[2] != 0).any())
    want = nova.nova_q4_linear_backward(y.contiguous(), Wb, K, group)
    nova.nova_q4_linear_backward(y, Wb, K, group, dx=x)
    assert torch.equal(x, want)
