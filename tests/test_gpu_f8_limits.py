"""Layouts and results beyond 2^32 bytes, two calls at once on two streams, workspaces that hold anything, long sums: 8-bit float layers where offsets and orders go wrong first."""
import pytest
import torch

from paper_2512_18453_amd import nova

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def normal(*shape, seed=0, dtype=BF16):
    return torch.randn(shape, device=DEV, generator=torch.Generator(DEV).manual_seed(seed)).to(dtype)


def test_layout_of_more_than_2_to_the_32_bytes():
    N, K = 65552, 65664
    assert nova.nova_f8_bytes(N, K, 128) > 1 << 32
    w, last = normal(1, K, seed=1), normal(16, K, seed=2)
    few = nova.nova_f8_quantize(torch.cat([w.expand(16, K), last]), 1)
    Wq = nova.nova_f8_quantize(w.expand(N, K), 1)
    # the last panel of rows is another
    panel = K // 128 * 2048
    Wq[(N // 16 - 1) * panel:N // 16 * panel] = few[panel:2 * panel]
    scales = Wq[N * K:].view(F32).view(K // 128, N)
    scales[:, N - 16:] = few[32 * K:].view(F32).view(K // 128, 32)[:, 16:]
    for M in (1, 40, 130):
        x = nova.nova_f8_quantize(normal(M, K, seed=3), 1)
        want = nova.nova_f8_matmul(x, few, M, 32, K, block_b=1, dtype=F32)
        got = nova.nova_f8_matmul(x, Wq, M, N, K, block_b=1, dtype=F32)
        # The sums of fewer columns are cut into other pieces: 513 additions each, of partial sums that are below 2^10 (four standard deviations of 65664 products), which
        # round by 2^-15 at most, on both sides
        bound = 2 * 513 * 2.0 ** -15
        torch.testing.assert_close(got[:, :N - 16:4096], want[:, :1].expand(M, 16), rtol=0, atol=bound)
        torch.testing.assert_close(got[:, N - 16:], want[:, 16:], rtol=0, atol=bound)
    codes, s = nova.nova_f8_unpack(Wq, N, K, 1)
    small = nova.nova_f8_unpack(few, 32, K, 1)
    assert torch.equal(codes[-16:].view(torch.uint8), small[0][16:].view(torch.uint8)) and torch.equal(s[-17:], small[1][15:])
    assert torch.equal(codes[0].view(torch.uint8), small[0][0].view(torch.uint8)) and torch.equal(codes[N - 17].view(torch.uint8), small[0][0].view(torch.uint8))


def test_results_of_more_than_2_to_the_32_bytes():
    M, N, K = 66003, 33000, 130
    x, w = normal(M, K, seed=1), normal(N, K, seed=2)
    Wq = nova.nova_f8_quantize(w, 128)
    y = nova.nova_f8_linear(x, Wq, N)
    for rows in (slice(0, 130), slice(32700, 32900), slice(M - 131, M)):
        assert torch.equal(y[rows], nova.nova_f8_linear(x[rows], Wq, N))                     # K fits one cut: the sums are the same
    dy = normal(M, 40, seed=3)
    _, dw, db = nova.nova_f8_linear_backward(dy, None, x)
    assert bool(dw.isfinite().all()) and torch.allclose(db.double(), dy.double().sum(0), rtol=1e-5, atol=1e-3)


def test_transposed_of_more_than_2_to_the_32_bytes():
    rows, columns = 65664, 65552
    Xq = nova.nova_f8_quantize(normal(1, columns, seed=4).expand(rows, columns), 1, transposed=True)
    codes, scales = nova.nova_f8_unpack(Xq, columns, rows, 1)
    x = normal(1, columns, seed=4)[0].float()
    at = torch.tensor([0, 5, columns - 17, columns - 1], device=DEV)
    # a column of one number: its code is the largest, with the number's sign
    assert torch.equal(codes[at][:, ::8192].float(), (448.0 * x[at].sign()).unsqueeze(1).expand(-1, 9))
    torch.testing.assert_close(scales[at], (x[at].abs() / 448).unsqueeze(1).expand(-1, rows // 128), rtol=1e-6, atol=0)


@pytest.mark.parametrize("M", [1, 32, 200])
def test_two_streams_at_once(M):
    """Two calls of different layers, each on a stream and with a workspace of its own, many times over; workspaces begin with anything."""
    N, K = 1000, 4096
    layers = [(nova.nova_f8_quantize(normal(N, K, seed=s), 128), normal(M, K, seed=10 + s)) for s in (1, 2)]
    want = [nova.nova_f8_linear(x, W, N) for W, x in layers]
    streams, outs = [torch.cuda.Stream() for _ in layers], [[] for _ in layers]
    work = [torch.full((nova.nova_f8_linear_workspace_bytes(M, N, K, BF16),), 0xFF, dtype=torch.uint8, device=DEV) for _ in layers]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, (W, x) in enumerate(layers):
            with torch.cuda.stream(streams[i]):
                outs[i].append(nova.nova_f8_linear(x, W, N, workspace=work[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in outs[i])


@pytest.mark.parametrize("M", [1, 17, 70])
def test_long_sums(M):
    """Ones: every partial sum is a whole number below 2^24, the result is K exactly."""
    N, K = 5, 1 << 22
    W, x = torch.ones((1, K), device=DEV, dtype=F16), torch.ones((1, K), device=DEV, dtype=F16)
    codes = torch.full((N, K), 1.0, device=DEV).to(torch.float8_e4m3fn)
    Wq = nova.nova_f8_pack(codes, torch.ones((N, K // 128), device=DEV), 1)
    Xq = nova.nova_f8_pack(codes[:1].expand(M, K).contiguous(), torch.ones((M, K // 128), device=DEV), 1)
    assert bool((nova.nova_f8_matmul(Xq, Wq, M, N, K, block_b=1, dtype=F32) == K).all())
    assert bool((nova.nova_f8_matmul(Xq, Wq, M, N, K, block_b=1, dtype=BF16) == K).all())
    dy = torch.ones((1, N), device=DEV, dtype=F16)
    dx, _, _ = nova.nova_f8_linear_backward(dy.expand(M, N), nova.nova_f8_quantize(W.expand(N, K), 128, transposed=True), None, K=K)
    assert bool((dx == N).all())


def test_more_rows_than_the_weights_gradient_sums_in_one_piece():
    M, N, K = 300001, 24, 40
    dy, x = (torch.randint(-1, 2, (M, n), device=DEV, generator=torch.Generator(DEV).manual_seed(n)).to(F16) for n in (N, K))
    _, dw, db = nova.nova_f8_linear_backward(dy, None, x)
    # whole numbers: scales of 1/448 (1/57344) are not powers of two, so codes are exact and scales are rounded: each product by 3 2^-24, sums as they are
    want, terms = dy.double().T @ x.double(), dy.double().abs().T @ x.double().abs()
    assert bool(((dw.double() - want).abs() <= (3 + M / 128) * 2.0 ** -24 * terms).all())
    assert torch.equal(db.double(), dy.double().sum(0))
