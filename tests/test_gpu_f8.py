"""Layers in 8-bit floating point: quantisation bit for bit, the layout's bytes, products and gradients against 64-bit plain forms with bounds that count every rounding,
strides, masks of the ReLU, values beyond numbers, graphs and streams."""
import pytest
import torch

from paper_2512_18453_amd import nova
from tests import plain_training as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
HALF_STEP = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
SMALLEST = {F32: 2.0 ** -149, F16: 2.0 ** -24, BF16: 2.0 ** -133}


def normal(*shape, seed=0, dtype=F32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def strided(t, gap=5, at=3):
    """The same matrix on the device as a part of a wider one that holds NaN elsewhere."""
    wide = torch.full((t.shape[0], t.shape[1] + gap + at), float("nan"), dtype=t.dtype, device=DEV)
    wide[:, at:at + t.shape[1]] = t.to(DEV)
    return wide[:, at:at + t.shape[1]]


def same_codes(got, want):
    assert torch.equal(got[0].cpu().view(torch.uint8), want[0].view(torch.uint8))
    assert torch.equal(got[1].cpu().view(torch.int32) & -1, want[1].view(torch.int32)) or torch.equal(
        got[1].cpu().nan_to_num(nan=-1.0), want[1].nan_to_num(nan=-1.0))


def near(got, want, bound, dtype):
    """got is want, summed in binary32 with an error below `bound`, rounded once to dtype."""
    err = (got.double().cpu() - want).abs()
    allowed = bound + HALF_STEP[dtype] * (want.abs() + bound) + SMALLEST[dtype]
    over = (err - allowed).max().item()
    assert over <= 0, over


# ---- quantisation ----

@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (5, 7), (16, 128), (17, 129), (130, 300), (129, 8), (300, 2055)])
def test_quantize(shape, transposed, block, dtype):
    for format in (nova.NOVA_F8_E4M3, nova.NOVA_F8_E5M2):
        x = normal(*shape, seed=sum(shape), dtype=dtype) * torch.logspace(-3, 3, shape[1]).to(dtype)
        x[shape[0] // 2] = 0
        want = plain.quantized(x.T if transposed else x, format, block)
        for src in (x.to(DEV), strided(x)):
            Xq = torch.full((nova.nova_f8_bytes(*want[0].shape, block),), 0xAA, dtype=torch.uint8, device=DEV)
            assert nova.nova_f8_quantize(src, block, format=format, transposed=transposed, Xq=Xq) is Xq
            same_codes(nova.nova_f8_unpack(Xq, *want[0].shape, block, format=format), want)
            if block == 128 or not transposed:
                # everything, padding included, is what packing the same codes writes
                packed = nova.nova_f8_pack(want[0].to(DEV), want[1].to(DEV), block)
                assert torch.equal(packed, Xq)


def test_one_row_for_all():
    x = normal(1, 300, seed=4, dtype=BF16)
    Xq = nova.nova_f8_quantize(x.to(DEV).expand(40, 300), 1)
    same_codes(nova.nova_f8_unpack(Xq, 40, 300, 1), plain.quantized(x.expand(40, 300), 0, 1))


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("transposed", [False, True])
def test_values_beyond_numbers(block, transposed):
    x = normal(40, 700, seed=1)
    x[3, 5], x[7, 200], x[8, 300], x[9, 301] = float("inf"), float("nan"), -float("inf"), 3e38
    x[:, 512:640] = 0
    x[20, 512:640] = 2.0 ** -149                                 # a scale that rounds to zero
    x[21, 512:640] = 700 * 2.0 ** -149                           # ... that is subnormal, and half of what it should be
    x[21, 515] = -2.0 ** -149
    for format in (0, 1):
        want = plain.quantized(x.T if transposed else x, format, block)
        Xq = nova.nova_f8_quantize(x.to(DEV), block, format=format, transposed=transposed)
        same_codes(nova.nova_f8_unpack(Xq, *want[0].shape, block, format=format), want)


def test_every_quotient_of_short_numbers():
    """All positive binary16 numbers in blocks under maxima of every significand: quotients on the borders between codes are frequent among these."""
    every = torch.arange(0, 0x7C00, dtype=torch.int16).view(F16)
    x = every[every <= 1.0].repeat(40)
    x = x[torch.randperm(len(x), generator=torch.Generator().manual_seed(2))][:4096 * 127].view(4096, 127)
    top = (1 + torch.arange(4096) % 1024 / 1024.0).to(F16)
    x = torch.cat([top.unsqueeze(1), x], 1)
    for format in (0, 1):
        same_codes(nova.nova_f8_unpack(nova.nova_f8_quantize(x.to(DEV), 1, format=format), 4096, 128, 1, format=format), plain.quantized(x, format, 1))


def test_every_scale_of_binary32():
    """Random binary32 numbers of all sizes, with scales from the subnormal to the largest."""
    gen = torch.Generator().manual_seed(8)
    x = torch.randint(0, 0x7F800000, (2048, 1), generator=gen, dtype=torch.int32)
    spread = torch.randint(0, 12 << 23, (2048, 512), generator=gen, dtype=torch.int32)
    x = (x - spread).clamp(min=0).view(F32) * (torch.randint(0, 2, (2048, 512), generator=gen) * 2 - 1)
    for format in (0, 1):
        for transposed in (False, True):
            want = plain.quantized(x.T if transposed else x, format, 1)
            same_codes(nova.nova_f8_unpack(nova.nova_f8_quantize(x.to(DEV), 1, format=format, transposed=transposed), *want[0].shape, 1, format=format), want)


def test_layout_as_documented():
    codes, scales = plain.quantized(normal(19, 200, seed=3), 0, 1)
    Xq = nova.nova_f8_pack(codes.to(DEV), scales.to(DEV), 1).cpu()
    raw = codes.view(torch.uint8)
    for r in range(32):
        for k in range(0, 256, 3):
            at = (r // 16 * 2 + k // 128) * 2048 + 1024 * (k % 32 // 16) + 256 * (k % 128 // 32) + 16 * (r % 16) + k % 16
            assert Xq[at] == (raw[r, k] if r < 19 and k < 200 else 0), (r, k)
    tail = Xq[4 * 2048:].view(F32).view(2, 32)
    assert torch.equal(tail[:, :19].T.contiguous(), scales) and not tail[:, 19:].any()
    codes, scales = plain.quantized(normal(140, 300, seed=3), 1, 128)
    T = nova.nova_f8_pack(codes.to(DEV), scales.to(DEV), 128, transposed=True)
    got = nova.nova_f8_unpack(T, 300, 140, 128, format=1)
    assert torch.equal(got[0].cpu().view(torch.uint8), codes.view(torch.uint8).T) and torch.equal(got[1].cpu(), scales.T)
    assert torch.equal(nova.nova_f8_pack(codes.view(torch.uint8).to(DEV), scales.to(DEV), 128, transposed=True), T)


# ---- products ----

def operand(rows, columns, format, block, seed):
    codes, scales = plain.quantized(normal(rows, columns, seed=seed), format, block)
    return (plain.values(codes, scales, block), plain.lowest_values(scales, rows, columns, format, block)), nova.nova_f8_pack(codes.to(DEV), scales.to(DEV), block)


def quantized_operand(v, format, block):
    codes, scales = plain.quantized(v, format, block)
    return plain.values(codes, scales, block), plain.lowest_values(scales, *codes.shape, format, block)


def product(a, b, dtype):
    """(values, bound) of operands as above for results of dtype."""
    want, bound = plain.product(a[0], b[0])
    return want, bound if dtype == F32 else bound + plain.cut_off(a[0], b[0], (a[1], b[1]))


SIZES = [(1, 1, 1), (1, 100, 129), (2, 17, 128), (7, 130, 300), (16, 128, 256), (17, 16, 2048), (33, 259, 1000), (65, 64, 64), (130, 250, 640), (257, 300, 257), (300, 700, 4100)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("blocks", [(1, 128), (1, 1), (128, 1), (128, 128)])
def test_matmul(M, N, K, blocks):
    for case, (fa, fb, dtype) in enumerate([(0, 0, F32), (1, 0, BF16), (0, 1, F16), (1, 1, F32)]):
        a, Aq = operand(M, K, fa, blocks[0], seed=M + K + case)
        b, Bq = operand(N, K, fb, blocks[1], seed=N + K + case + 50)
        want, bound = product(a, b, dtype)
        out = torch.full((M, N + 7), 5.0, dtype=dtype, device=DEV)
        got = nova.nova_f8_matmul(Aq, Bq, M, N, K, block_a=blocks[0], block_b=blocks[1], format_a=fa, format_b=fb, out=out[:, 2:N + 2])
        near(got, want, bound, dtype)
        assert bool((out[:, :2] == 5).all()) and bool((out[:, N + 2:] == 5).all())          # beside the result nothing is written
        again = nova.nova_f8_matmul(Aq, Bq, M, N, K, block_a=blocks[0], block_b=blocks[1], format_a=fa, format_b=fb, dtype=dtype)
        assert torch.equal(again, got)


@pytest.mark.parametrize("M,N,K", SIZES + [(1, 4096, 8200), (520, 1030, 390), (2100, 2200, 1000)])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_matmul_of_whole_numbers(M, N, K, dtype):
    """Codes -1, 0, 1 under scales of 1 and 2 (2^-1): sums are whole multiples of 1/4 below 2^9, which every way of summing and binary16 hold exactly."""
    gen = torch.Generator().manual_seed(M + N + K)

    def draw(rows, block):
        codes = torch.randint(-1, 2, (rows, K), generator=gen) * (torch.randint(0, 4, (rows, K), generator=gen) == 0)
        scales = 2.0 ** torch.randint(-1, 2, (-(-rows // block), -(-K // 128)), generator=gen)
        return codes, scales.float()
    for block_a, block_b in ((1, 128), (1, 1), (128, 1)):
        for fa, fb in ((0, 0), (1, 0), (0, 1), (1, 1)):
            (a, sa), (b, sb) = draw(M, block_a), draw(N, block_b)
            a8, b8 = a.float().to(plain.FORMATS[fa]), b.float().to(plain.FORMATS[fb])
            want = plain.values(a8, sa, block_a) @ plain.values(b8, sb, block_b).T
            assert want.abs().max() < 512
            got = nova.nova_f8_matmul(nova.nova_f8_pack(a8.to(DEV), sa.to(DEV), block_a), nova.nova_f8_pack(b8.to(DEV), sb.to(DEV), block_b), M, N, K, block_a=block_a,
                                      block_b=block_b, format_a=fa, format_b=fb, dtype=dtype)
            assert torch.equal(got.cpu().double(), want), (block_a, block_b, fa, fb)


@pytest.mark.parametrize("M,N,K", [(1, 100, 129), (20, 130, 4100), (150, 259, 300), (300, 700, 257), (2100, 2200, 900)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_bias_relu_add(M, N, K, dtype):
    a, Aq = operand(M, K, 0, 1, seed=1)
    b, Bq = operand(N, K, 0, 128, seed=2)
    bias, before = normal(N, seed=3, dtype=dtype), normal(M, N, seed=4, dtype=dtype)
    want, bound = product(a, b, dtype)
    with_bias = want + bias.double()
    more = 2.0 ** -24 * (with_bias.abs() + bound)                                            # one more addition
    args = (Aq, Bq, M, N, K)
    near(nova.nova_f8_matmul(*args, bias=bias.to(DEV), dtype=dtype), with_bias, bound + more, dtype)
    near(nova.nova_f8_matmul(*args, bias=bias.to(DEV), dtype=dtype, flags=nova.NOVA_FLAG_RELU), with_bias.clamp(min=0.0), bound + more, dtype)
    out = strided(before)
    nova.nova_f8_matmul(*args, bias=bias.to(DEV), out=out, flags=nova.NOVA_FLAG_ADD)
    near(out, with_bias + before.double(), bound + 2 * more + 2.0 ** -23 * before.double().abs(), dtype)


@pytest.mark.parametrize("M,N,K", [(1, 1000, 4096), (1, 4096, 513), (3, 130, 25088), (8, 50, 1), (32, 259, 4096), (64, 300, 300), (100, 128, 128), (260, 520, 900)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_linear(M, N, K, dtype):
    x = normal(M, K, seed=5, dtype=dtype)
    w, Wq = operand(N, K, 0, 128, seed=6)
    bias = normal(N, seed=7, dtype=dtype)
    want, bound = product(quantized_operand(x, 0, 1), w, dtype)
    want = want + bias.double()
    more = 2.0 ** -24 * (want.abs() + bound)
    y = torch.full((M, N + 3), -9.0, dtype=dtype, device=DEV)
    got = nova.nova_f8_linear(strided(x), Wq, N, bias=bias.to(DEV), y=y[:, 1:N + 1], flags=nova.NOVA_FLAG_RELU)
    near(got, want.clamp(min=0.0), bound + more, dtype)
    assert bool((y[:, 0] == -9).all()) and bool((y[:, N + 1:] == -9).all())
    assert torch.equal(nova.nova_f8_linear(x.to(DEV), Wq, N, bias=bias.to(DEV), flags=nova.NOVA_FLAG_RELU), got)


def gradients(dy, y, x, w, format, dtype, dw_dtype):
    d = dy.double() if y is None else torch.where(y > 0, dy.double(), 0.0)
    dx = product(quantized_operand(d, format, 1), (w[0].T, w[1].T), dtype)
    dw = product(quantized_operand(d.T, format, 1), quantized_operand(x.T, 0, 1), dw_dtype)
    return dx, dw, d


@pytest.mark.parametrize("M,N,K", [(1, 5, 3), (1, 1000, 4096), (32, 300, 257), (17, 128, 128), (130, 259, 300), (300, 131, 700)])
@pytest.mark.parametrize("dtype,format,relu", [(F32, 0, True), (F16, 1, True), (BF16, 0, False), (F32, 1, False)])
def test_backward(M, N, K, dtype, format, relu):
    dy, x = normal(M, N, seed=8, dtype=dtype), normal(M, K, seed=9, dtype=dtype)
    y = normal(M, N, seed=10, dtype=dtype).clamp(min=0.0) if relu else None
    codes, scales = plain.quantized(normal(N, K, seed=11), 0, 128)
    w, WqT = (plain.values(codes, scales, 128), plain.lowest_values(scales, N, K, 0, 128)), nova.nova_f8_pack(codes.to(DEV), scales.to(DEV), 128, transposed=True)
    (dx, dx_bound), (dw, dw_bound), d = gradients(dy, y, x, w, format, dtype, F32)
    on = dict(y=None if y is None else strided(y), format=format)
    got = nova.nova_f8_linear_backward(strided(dy), WqT, strided(x), **on)
    near(got[0], dx, dx_bound, dtype)
    near(got[1], dw, dw_bound, F32)
    # 128 rows are added in binary32, those sums in binary64
    near(got[2], d.sum(0), 128 * 2.0 ** -24 * d.abs().sum(0), F32)
    # the parts one by one, and added to what is there
    assert torch.equal(nova.nova_f8_linear_backward(dy.to(DEV), WqT, None, K=K, need_dbias=False, y=None if y is None else y.to(DEV), format=format)[0], got[0])
    only = nova.nova_f8_linear_backward(dy.to(DEV), None, x.to(DEV), y=None if y is None else y.to(DEV), format=format)
    assert only[0] is None and torch.equal(only[1], got[1]) and torch.equal(only[2], got[2])
    before, before_bias = normal(N, K, seed=12), normal(N, seed=13)
    dw_out, db_out = strided(before), before_bias.to(DEV)
    nova.nova_f8_linear_backward(dy.to(DEV), None, x.to(DEV), y=None if y is None else y.to(DEV), format=format, dw=dw_out, dbias=db_out, flags=nova.NOVA_FLAG_ADD)
    near(dw_out, dw + before.double(), dw_bound, F32)
    near(db_out, d.sum(0) + before_bias.double(), 128 * 2.0 ** -24 * d.abs().sum(0), F32)
    if dtype != F32:
        (_, _), (dw, dw_bound), _ = gradients(dy, y, x, w, format, dtype, dtype)
        near(nova.nova_f8_linear_backward(dy.to(DEV), None, x.to(DEV), y=None if y is None else y.to(DEV), format=format, dw_dtype=dtype)[1], dw, dw_bound, dtype)
        with pytest.raises(nova.NovaError):
            nova.nova_f8_linear_backward(dy.to(DEV), None, x.to(DEV), dw_dtype=F16 if dtype == BF16 else BF16)
    if format == 0:
        bias_only = nova.nova_f8_linear_backward(dy.to(DEV), None, None, K=K, y=None if y is None else y.to(DEV))
        assert bias_only[:2] == (None, None) and torch.equal(bias_only[2], got[2])


def whole_numbers(rows, columns, seed):
    """Whole numbers up to 7, one of them in every 128 neighbours in both directions: scales are 2^-6 (2^-13), every code is exact in either format's four (three) bits."""
    v = torch.randint(-4, 5, (rows, columns), generator=torch.Generator().manual_seed(seed)).float()
    r, c = torch.arange(rows).unsqueeze(1), torch.arange(columns)
    v[(r + c) % 32 == 0] = 7.0
    return v


def test_gradients_against_differences():
    """On whole numbers nothing is rounded, the layer is linear in x, W and b, and the gradients are its differences exactly."""
    M, N, K = 40, 64, 160
    x, w, dy, b = whole_numbers(M, K, 1), whole_numbers(N, K, 2), whole_numbers(M, N, 3), whole_numbers(1, N, 4)[0]

    def layer(x, w, b):
        return nova.nova_f8_linear(x.to(DEV), nova.nova_f8_quantize(w.to(DEV), 128), N, bias=b.to(DEV)).double().cpu()
    dx, dw, db = (g.double().cpu() for g in nova.nova_f8_linear_backward(dy.to(DEV), nova.nova_f8_quantize(w.to(DEV), 128, transposed=True), x.to(DEV), format=0))
    base = layer(x, w, b)
    assert torch.equal(base, x.double() @ w.double().T + b.double())
    for i, j in ((0, 1), (5, 77), (39, 130)):
        step = x.clone()
        step[i, j] += 1 if abs(x[i, j]) < 7 else 0
        assert ((layer(step, w, b) - base) * dy).sum() == dx[i, j] * (step - x)[i, j]
        step = w.clone()
        step[i, j] += 1 if abs(w[i, j]) < 7 else 0
        assert ((layer(x, step, b) - base) * dy).sum() == dw[i, j] * (step - w)[i, j]
        step = b.clone()
        step[i] += 1
        assert ((layer(x, w, step) - base) * dy).sum() == db[i]


@pytest.mark.parametrize("M", [1, 20, 200])
def test_nan_and_infinity_stay_in_their_rows(M):
    N, K = 150, 300
    x = normal(M, K, seed=1)
    x[M // 2, 140] = float("inf")
    w, Wq = operand(N, K, 0, 128, seed=2)
    y = nova.nova_f8_linear(x.to(DEV), Wq, N, flags=nova.NOVA_FLAG_RELU).cpu()
    assert bool(y[M // 2].isnan().all()) and bool(y[[m for m in range(M) if m != M // 2]].isfinite().all())
    dy = normal(M, N, seed=3)
    dy[M // 2, 3] = float("nan")
    gate = torch.ones(M, N)
    gate[M // 2, 3] = 0.0                                        # a closed place hides it
    _, dw, db = nova.nova_f8_linear_backward(dy.to(DEV), None, normal(M, K, seed=4).to(DEV), y=gate.to(DEV))
    assert bool(dw.isfinite().all()) and bool(db.isfinite().all())
    dx, dw, db = nova.nova_f8_linear_backward(dy.to(DEV), nova.nova_f8_quantize(normal(N, K, seed=2).to(DEV), 128, transposed=True), normal(M, K, seed=4).to(DEV))
    assert bool(dx[M // 2].isnan().all()) and bool(dw[3].isnan().all()) and bool(db[3].isnan())
    assert int(dx.isnan().any(1).sum()) == 1 and int(dw.isnan().any(1).sum()) == 1 and int(db.isnan().sum()) == 1


def test_no_rows():
    w, Wq = operand(30, 200, 0, 128, seed=1)
    x, dy = torch.empty((0, 200), device=DEV), torch.empty((0, 30), device=DEV)
    assert nova.nova_f8_linear(x, Wq, 30).shape == (0, 30)
    dw, db = torch.full((30, 200), 3.0, device=DEV), torch.full((30,), 3.0, device=DEV)
    nova.nova_f8_linear_backward(dy, None, x, dw=dw, dbias=db, flags=nova.NOVA_FLAG_ADD)
    assert bool((dw == 3).all()) and bool((db == 3).all())
    nova.nova_f8_linear_backward(dy, None, x, dw=dw, dbias=db)
    assert not dw.any() and not db.any()


def test_rows_that_the_relu_closed():
    """Rows and columns of the gradient that the gate closes whole: scales of zero."""
    M, N, K = 140, 200, 150
    dy, x = normal(M, N, seed=1).to(DEV), normal(M, K, seed=2).to(DEV)
    y = torch.ones((M, N), device=DEV)
    y[5], y[:, 7] = 0.0, -1.0
    dx, dw, db = nova.nova_f8_linear_backward(dy, nova.nova_f8_quantize(normal(N, K, seed=3).to(DEV), 128, transposed=True), x, y=y)
    assert not dx[5].any() and not dw[7].any() and db[7] == 0 and bool(dx.isfinite().all())


@pytest.mark.parametrize("M,N,K", [(1, 1000, 4096), (32, 520, 2100), (300, 260, 513)])
def test_graph_of_a_training_step(M, N, K):
    """Forward and backward on another stream, captured and replayed with new inputs, against the calls; two graphs share their workspace."""
    w = normal(N, K, seed=1)
    Wq, WqT = nova.nova_f8_quantize(w.to(DEV), 128), nova.nova_f8_quantize(w.to(DEV), 128, transposed=True)
    x, dy = normal(M, K, seed=2, dtype=BF16).to(DEV), normal(M, N, seed=3, dtype=BF16).to(DEV)
    ws = torch.full((max(nova.nova_f8_linear_workspace_bytes(M, N, K, BF16), nova.nova_f8_linear_backward_workspace_bytes(M, N, K, BF16)),), 0xFF, dtype=torch.uint8,
                    device=DEV)
    y, dx = torch.empty((M, N), dtype=BF16, device=DEV), torch.empty((M, K), dtype=BF16, device=DEV)
    dw, db = torch.empty((N, K), device=DEV), torch.empty((N,), device=DEV)

    def forward():
        nova.nova_f8_linear(x, Wq, N, y=y, flags=nova.NOVA_FLAG_RELU, workspace=ws)

    def backward():
        nova.nova_f8_linear_backward(dy, WqT, x, y=y, dx=dx, dw=dw, dbias=db, workspace=ws)
    graphs = []
    for step in (forward, backward):
        graphs.append(torch.cuda.CUDAGraph())
        torch.cuda.synchronize()
        with torch.cuda.graph(graphs[-1]):
            step()
    for seed in range(3):
        x.copy_(normal(M, K, seed=20 + seed, dtype=BF16))
        dy.copy_(normal(M, N, seed=30 + seed, dtype=BF16))
        forward()
        backward()
        want = [t.clone() for t in (y, dx, dw, db)]
        for t in (y, dx, dw, db):
            t.fill_(7.0)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((y, dx, dw, db), want))
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            other = nova.nova_f8_linear(x, Wq, N, flags=nova.NOVA_FLAG_RELU)
        side.synchronize()
        assert torch.equal(other, want[0])


def test_refusals_of_the_binding():
    w, Wq = operand(30, 200, 0, 128, seed=1)
    x = normal(4, 200).to(DEV)
    with pytest.raises(ValueError):
        nova.nova_f8_linear(x.T.contiguous().T, Wq, 30)                                  # elements of a row apart
    with pytest.raises(ValueError):
        nova.nova_f8_linear(x, Wq, 30, bias=torch.zeros(30, dtype=F16, device=DEV))
    with pytest.raises(nova.NovaError):
        nova.nova_f8_linear(x, Wq[:-16], 30)
    with pytest.raises(nova.NovaError):
        nova.nova_f8_linear(x, Wq, 30, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(nova.NovaError):
        nova.nova_f8_linear(x, Wq, 30, flags=nova.NOVA_FLAG_POOL2)
    with pytest.raises(ValueError):
        nova.nova_f8_matmul(Wq, Wq, 30, 30, 200, block_a=128, flags=nova.NOVA_FLAG_ADD)
    with pytest.raises(ValueError):
        nova.nova_f8_unpack(Wq, 30, 200, 128, format=7)
    with pytest.raises(ValueError):
        nova.nova_f8_linear_backward(normal(4, 30).to(DEV), None, x, dx=torch.empty_like(x))
    with pytest.raises(ValueError):
        nova.nova_f8_linear_backward(normal(4, 30).to(DEV), None, x, flags=nova.NOVA_FLAG_ADD)
