"""The calls that train fully connected layers, as a table of cases that can be timed and compared: layers in 8-bit floating point with a
scale per block of 128 (forward, and the gradients of input, weights and bias), products of operands that are laid out already, the
quantisation itself, and dropout whose mask comes from a counter and is never stored (forward and gradient).

    own                  False: the operators in elementary torch operations; True: through the library
    listed()             the cases that are always looked at
    draw(rng)            one more of the same ranges
    prepare(case, seed)  what a program has in hand before the call
    run(state)           one pass; returns its outputs
    work(case)           bytes and operations a pass cannot do without
    exact(case, seed)    the same outputs in 64 bits
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST_CODE = {"e4m3": 448.0, "e5m2": 57344.0}
BLOCK = 128

LARGEST_PRODUCTS = 8192 * 8192 * 8192                 # multiply-adds of the largest listed case
LARGEST_MATRIX = 4096 * 25088                         # weights of the widest listed layer
LARGEST_DROPPED = 8192 * 8192                         # elements of the largest listed dropout


def _linear(name, M, N, K, dtype, bias=False, relu=False):
    return dict(name=name, kind="linear", M=M, N=N, K=K, dtype=dtype, bias=bias, relu=relu)


def _backward(name, M, N, K, dtype, format, dw, relu=False):
    return dict(name=name, kind="linear_backward", M=M, N=N, K=K, dtype=dtype, format=format, dw=dw, relu=relu)


def _matmul(name, M, N, K, dtype, formats, block_b):
    return dict(name=name, kind="matmul", M=M, N=N, K=K, dtype=dtype, format_a=formats[0], format_b=formats[1], block_b=block_b)


def _quantize(name, rows, columns, dtype, format, block, transposed):
    return dict(name=name, kind="quantize", rows=rows, columns=columns, dtype=dtype, format=format, block=block, transposed=transposed)


def _dropout(name, rows, columns, dtype, p, relu=False, residual=False):
    return dict(name=name, kind="dropout", rows=rows, columns=columns, dtype=dtype, p=p, relu=relu, residual=residual)


def listed():
    return [
        # the layer that gives the 1000 classes of one image: the smallest call, where latency counts
        _linear("classes_one_image_f32", 1, 1000, 4096, "f32", bias=True),
        # the first fully connected layer behind the 13-layer stack (512 x 7 x 7 features), one image: the weights are read once
        _linear("fc1_one_image_f16", 1, 4096, 25088, "f16", bias=True, relu=True),
        # the same layer at the batch the stack is quoted on
        _linear("fc1_batch_f16", 32, 4096, 25088, "f16", bias=True, relu=True),
        # a square projection of many tokens at once, quantised on the way
        _linear("many_rows_bf16", 4096, 8192, 8192, "bf16"),
        # two operands with a scale per row and block, as of a gradient's product with what was saved; sizes that are whole numbers of nothing
        _matmul("odd_sizes_f32", 517, 5001, 2055, "f32", ("e5m2", "e4m3"), 1),
        # tokens laid out once for several projections, weights with a scale per 128 x 128: the matrix units bind; the largest call
        _matmul("square_bf16", 8192, 8192, 8192, "bf16", ("e4m3", "e4m3"), 128),
        # the backward pass through the second fully connected layer and its ReLU at batch 32, the weights' gradient in binary32 for an optimizer's own copy
        _backward("fc2_backward_f16", 32, 4096, 4096, "f16", "e5m2", "f32", relu=True),
        # ... and through a wide projection of many tokens, the weights' gradient in the layer's type
        _backward("many_rows_backward_bf16", 4096, 4096, 16384, "bf16", "e4m3", "bf16"),
        # what a training step does to the first layer's weights after their update
        _quantize("fc1_weights_f16", 4096, 25088, "f16", "e4m3", 128, False),
        # a batch's activations for the product that gives the weights' gradient, sizes that are whole numbers of nothing
        _quantize("odd_activations_bf16", 4099, 5003, "bf16", "e4m3", 1, True),
        # dropout behind the second layer's ReLU at batch 32, and its gradient
        _dropout("fc2_dropout_f16", 32, 4096, "f16", 0.5, relu=True),
        # dropout of a branch that is added to what went round it, many tokens, and its gradient
        _dropout("branch_dropout_bf16", 8192, 8192, "bf16", 0.1, residual=True),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_backward", "linear_backward", "matmul", "quantize", "dropout"])
    dtype = rng.choice(["f32", "f16", "f16", "bf16", "bf16"])
    if kind == "quantize":
        while True:
            rows, columns = _log_uniform(rng, 1, 32768), _log_uniform(rng, 1, 32768)
            if rows * columns <= LARGEST_MATRIX // (2 if dtype == "f32" else 1):
                break
        return dict(kind=kind, rows=rows, columns=columns, dtype=dtype, format=rng.choice(["e4m3", "e4m3", "e5m2"]), block=rng.choice([1, 128]),
                    transposed=rng.random() < 0.5)
    if kind == "dropout":
        while True:
            rows, columns = _log_uniform(rng, 1, 65536), _log_uniform(rng, 1, 65536)
            if rows * columns <= LARGEST_DROPPED // (2 if dtype == "f32" else 1):
                break
        relu = rng.random() < 0.4
        return dict(kind=kind, rows=rows, columns=columns, dtype=dtype, p=rng.choice([0.0, 0.05, 0.1, 0.3, 0.5, 0.9]), relu=relu,
                    residual=not relu and rng.random() < 0.5)
    while True:
        M = 1 if kind == "linear" and rng.random() < 0.3 else _log_uniform(rng, 1, 8192)
        N, K = _log_uniform(rng, 100, 25088), _log_uniform(rng, 100, 25088)
        if rng.random() < 0.5:
            N, K = max(128, N // 128 * 128), max(128, K // 128 * 128)
        if N * K <= LARGEST_MATRIX and M * N * K <= LARGEST_PRODUCTS // (2 if kind == "linear_backward" else 1):
            break
    if kind == "linear":
        return dict(kind=kind, M=M, N=N, K=K, dtype=dtype, bias=rng.random() < 0.5, relu=rng.random() < 0.4)
    if kind == "matmul":
        return dict(kind=kind, M=M, N=N, K=K, dtype=dtype, format_a=rng.choice(["e4m3", "e5m2"]), format_b=rng.choice(["e4m3", "e4m3", "e5m2"]),
                    block_b=rng.choice([1, 128]))
    return dict(kind=kind, M=M, N=N, K=K, dtype=dtype, format=rng.choice(["e4m3", "e5m2"]), dw=rng.choice(["f32", dtype]), relu=rng.random() < 0.4)


# ---- blocks of 128 (the plain form of the quantisation) ----

def _blocks(v, block):
    """v [rows, columns] in 32 bits, padded with zeros to whole blocks: [rows of blocks, block, chunks, 128]."""
    rows, columns = v.shape
    padded = torch.nn.functional.pad(v, (0, -columns % BLOCK, 0, -rows % block))
    return padded.view(padded.shape[0] // block, block, padded.shape[1] // BLOCK, BLOCK)


def _quantized(v, format, block):
    """(codes [rows, columns], scales [ceil(rows / block), ceil(columns / 128)]): scale = max|v| / largest code, code = v / scale rounded."""
    rows, columns = v.shape
    b = _blocks(v.float(), block)
    # (quotients of short significands lie on borders between codes often: a division by a number must not become a product with its inverse)
    scales = (b.abs().amax((1, 3)).double() / LARGEST_CODE[format]).float()
    s = scales[:, None, :, None]
    codes = torch.where(s > 0, b / s, 0.0).to(FORMATS[format])
    return codes.view(b.shape[0] * block, -1)[:rows, :columns].contiguous(), scales


def _values(codes, scales, block):
    rows, columns = codes.shape
    return codes.float() * scales.repeat_interleave(block, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :columns]


# ---- counters to random words (Philox 4x32-10: Salmon, Moraes, Dror, Shaw, SC 2011) ----

def _philox(c, key):
    """Four tensors of 32-bit words (int64) -> four."""
    low = 0xFFFFFFFF
    k0, k1 = key & low, key >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57           # (both are below 2^64; int64 keeps all of their bits)
        c = [(b >> 32 & low) ^ c[1] ^ k0, b & low, (a >> 32 & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c


def _halves(rows, columns, seed, offset, second):
    """16 random bits per element: eight elements of a row share a counter (column / 8, row, offset), two to a word, the low half first."""
    groups = -(-columns // 8)
    column = torch.arange(groups, device=DEV).expand(rows, groups)
    row = torch.arange(rows, device=DEV).unsqueeze(1).expand(rows, groups) + (1 << 31) * second
    zero = torch.zeros_like(column)
    words = torch.stack(_philox([column, row, zero + (offset & 0xFFFFFFFF), zero + (offset >> 32)], seed), 2)
    return torch.stack([words & 0xFFFF, words >> 16], 3).view(rows, groups * 8)[:, :columns]


def _kept(s):
    """Whether an element stays: its 32 random bits are at least p 2^32."""
    case = s["case"]
    args = (case["rows"], case["columns"], s["seed"], s["offset"])
    return (_halves(*args, 0) << 16 | _halves(*args, 1)) >= int(case["p"] * 2.0 ** 32 + 0.5)


# ---- inputs ----

def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=gen)

    def activations(M, K):
        # a few inputs are much larger than the others, as in trained networks: what blocks have their own scales for
        loud = 1.0 + 19.0 * (torch.rand((K,), device=DEV, generator=gen) < 0.005)
        return (normal(M, K) * loud).to(dtype)

    if case["kind"] == "dropout":
        R, C = case["rows"], case["columns"]
        s = dict(x=normal(R, C).to(dtype), dy=(normal(R, C) / R).to(dtype), residual=normal(R, C).to(dtype) if case["residual"] else None)
        return dict(s, seed=(seed * 0x9E3779B97F4A7C15 + 1) % 2 ** 63, offset=seed % 1000)
    if case["kind"] == "quantize":
        return dict(x=activations(case["rows"], case["columns"]))
    M, N, K = case["M"], case["N"], case["K"]
    if case["kind"] == "matmul":
        a, sa = _quantized(activations(M, K), case["format_a"], 1)
        b, sb = _quantized(normal(N, K) * math.sqrt(2.0 / K), case["format_b"], case["block_b"])
        return dict(a=a, sa=sa, b=b, sb=sb)
    w, sw = _quantized(normal(N, K) * math.sqrt(2.0 / K), "e4m3", 128)
    if case["kind"] == "linear":
        return dict(x=activations(M, K), w=w, sw=sw, bias=(0.1 * normal(N)).to(dtype) if case["bias"] else None)
    return dict(x=activations(M, K), w=w, sw=sw, dy=(normal(M, N) / M).to(dtype), y=torch.relu(normal(M, N)).to(dtype) if case["relu"] else None)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["kind"], s["case"] = case["kind"], case
    if own:
        from paper_2512_18453_amd import nova
        dtype, kind = DTYPES[case["dtype"]], case["kind"]
        if kind in ("linear", "linear_backward"):
            M, N, K = case["M"], case["N"], case["K"]
            s["Wq"] = nova.nova_f8_pack(s["w"], s["sw"], 128, transposed=kind == "linear_backward")
            if kind == "linear":
                s["out"] = torch.empty((M, N), dtype=dtype, device=DEV)
                need = nova.nova_f8_linear_workspace_bytes(M, N, K, dtype)
            else:
                s["dx"] = torch.empty((M, K), dtype=dtype, device=DEV)
                s["dw"], s["dbias"] = torch.empty((N, K), dtype=DTYPES[case["dw"]], device=DEV), torch.empty((N,), device=DEV)
                need = nova.nova_f8_linear_backward_workspace_bytes(M, N, K, dtype)
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        elif kind == "matmul":
            M, N, K = case["M"], case["N"], case["K"]
            s["Aq"], s["Bq"] = nova.nova_f8_pack(s["a"], s["sa"], 1), nova.nova_f8_pack(s["b"], s["sb"], case["block_b"])
            s["out"] = torch.empty((M, N), dtype=dtype, device=DEV)
            s["workspace"] = torch.empty(nova.nova_f8_matmul_workspace_bytes(M, N, K, 1, case["block_b"], dtype), dtype=torch.uint8, device=DEV)
        elif kind == "quantize":
            rows, columns = (case["columns"], case["rows"]) if case["transposed"] else (case["rows"], case["columns"])
            s["Xq"] = torch.empty(nova.nova_f8_bytes(rows, columns, case["block"]), dtype=torch.uint8, device=DEV)
        else:
            s["out"], s["dx"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    return s


# ---- the plain forms ----

def _plain_linear(s):
    case = s["case"]
    y = _values(*_quantized(s["x"], "e4m3", 1), 1) @ _values(s["w"], s["sw"], 128).T
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["relu"]:
        y = torch.where(y < 0, 0.0, y)
    return y.to(s["x"].dtype)


def _plain_linear_backward(s):
    case = s["case"]
    d = s["dy"].float()
    if s["y"] is not None:
        d = torch.where(s["y"] > 0, d, 0.0)
    dx = _values(*_quantized(d, case["format"], 1), 1) @ _values(s["w"], s["sw"], 128)
    # the weights' gradient sums over the rows, so there the blocks run along them
    dw = _values(*_quantized(d.T, case["format"], 1), 1) @ _values(*_quantized(s["x"].T, "e4m3", 1), 1).T
    return dict(dx=dx.to(s["dy"].dtype), dw=dw.to(DTYPES[case["dw"]]), dbias=d.sum(0, dtype=torch.float64).float())


def _plain_matmul(s):
    return (_values(s["a"], s["sa"], 1) @ _values(s["b"], s["sb"], s["case"]["block_b"]).T).to(DTYPES[s["case"]["dtype"]])


def _plain_quantize(s):
    case = s["case"]
    codes, scales = _quantized(s["x"].T if case["transposed"] else s["x"], case["format"], case["block"])
    return dict(codes=codes, scales=scales)


def _plain_dropout(s):
    case = s["case"]
    keep, factor = _kept(s), 1.0 / (1.0 - case["p"])
    x = s["x"].float()
    if case["relu"]:
        x = torch.where(x < 0, 0.0, x)
    y = torch.where(keep, x * factor, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    dx = torch.where(keep & (s["x"] > 0) if case["relu"] else keep, s["dy"].float() * factor, 0.0)
    return dict(y=y.to(s["x"].dtype), dx=dx.to(s["x"].dtype))


def run(s):
    if not own:
        return {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "matmul": _plain_matmul, "quantize": _plain_quantize,
                "dropout": _plain_dropout}[s["kind"]](s)
    from paper_2512_18453_amd import nova
    case, kind = s["case"], s["kind"]
    formats = {"e4m3": nova.NOVA_F8_E4M3, "e5m2": nova.NOVA_F8_E5M2}
    flags = nova.NOVA_FLAG_RELU if case.get("relu") else 0
    if kind == "linear":
        return nova.nova_f8_linear(s["x"], s["Wq"], case["N"], bias=s["bias"], y=s["out"], flags=flags, workspace=s["workspace"])
    if kind == "linear_backward":
        dx, dw, dbias = nova.nova_f8_linear_backward(s["dy"], s["Wq"], s["x"], y=s["y"], format=formats[case["format"]], dx=s["dx"], dw=s["dw"],
                                                     dbias=s["dbias"], workspace=s["workspace"])
        return dict(dx=dx, dw=dw, dbias=dbias)
    if kind == "matmul":
        return nova.nova_f8_matmul(s["Aq"], s["Bq"], case["M"], case["N"], case["K"], block_a=1, block_b=case["block_b"],
                                   format_a=formats[case["format_a"]], format_b=formats[case["format_b"]], out=s["out"], workspace=s["workspace"])
    if kind == "quantize":
        Xq = nova.nova_f8_quantize(s["x"], case["block"], format=formats[case["format"]], transposed=case["transposed"], Xq=s["Xq"])
        rows, columns = (case["columns"], case["rows"]) if case["transposed"] else (case["rows"], case["columns"])
        codes, scales = nova.nova_f8_unpack(Xq, rows, columns, case["block"], format=formats[case["format"]])
        return dict(codes=codes, scales=scales)
    y = nova.nova_dropout(s["x"], case["p"], s["seed"], offset=s["offset"], residual=s["residual"], flags=flags, y=s["out"])
    dx = nova.nova_dropout_backward(s["dy"], case["p"], s["seed"], offset=s["offset"], gate=s["x"] if case["relu"] else None, dx=s["dx"])
    return dict(y=y, dx=dx)


def work(case):
    es = SIZES[case["dtype"]]
    if case["kind"] == "dropout":
        # forward: x (and the residual) in, y out; gradient: dy (and what the ReLU saw) in, dx out
        n = case["rows"] * case["columns"]
        return {"bytes": n * es * (4 + case["residual"] + case["relu"]), "flops": 0.0}
    if case["kind"] == "quantize":
        # the layout is written, and read and written once more as rows of codes
        n = case["rows"] * case["columns"]
        return {"bytes": n * (es + 3.0), "flops": 0.0}
    M, N, K = case["M"], case["N"], case["K"]
    scales = lambda rows, columns, block: 4.0 * -(-rows // block) * -(-columns // BLOCK)  # noqa: E731
    if case["kind"] == "linear":
        return {"bytes": N * K + scales(N, K, 128) + (M * K + M * N) * es + N * es * case["bias"], "flops": 2.0 * M * N * K}
    if case["kind"] == "matmul":
        return {"bytes": M * K + N * K + scales(M, K, 1) + scales(N, K, case["block_b"]) + M * N * es, "flops": 2.0 * M * N * K}
    return {"bytes": N * K + scales(N, K, 128) + (M * N * (1 + case["relu"]) + 2 * M * K) * es + N * K * SIZES[case["dw"]] + 4 * N, "flops": 4.0 * M * N * K}


# ---- the definition in 64 bits ----

def _exact_codes(v, scale, format):
    """v / scale, rounded to 32 bits and then to the code: a whole number of steps of 2^-3 (2^-2) of its power of two, ties to even."""
    bits, lowest = (3, -6) if format == "e4m3" else (2, -14)
    q = (v / scale.clamp(min=1e-300)).float().double()
    exponent = (torch.frexp(q).exponent.to(torch.int64) - 1).clamp(min=lowest) - bits
    step = (exponent + 1023 << 52).view(torch.float64)
    return (torch.round(q / step) * step).clamp(-LARGEST_CODE[format], LARGEST_CODE[format])


def _exact_quantized(v, format, block):
    """The values of the codes, and the scale of every one of them, both [rows, columns]; the scales by block."""
    rows, columns = v.shape
    v = v.double()
    chunks, bands = range(0, columns, BLOCK), -(-rows // block)
    by_band = torch.zeros((bands * block, columns), dtype=torch.float64, device=DEV)
    by_band[:rows] = v.abs()
    top = torch.stack([by_band[:, c:c + BLOCK].amax(1).view(bands, block).amax(1) for c in chunks], 1)
    del by_band
    scales = (top / LARGEST_CODE[format]).float().double()
    every = torch.empty_like(v)
    for i, c in enumerate(chunks):
        every[:, c:c + BLOCK] = scales[:, i].repeat_interleave(block)[:rows, None]
    return _exact_codes(v, every, format), every, scales


def _exact_values(codes, scales, block):
    out = codes.double()
    for i, c in enumerate(range(0, codes.shape[1], BLOCK)):
        out[:, c:c + BLOCK] *= scales[:, i].double().repeat_interleave(block)[:codes.shape[0], None]
    return out


def _exact_kept(case, seed, offset):
    """The same random bits from numpy's unsigned words."""
    R, groups, low = case["rows"], -(-case["columns"] // 8), np.uint64(0xFFFFFFFF)
    halves = []
    for second in (0, 1):
        c = [np.tile(np.arange(groups, dtype=np.uint64), R), np.repeat(np.arange(R, dtype=np.uint64), groups) | np.uint64(second << 31),
             np.full(R * groups, offset & 0xFFFFFFFF, np.uint64), np.full(R * groups, offset >> 32, np.uint64)]
        for r in range(10):
            k0, k1 = np.uint64(((seed & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF), np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(b >> np.uint64(32)) ^ c[1] ^ k0, b & low, (a >> np.uint64(32)) ^ c[3] ^ k1, a & low]
        halves.append(np.stack(c, 1).astype("<u4").view("<u2").reshape(R, groups * 8)[:, :case["columns"]].astype(np.uint32))
    u = torch.from_numpy((halves[0] << np.uint32(16) | halves[1]).astype(np.float64)).to(DEV)
    return u >= math.floor(case["p"] * 2.0 ** 32 + 0.5)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "dropout":
        keep = _exact_kept(case, s["seed"], s["offset"]).double()
        open_ = (s["x"].double() > 0).double() if case["relu"] else 1.0
        y = s["x"].double() * open_ * keep / (1.0 - case["p"])
        return dict(y=y if s["residual"] is None else y + s["residual"].double(), dx=s["dy"].double() * open_ * keep / (1.0 - case["p"]))
    if kind == "quantize":
        codes, _, scales = _exact_quantized(s["x"].T if case["transposed"] else s["x"], case["format"], case["block"])
        return dict(codes=codes, scales=scales)
    if kind == "matmul":
        return _exact_values(s["a"], s["sa"], 1) @ _exact_values(s["b"], s["sb"], case["block_b"]).T
    w = _exact_values(s["w"], s["sw"], 128)
    if kind == "linear":
        codes, every, _ = _exact_quantized(s["x"], "e4m3", 1)
        y = (codes * every) @ w.T
        if s["bias"] is not None:
            y += s["bias"].double()
        return y.clamp(min=0.0) if case["relu"] else y
    d = s["dy"].double()
    if s["y"] is not None:
        d = d * (s["y"].double() > 0)
    codes, every, _ = _exact_quantized(d, case["format"], 1)
    dx = (codes * every) @ w
    codes, every, _ = _exact_quantized(d.T, case["format"], 1)
    left = codes * every
    codes, every, _ = _exact_quantized(s["x"].T, "e4m3", 1)
    return dict(dx=dx, dw=left @ (codes * every).T, dbias=d.sum(0))
