"""The calls of the operators behind a convolution stack, as a table of cases that can be timed and compared: layers whose weights
are stored in 4 bits with a scale per group (forward, and the gradient of their input), and log probabilities with entropy and
top alternatives (forward, and the gradient of the logits).

    own                  False: the operators in elementary torch operations; True: through the library
    listed()             the cases that are always looked at
    draw(rng)            one more of the same ranges
    prepare(case, seed)  what a program has in hand before the call
    run(state)           one pass; returns its outputs
    work(case)           bytes and operations a pass cannot do without
    exact(case, seed)    the same outputs in 64 bits
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}

LARGEST_PRODUCTS = 1024 * 8192 * 8192                 # multiply-adds of the largest listed layer
LARGEST_WEIGHTS = 100003 * 2055                       # weights of the widest listed layer
LARGEST_LOGITS = 1024 * 131072                        # logits of the largest listed call


def _linear(name, M, N, K, group, dtype, bias=False, relu=False, backward=False):
    return dict(name=name, kind="linear_backward" if backward else "linear", M=M, N=N, K=K, group=group, dtype=dtype, bias=bias, relu=relu)


def _logprobs(name, R, V, dtype, top=0, mask="none", scale=1.0, backward=False):
    return dict(name=name, kind="logprobs_backward" if backward else "logprobs", R=R, V=V, dtype=dtype, top=top, mask=mask, scale=scale)


def listed():
    return [
        # the first fully connected layer behind the 13-layer stack (512 x 7 x 7 features), one image: the weights are read once
        _linear("fc1_one_image_f16", 1, 4096, 25088, 128, "f16", bias=True, relu=True),
        # the same layer at the batch the stack is quoted on
        _linear("fc1_batch_f16", 32, 4096, 25088, 128, "f16", bias=True, relu=True),
        # the layer that gives the 1000 classes of one image, in binary32: the smallest call
        _linear("classes_one_image_f32", 1, 1000, 4096, 64, "f32", bias=True),
        # a vocabulary's logits of a few sequences that each ask for one token; sizes that are whole numbers of nothing, the smallest groups
        _linear("vocabulary_few_bf16", 5, 100003, 2055, 32, "bf16"),
        # a square projection of many tokens at once: the matrix units bind, not the weights
        _linear("many_rows_bf16", 1024, 8192, 8192, 128, "bf16"),
        # the gradient that goes back through the second fully connected layer and its ReLU at batch 32
        _linear("fc2_backward_f16", 32, 4096, 4096, 128, "f16", relu=True, backward=True),
        # the gradient through a wide projection of many tokens
        _linear("many_rows_backward_bf16", 512, 4096, 16384, 128, "bf16", backward=True),
        # what a classifier answers for a batch of images: the class's log probability, entropy, five best classes
        _logprobs("classes_f16", 32, 1000, "f16", top=5),
        # one generated token over a large vocabulary, some of it not allowed, twenty alternatives, a temperature
        _logprobs("one_token_bf16", 1, 131071, "bf16", top=20, mask="rows", scale=1.25),
        # scoring given tokens of a long text: the largest call
        _logprobs("scoring_bf16", 1024, 131072, "bf16", top=8),
        # the training step of a classifier's last layer: gradient of the class log probabilities with an entropy term
        _logprobs("classes_backward_f32", 32, 1000, "f32", backward=True),
        # the gradient of the log probabilities of a long text
        _logprobs("scoring_backward_bf16", 1024, 131072, "bf16", backward=True),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_backward", "logprobs", "logprobs", "logprobs_backward"])
    dtype = rng.choice(["f32", "f16", "f16", "bf16", "bf16"])
    if kind.startswith("linear"):
        # one token half of the time, as a serving program calls it; layers from a few hundred weights to the widest listed
        M = 1 if kind == "linear" and rng.random() < 0.4 else _log_uniform(rng, 1, 1024)
        while True:
            N, K = _log_uniform(rng, 100, 100003), _log_uniform(rng, 100, 25088)
            if rng.random() < 0.5:
                N, K = max(128, N // 128 * 128), max(128, K // 128 * 128)
            if N * K <= LARGEST_WEIGHTS and M * N * K <= LARGEST_PRODUCTS // (2 if kind == "linear_backward" else 1):
                break
        return dict(kind=kind, M=M, N=N, K=K, group=rng.choice([32, 64, 128, 128]), dtype=dtype, bias=kind == "linear" and rng.random() < 0.5,
                    relu=rng.random() < 0.4)
    largest = LARGEST_LOGITS // (2 if dtype == "f32" else 1)
    while True:
        R, V = _log_uniform(rng, 1, 4096), _log_uniform(rng, 100, 262144)
        if R * V <= largest:
            break
    mask = rng.choice(["none", "none", "rows", "shared"])
    if kind == "logprobs_backward":
        return dict(kind=kind, R=R, V=V, dtype=dtype, top=0, mask=mask, scale=rng.choice([1.0, 1.0, 0.7, 1.25]))
    return dict(kind=kind, R=R, V=V, dtype=dtype, top=min(V, rng.choice([0, 1, 5, 10, 20, 50])), mask=mask, scale=rng.choice([1.0, 1.0, 0.7, 1.25]))


def _groups(case):
    return -(-case["K"] // case["group"])


def _weights(case, gen):
    """He-normal weights, one group after the other scaled to the range of a code: codes in [-8, 7] and scales."""
    N, K, G, g = case["N"], case["K"], _groups(case), case["group"]
    codes = torch.empty((N, K), dtype=torch.int8, device=DEV)
    scales = torch.empty((N, G), dtype=DTYPES[case["dtype"]], device=DEV)
    step = max(1, (1 << 26) // (G * g))
    for lo in range(0, N, step):
        rows = min(step, N - lo)
        w = torch.randn((rows, G, g), device=DEV, generator=gen) * math.sqrt(2.0 / K)
        s = (w.abs().amax(2) / 7.0).to(scales.dtype)
        c = torch.clamp(torch.round(w / s.float().unsqueeze(2)), -8, 7)
        codes[lo:lo + rows] = c.to(torch.int8).reshape(rows, G * g)[:, :K]
        scales[lo:lo + rows] = s
    return codes, scales


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, device=DEV, generator=gen)

    if case["kind"] == "linear":
        s = dict(x=normal(case["M"], case["K"]).abs().to(dtype))
        s["codes"], s["scales"] = _weights(case, gen)
        s["bias"] = (0.1 * normal(case["N"])).to(dtype) if case["bias"] else None
        return s
    if case["kind"] == "linear_backward":
        s = dict(dy=normal(case["M"], case["N"]).to(dtype))
        s["codes"], s["scales"] = _weights(case, gen)
        s["y"] = torch.relu(normal(case["M"], case["N"])).to(dtype) if case["relu"] else None
        return s
    # Logits: mostly noise, a few entries of each row well above it, as a trained network's are
    R, V = case["R"], case["V"]
    logits = torch.empty((R, V), dtype=dtype, device=DEV)
    step = max(1, (1 << 27) // V)
    for lo in range(0, R, step):
        logits[lo:lo + step] = (2.0 * normal(min(step, R - lo), V)).to(dtype)
    peaks = torch.randint(0, V, (R, 8), device=DEV, generator=gen)
    logits.scatter_(1, peaks, (8.0 + 4.0 * normal(R, 8)).to(dtype))
    targets = torch.where(torch.rand((R,), device=DEV, generator=gen) < 0.7, peaks[:, 0], torch.randint(0, V, (R,), device=DEV, generator=gen))
    mask = None
    if case["mask"] != "none":
        mask = torch.rand((R if case["mask"] == "rows" else 1, V), device=DEV, generator=gen) < 0.8
    s = dict(logits=logits, targets=targets, mask=mask, scale=case["scale"], top=case["top"])
    if case["kind"] == "logprobs_backward":
        s["g_logprob"], s["g_entropy"] = normal(R) / R, 0.01 * normal(R) / R
        stats, entropy = [], []
        for lo in range(0, R, step):
            part = dict(s, logits=logits[lo:lo + step], mask=mask if mask is None or mask.shape[0] == 1 else mask[lo:lo + step])
            z, best, e, total = _softmax(part, torch.float64)
            stats.append(torch.stack([best, torch.log(total)], 1).float())
            entropy.append(_entropy(z, e, total).float())
        s["stats"], s["entropy"] = torch.cat(stats), torch.cat(entropy)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["kind"], s["case"] = case["kind"], case
    if own:
        from paper_2512_18453_amd import nova
        dtype = DTYPES[case["dtype"]]
        if case["kind"].startswith("linear"):
            back = case["kind"] == "linear_backward"
            direction = nova.NOVA_Q4_BACKWARD if back else nova.NOVA_Q4_FORWARD
            s["Wq"] = nova.nova_q4_pack(s["codes"], s["scales"], case["group"], direction)
            s["out"] = torch.empty((case["M"], case["K"] if back else case["N"]), dtype=dtype, device=DEV)
            s["workspace"] = torch.empty(nova.nova_q4_linear_workspace_bytes(case["M"], case["N"], case["K"], case["group"], dtype, direction),
                                         dtype=torch.uint8, device=DEV)
        elif case["kind"] == "logprobs":
            s["workspace"] = torch.empty(nova.nova_logprobs_workspace_bytes(case["R"], case["V"], case["top"], dtype), dtype=torch.uint8, device=DEV)
        else:
            s["out"] = torch.empty_like(s["logits"])
    return s


# ---- the plain forms ----

def _dequantised(s, K, group, dtype=torch.float32):
    scales = s["scales"].to(dtype).repeat_interleave(group, 1)[:, :K]
    return s["codes"].to(dtype) * scales


def _softmax(s, dtype=torch.float32):
    """Differences to the row's largest allowed logit, scaled; that logit; their exponentials and the sum."""
    x = s["logits"].to(dtype)
    if s["mask"] is not None:
        x = torch.where(s["mask"], x, -math.inf)
    best = x.amax(1)
    z = (x - best.unsqueeze(1)) * s["scale"]
    e = torch.exp(z)
    return z, best, e, e.sum(1)


def _entropy(z, e, total):
    return torch.log(total) - torch.where(e > 0, e * z, 0.0).sum(1) / total


def _plain_linear(s):
    case = s["case"]
    y = s["x"].float() @ _dequantised(s, case["K"], case["group"]).T
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["relu"]:
        y = torch.where(y < 0, 0.0, y)
    return y.to(s["x"].dtype)


def _plain_linear_backward(s):
    case = s["case"]
    dy = s["dy"].float()
    if s["y"] is not None:
        dy = torch.where(s["y"] > 0, dy, 0.0)
    return (dy @ _dequantised(s, case["K"], case["group"])).to(s["dy"].dtype)


def _plain_logprobs(s):
    z, best, e, total = _softmax(s)
    log_sum = torch.log(total)
    logprob = z.gather(1, s["targets"].unsqueeze(1)).squeeze(1) - log_sum
    outputs = dict(logprob=logprob, entropy=_entropy(z, e, total), stats=torch.stack([best, log_sum], 1))
    if s["top"]:
        left, values, ids = z.clone(), [], []
        for _ in range(s["top"]):
            first = left.argmax(1, keepdim=True)
            value = left.gather(1, first)
            values.append(value - log_sum.unsqueeze(1))
            ids.append(torch.where(value == -math.inf, -1, first))
            left.scatter_(1, first, -math.inf)
        outputs["top_logprobs"], outputs["top_ids"] = torch.cat(values, 1), torch.cat(ids, 1)
    return outputs


def _plain_logprobs_backward(s):
    x = s["logits"].float()
    if s["mask"] is not None:
        x = torch.where(s["mask"], x, -math.inf)
    lp = (x - s["stats"][:, :1]) * s["scale"] - s["stats"][:, 1:]
    p = torch.exp(lp)
    grad = -s["g_logprob"].unsqueeze(1) * p - s["g_entropy"].unsqueeze(1) * torch.where(p > 0, p * (lp + s["entropy"].unsqueeze(1)), 0.0)
    chosen = s["targets"].unsqueeze(1)
    allowed = (x.gather(1, chosen) > -math.inf).float()
    grad.scatter_add_(1, chosen, s["g_logprob"].unsqueeze(1) * allowed)
    return (s["scale"] * grad).to(s["logits"].dtype)


def run(s):
    if not own:
        return {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "logprobs": _plain_logprobs,
                "logprobs_backward": _plain_logprobs_backward}[s["kind"]](s)
    from paper_2512_18453_amd import nova
    case = s["case"]
    if s["kind"] == "linear":
        return nova.nova_q4_linear(s["x"], s["Wq"], case["N"], case["group"], bias=s["bias"], y=s["out"],
                                   flags=nova.NOVA_FLAG_RELU if case["relu"] else 0, workspace=s["workspace"])
    if s["kind"] == "linear_backward":
        return nova.nova_q4_linear_backward(s["dy"], s["Wq"], case["K"], case["group"], y=s["y"], dx=s["out"], workspace=s["workspace"])
    if s["kind"] == "logprobs":
        got = nova.nova_logprobs(s["logits"], s["targets"], mask=s["mask"], scale=s["scale"], top=s["top"], workspace=s["workspace"])
        outputs = dict(logprob=got.logprob, entropy=got.entropy, stats=got.stats)
        if s["top"]:
            outputs["top_logprobs"], outputs["top_ids"] = got.top_logprobs, got.top_ids
        return outputs
    return nova.nova_logprobs_backward(s["logits"], s["stats"], s["targets"], g_logprob=s["g_logprob"], entropy=s["entropy"],
                                       g_entropy=s["g_entropy"], mask=s["mask"], scale=s["scale"], dlogits=s["out"])


def work(case):
    es = SIZES[case["dtype"]]
    if case["kind"].startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        weights = N * K / 2 + N * _groups(case) * es
        extra = N * es * case["bias"] if case["kind"] == "linear" else M * N * es * case["relu"]
        return {"bytes": weights + (M * K + M * N) * es + extra, "flops": 2.0 * M * N * K}
    R, V = case["R"], case["V"]
    masks = {"none": 0, "rows": R * V, "shared": V}[case["mask"]]
    if case["kind"] == "logprobs":
        return {"bytes": R * V * es + masks + R * (8 + 4 + 4 + 8 + 12 * case["top"]), "flops": 6.0 * R * V}
    return {"bytes": 2 * R * V * es + masks + R * (8 + 8 + 4 + 4 + 4), "flops": 10.0 * R * V}


# ---- the definition in 64 bits ----

def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"].startswith("linear"):
        # (one block of the reduction at a time, so that the weights in 64 bits need not all be there together)
        M, N, K, g = case["M"], case["N"], case["K"], case["group"]
        back = case["kind"] == "linear_backward"
        left = s["dy"].double() if back else s["x"].double()
        if back and s["y"] is not None:
            left = left * (s["y"].double() > 0)
        out = torch.zeros((M, K if back else N), dtype=torch.float64, device=DEV)
        for j in range(0, K, 16 * g):
            hi = min(K, j + 16 * g)
            block = s["codes"][:, j:hi].double()
            for k in range(j, hi, g):
                block[:, k - j:k - j + g] *= s["scales"][:, k // g].double().unsqueeze(1)
            if back:
                out[:, j:hi] = left @ block
            else:
                out += left[:, j:hi] @ block.T
        if not back:
            if s["bias"] is not None:
                out += s["bias"].double()
            if case["relu"]:
                out.clamp_(min=0.0)
        return out
    R, V, top, c = case["R"], case["V"], case["top"], case["scale"]
    rows = torch.arange(R, device=DEV)
    parts = []
    step = max(1, (1 << 25) // V)
    for lo in range(0, R, step):
        block = s["logits"][lo:lo + step].double()
        keep = torch.ones_like(block, dtype=torch.bool)
        if s["mask"] is not None:
            keep = (s["mask"] if s["mask"].shape[0] == 1 else s["mask"][lo:lo + step]).expand_as(block)
        block = block.masked_fill(~keep, -math.inf)
        t = s["targets"][lo:lo + step]
        i = rows[:block.shape[0]]
        if case["kind"] == "logprobs":
            lse = torch.logsumexp(c * block, 1)
            lp = c * block - lse.unsqueeze(1)
            p = lp.exp()
            best = block.max(1).values
            got = [lp[i, t], -torch.nan_to_num(p * lp).sum(1), torch.stack([best, lse - c * best], 1)]
            if top:
                # (a stable sort leaves equal logits in the order of their index)
                order = torch.sort(block, dim=1, descending=True, stable=True).indices[:, :top]
                chosen = lp.gather(1, order)
                got += [chosen, torch.where(chosen == -math.inf, -1, order)]
            parts.append(got)
        else:
            # the gradient at the statistics that the call is given, which the forward pass rounded to 32 bits
            best, log_sum, H = s["stats"][lo:lo + step, :1].double(), s["stats"][lo:lo + step, 1:].double(), s["entropy"][lo:lo + step, None].double()
            a, h = s["g_logprob"][lo:lo + step, None].double(), s["g_entropy"][lo:lo + step, None].double()
            lp = c * (block - best) - log_sum
            p = lp.exp()
            hit = torch.zeros_like(block)
            hit[i, t] = 1.0
            parts.append([c * (a * (hit * keep - p) - h * torch.nan_to_num(p * (lp + H)))])
    whole = [torch.cat(column) for column in zip(*parts)]
    if case["kind"] == "logprobs_backward":
        return whole[0]
    return dict(zip(["logprob", "entropy", "stats", "top_logprobs", "top_ids"], whole))
