"""The fully connected layers of the example as they train: every call of a step against its formula in 64 bits on the tensors that the step left, and a captured step against
the calls.  On small images."""
import pytest
import torch

import vgg16_classify
from paper_2512_18453_amd import nova
from tests import plain_training as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, F32 = torch.float16, torch.float32
HALF_STEP = 2.0 ** -11


def operand(v, format, block):
    codes, scales = plain.quantized(v, format, block)
    return plain.values(codes, scales, block), plain.lowest_values(scales, *codes.shape, format, block)


def near(got, want, bound, half_step):
    err = (got.double().cpu() - want).abs()
    over = (err - bound - half_step * (want.abs() + bound) - 2.0 ** -24).max().item()
    assert over <= 0, over


def narrow(a, b):
    want, bound = plain.product(a[0], b[0])
    return want, bound + plain.cut_off(a[0], b[0], (a[1], b[1]))


@pytest.mark.parametrize("batch", [1, 6, 40])
def test_gradients_of_a_step(batch, capsys):
    run = vgg16_classify.main(["--batch", str(batch), "--size", "32", "--m", "4", "--reps", "1", "--train", "2"])
    assert '"training": {"steps": 2' in capsys.readouterr().out
    head, labels, g = run["trained"], run["labels"], run["g"]
    step = int(head.step)
    assert step == 2
    logits = head.logits(run["features"])
    answers = nova.nova_logprobs(logits, labels)
    head.gradient(logits, labels, answers, g)
    torch.cuda.synchronize()
    x = run["features"]
    for i, L in enumerate(head.layers):
        assert torch.equal(L["x"], x)
        want, bound = narrow(operand(x, 0, 1), operand(L["weight"], 0, 128))
        want = want + L["bias"].double().cpu()
        bound = bound + 2.0 ** -24 * (want.abs() + bound)
        near(L["y"], want.clamp(min=0.0) if L["hidden"] else want, bound, HALF_STEP)
        x = L["y"]
        if L["hidden"]:
            keep = plain.kept(batch, L["N"], head.p, head.seed + i, step)
            assert torch.equal(L["kept"].cpu(), torch.where(keep, x.cpu() * 2, 0.0))             # p = 1/2: doubled, which rounds nothing
            x = L["kept"]
    lp = torch.log_softmax(logits.double(), 1)
    dlogits = g.double().unsqueeze(1) * (torch.nn.functional.one_hot(labels, 1000).double() - lp.exp())
    # p = exp((x - M) - L) in binary32: the exponent is off by its terms' roundings, (|x - M| + |L| + 4) 2^-23 with those of exp, and p by as much of itself; where p is
    # nearly 1 that is all that is left of 1 - p
    terms = (logits.double() - answers.stats[:, :1].double()).abs() + answers.stats[:, 1:].double().abs() + 4
    near(head.dlogits, dlogits.cpu(), (g.double().abs().unsqueeze(1) * lp.exp() * terms * 2.0 ** -23).cpu(), HALF_STEP)
    d = head.dlogits
    for i, L in reversed(list(enumerate(head.layers))):
        if L["hidden"]:
            keep = plain.kept(batch, L["N"], head.p, head.seed + i, step)
            assert torch.equal(L["dy"].cpu(), torch.where(keep, d.cpu() * 2, 0.0))
            d = L["dy"]
        gated = torch.where(L["y"] > 0, d, 0.0) if L["hidden"] else d
        dw, bound = plain.product(operand(gated.T, 1, 1)[0], operand(L["x"].T, 0, 1)[0])
        near(L["dw"], dw, bound, 2.0 ** -24)
        near(L["dbias"], gated.double().sum(0).cpu(), 128 * 2.0 ** -24 * gated.double().abs().sum(0).cpu(), 2.0 ** -24)
        if i:
            near(L["dx"], *narrow(operand(gated, 1, 1), tuple(t.T for t in operand(L["weight"], 0, 128))), HALF_STEP)
            d = L["dx"]


def test_captured_step():
    """Steps replayed from one graph leave the weights that the calls leave: masks follow the step number on the device."""
    batch, features = 8, 512
    x = torch.randn((batch, features), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).half()
    labels = torch.arange(batch, device=DEV)
    g = torch.full((batch,), -1.0 / batch, device=DEV)
    called, captured = (vgg16_classify.TrainedHead(torch.Generator(DEV).manual_seed(2), batch, features, rate=0.01) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        answers = captured.train(x, labels, g)
    for step in range(3):
        want = called.train(x, labels, g)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(answers.logprob, want.logprob), step
        for p, q in zip(called.layers, captured.layers):
            assert torch.equal(p["weight"], q["weight"]) and torch.equal(p["bias"], q["bias"]) and torch.equal(p["forward"], q["forward"])
    assert int(captured.step) == 3
