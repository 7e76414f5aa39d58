"""The example from pixels to answers, on small images: its layers, log probabilities and gradient against the same formulas in 64 bits on its own features, and the
graph of its forward pass against the calls."""
import pytest
import torch

import vgg16_classify
from paper_2512_18453_amd import nova

pytestmark = pytest.mark.gpu
F16 = torch.float16


@pytest.mark.parametrize("batch,group", [(1, 64), (6, 128), (40, 32)])
def test_answers_and_gradient(batch, group, capsys):
    run = vgg16_classify.main(["--batch", str(batch), "--size", "32", "--m", "4", "--group", str(group), "--reps", "1"])
    assert '"finite": true' in capsys.readouterr().out
    x, weights, outputs = run["features"].double(), [], []
    for L in run["head"].layers:
        codes, scales = nova.nova_q4_unpack(L["forward"], L["N"], L["K"], group, F16)
        back = nova.nova_q4_unpack(L["backward"], L["N"], L["K"], group, F16, nova.NOVA_Q4_BACKWARD)
        assert torch.equal(back[0], codes) and torch.equal(back[1], scales)
        W = codes.double() * scales.double().repeat_interleave(group, 1)[:, :L["K"]]
        x = x @ W.T + L["bias"].double()
        if L["flags"]:
            x = x.clamp(min=0.0)
        # every layer's result is rounded to binary16 once (2^-11 of it); a layer passes its input's error on with the norm of its weights, about that of its outputs
        assert (L["y"].double() - x).norm() <= 3 * 2.0 ** -11 * x.norm()
        x = L["y"].double()
        weights.append(W)
        outputs.append(x)
    a = run["answers"]
    lp = torch.log_softmax(run["logits"].double(), 1)
    labels = run["labels"]
    torch.testing.assert_close(a.logprob.double(), lp.gather(1, labels.unsqueeze(1)).squeeze(1), rtol=1e-5, atol=1e-5)
    torch.testing.assert_close(a.entropy.double(), -(lp.exp() * lp).sum(1), rtol=1e-5, atol=1e-5)
    order = torch.sort(run["logits"].double(), dim=1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(a.top_ids, order)
    d = run["g"].double().unsqueeze(1) * (torch.nn.functional.one_hot(labels, 1000).double() - lp.exp())
    for W, y, L in reversed(list(zip(weights, outputs, run["head"].layers))):
        d = (d * (y > 0) if L["flags"] else d) @ W
    # four roundings to binary16, some of them among its subnormal numbers (the smallest step 2^-24)
    assert (run["gradient"].double() - d).norm() <= 8 * 2.0 ** -11 * d.norm() + 2.0 ** -24 * d.numel() ** 0.5 * 100
    for p, q in zip(run["replayed"], a):
        assert torch.equal(p, q)
