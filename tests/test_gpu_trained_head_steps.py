"""What a training step of the example's fully connected layers does and how it is timed."""
import json

import pytest
import torch

import vgg16_classify
from tests.launches import launches

pytestmark = pytest.mark.gpu


def test_only_layouts_that_are_read_are_made():
    """The first layer's input takes no gradient, so nothing reads a layout of its weights' transpose."""
    head = vgg16_classify.TrainedHead(torch.Generator("cuda:0").manual_seed(2), 4, 512)
    for L, count in zip(head.layers, (1, 2, 2), strict=True):
        assert len(launches(lambda: head.lay_out(L))) == count
    assert [L["backward"] is None for L in head.layers] == [True, False, False]
    x = torch.randn((4, 512), device="cuda:0").half()
    g = torch.full((4,), -0.25, device="cuda:0")
    before = [L["weight"].clone() for L in head.layers]
    head.train(x, torch.arange(4, device="cuda:0"), g)
    assert all(bool((L["weight"] != w).any()) and bool(L["weight"].isfinite().all()) for L, w in zip(head.layers, before))


@pytest.mark.parametrize("steps", [1, 3])
def test_time_of_a_step(steps, capsys):
    """All steps but the first are timed: of one step alone there is no time."""
    vgg16_classify.main(["--batch", "2", "--size", "32", "--m", "4", "--reps", "1", "--train", str(steps)])
    training = json.loads(capsys.readouterr().out.splitlines()[-1])["training"]
    assert training["steps"] == steps and len(training["losses"]) == steps
    assert training["ms_per_step"] is None if steps == 1 else training["ms_per_step"] > 0
