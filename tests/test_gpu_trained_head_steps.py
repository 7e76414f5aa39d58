"""What a training step of the example's fully connected layers does and how it is timed."""
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
