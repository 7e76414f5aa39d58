"""Tensors in host memory are refused by the binding of 8-bit float layers and of dropout before the library sees an address, each with its name; also where there is no device to
ask for the current one.  CPU only."""
import pytest
import torch

from paper_2512_18453_amd import nova

F16 = torch.float16


@pytest.fixture(autouse=True)
def no_device_and_no_call(monkeypatch):
    """The question for the current device, which fails first without one, is answered; the stream is not asked for; no call that takes memory returns."""
    monkeypatch.setattr(nova, "_here", lambda *tensors: None)
    monkeypatch.setattr(nova, "_stream", lambda: None)

    def never(code, what):
        raise AssertionError(f"{what} was called")
    monkeypatch.setattr(nova, "_check", never)


def layout(rows, columns, block):
    return torch.zeros(nova.nova_f8_bytes(rows, columns, block), dtype=torch.uint8)


x, dy, half = torch.zeros(4, 8), torch.zeros(4, 6), torch.zeros(4, 8, dtype=F16)


@pytest.mark.parametrize("what,call", [
    ("x", lambda: nova.nova_f8_quantize(x, 1)),
    ("codes", lambda: nova.nova_f8_pack(x.to(torch.float8_e4m3fn), torch.zeros(4, 1), 1)),
    ("Xq", lambda: nova.nova_f8_unpack(layout(4, 8, 1), 4, 8, 1)),
    ("Aq", lambda: nova.nova_f8_matmul(layout(4, 8, 1), layout(6, 8, 128), 4, 6, 8)),
    ("x", lambda: nova.nova_f8_linear(x, layout(6, 8, 128), 6)),
    ("dy", lambda: nova.nova_f8_linear_backward(dy, layout(8, 6, 128), x)),
    ("x", lambda: nova.nova_dropout(half, 0.5, 1)),
    ("dy", lambda: nova.nova_dropout_backward(half, 0.5, 1)),
])
def test_host_tensors_are_refused(what, call):
    with pytest.raises(ValueError, match=f"^{what}: expected a (contiguous )?device tensor"):
        call()


@pytest.mark.parametrize("check", [lambda t: nova._rows(t, (4, 8), torch.float32, "it"), lambda t: nova._flat(t, 32, torch.float32, "it")])
def test_each_check_by_itself(check):
    with pytest.raises(ValueError, match="^it: expected"):
        check(x)


def test_bytes_by_itself():
    with pytest.raises(ValueError, match="^it: expected"):
        nova._bytes(torch.zeros(16, dtype=torch.uint8), "it")
