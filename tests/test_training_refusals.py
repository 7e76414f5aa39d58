"""What the calls of 8-bit float layers and of dropout refuse, before anything is launched: the C entry points with made-up addresses, which a refused call never
reads; sizes; the plain generator against published answers.  CPU only."""
import pytest
import torch

from paper_2512_18453_amd import nova
from tests import plain_training as plain

EINVAL, ENOSPC = -1, -5
F32, F16, BF16 = nova.NOVA_F32, nova.NOVA_F16, nova.NOVA_BF16
AT, BIG = 1 << 20, 1 << 60
NAN = float("nan")


def test_sizes():
    L = nova.lib()
    assert L.nova_f8_bytes(4096, 25088, 128) == 4096 * 25088 + 196 * 32 * 4
    assert L.nova_f8_bytes(4096, 25088, 1) == 4096 * 25088 + 196 * 4096 * 4
    assert L.nova_f8_bytes(17, 129, 1) == 2 * 2 * 2048 + 2 * 32 * 4
    assert L.nova_f8_bytes(17, 129, 128) == 2 * 2 * 2048 + 2 * 4
    most = 2 ** 31 - 128                                                            # (no overflow on the way)
    assert L.nova_f8_bytes(most, most, 1) == most * most + most // 128 * most * 4 and L.nova_f8_bytes(most, 1, 128) == most * 128 + most // 128 * 4
    for bad in ((most + 1, 1, 1), (1, most + 1, 1), (2 ** 31 - 1, 1, 128), (0, 1, 1), (1, 0, 1), (-1, 1, 1), (1, 1, 0), (1, 1, 64), (1, 1, 129)):
        assert L.nova_f8_bytes(*bad) == 0, bad
    for bad in ((-1, 4, 4, F16), (4, 0, 4, F16), (4, 4, 0, F16), (4, (1 << 24) + 1, 4, F16), (4, 4, (1 << 24) + 1, F16), (4, 4, 4, 3), (0, 4, 4, F16), (most + 1, 4, 4, F16)):
        assert L.nova_f8_linear_workspace_bytes(*bad) == 0, bad
        assert L.nova_f8_linear_backward_workspace_bytes(*bad) == 0, bad
        assert L.nova_f8_matmul_workspace_bytes(*bad[:3], 1, 128, bad[3]) == 0, bad
    assert L.nova_f8_matmul_workspace_bytes(4, 4, 4, 2, 128, F16) == 0 and L.nova_f8_matmul_workspace_bytes(4, 4, 4, 1, 16, F16) == 0


def refused(call, given, changes):
    for change, code in changes:
        assert set(change) <= set(given), change
        assert call(*{**given, **change}.values()) == code, change


def test_layouts():
    L = nova.lib()
    need = L.nova_f8_bytes(20, 300, 1)
    refused(L.nova_f8_quantize, dict(x=AT, ldx=300, rows=20, columns=300, dtype=F16, format=0, block=1, transposed=0, Xq=AT, Xq_bytes=need, stream=None),
            [(dict(x=None), EINVAL), (dict(Xq=None), EINVAL), (dict(Xq=AT + 8), EINVAL), (dict(rows=0), EINVAL), (dict(rows=2 ** 31 - 1, Xq_bytes=BIG), EINVAL), (dict(columns=-3), EINVAL), (dict(ldx=299), EINVAL),
             (dict(ldx=-300), EINVAL), (dict(dtype=3), EINVAL), (dict(format=2), EINVAL), (dict(format=-1), EINVAL), (dict(block=2), EINVAL), (dict(transposed=2), EINVAL),
             (dict(Xq_bytes=need - 1), ENOSPC), (dict(transposed=1, Xq_bytes=L.nova_f8_bytes(300, 20, 1) - 1), ENOSPC)])
    need = L.nova_f8_bytes(20, 300, 128)
    refused(L.nova_f8_pack, dict(codes=AT, scales=AT, rows=20, columns=300, block=128, transposed=0, Xq=AT, Xq_bytes=need, stream=None),
            [(dict(codes=None), EINVAL), (dict(scales=None), EINVAL), (dict(Xq=None), EINVAL), (dict(Xq=AT + 4), EINVAL), (dict(rows=0), EINVAL), (dict(columns=0), EINVAL),
             (dict(block=32), EINVAL), (dict(block=1, transposed=1, Xq_bytes=BIG), EINVAL), (dict(transposed=-1), EINVAL), (dict(Xq_bytes=need - 1), ENOSPC)])
    refused(L.nova_f8_unpack, dict(Xq=AT, Xq_bytes=need, rows=20, columns=300, block=128, codes=AT, scales=None, stream=None),
            [(dict(Xq=None), EINVAL), (dict(Xq=AT + 1), EINVAL), (dict(codes=None), EINVAL), (dict(rows=0), EINVAL), (dict(block=3), EINVAL), (dict(Xq_bytes=need - 1), ENOSPC)])


@pytest.mark.parametrize("M", [1, 3, 40, 500])
def test_products(M):
    L = nova.lib()
    N, K = 200, 5000
    a, b, ws = L.nova_f8_bytes(M, K, 1), L.nova_f8_bytes(N, K, 128), L.nova_f8_matmul_workspace_bytes(M, N, K, 1, 128, BF16)
    call = dict(Aq=AT, Aq_bytes=a, block_a=1, format_a=0, Bq=AT, Bq_bytes=b, block_b=128, format_b=0, bias=None, out=AT, ldout=N, M=M, N=N, K=K, dtype=BF16, flags=0,
                workspace=AT, workspace_bytes=BIG, stream=None)
    changes = [(dict(Aq=None), EINVAL), (dict(Aq=AT + 8), EINVAL), (dict(Bq=None), EINVAL), (dict(Bq=AT + 8), EINVAL), (dict(out=None), EINVAL), (dict(block_a=4), EINVAL),
               (dict(block_b=0), EINVAL), (dict(format_a=2), EINVAL), (dict(format_b=-1), EINVAL), (dict(M=-1), EINVAL), (dict(N=0), EINVAL), (dict(K=0), EINVAL),
               (dict(dtype=3), EINVAL), (dict(flags=2), EINVAL), (dict(flags=4), EINVAL), (dict(flags=1 | 8), EINVAL), (dict(Aq_bytes=a - 1), ENOSPC),
               (dict(Bq_bytes=b - 1), ENOSPC)]
    if M > 1:
        changes += [(dict(ldout=N - 1), EINVAL), (dict(ldout=0), EINVAL), (dict(ldout=-N), EINVAL)]
    if ws:
        changes += [(dict(workspace=None), EINVAL), (dict(workspace=AT + 4), EINVAL), (dict(workspace_bytes=ws - 1), ENOSPC)]
    refused(L.nova_f8_matmul, call, changes)
    assert L.nova_f8_matmul(*{**call, "M": 0, "Aq": None, "out": None}.values()) == 0           # nothing to do

    ws = L.nova_f8_linear_workspace_bytes(M, N, K, BF16)
    call = dict(x=AT, ldx=K, Wq=AT, Wq_bytes=b, bias=None, y=AT, ldy=N, M=M, N=N, K=K, dtype=BF16, flags=0, workspace=AT, workspace_bytes=ws, stream=None)
    changes = [(dict(x=None), EINVAL), (dict(Wq=None), EINVAL), (dict(Wq=AT + 2), EINVAL), (dict(y=None), EINVAL), (dict(M=-1), EINVAL), (dict(N=0), EINVAL),
               (dict(K=(1 << 24) + 1), EINVAL), (dict(dtype=-1), EINVAL), (dict(flags=8), EINVAL), (dict(flags=4), EINVAL), (dict(workspace=None), EINVAL),
               (dict(workspace=AT + 8), EINVAL), (dict(workspace_bytes=ws - 1), ENOSPC), (dict(Wq_bytes=b - 1), ENOSPC)]
    if M > 1:
        changes += [(dict(ldx=K - 1), EINVAL), (dict(ldx=-K), EINVAL), (dict(ldy=N - 1), EINVAL), (dict(ldy=0), EINVAL)]
    refused(L.nova_f8_linear, call, changes)
    assert L.nova_f8_linear(*{**call, "M": 0, "x": None, "y": None, "workspace": None, "workspace_bytes": 0}.values()) == 0

    ws, w = L.nova_f8_linear_backward_workspace_bytes(M, N, K, BF16), L.nova_f8_bytes(K, N, 128)
    call = dict(dy=AT, lddy=N, y=AT, ldy=N, format=1, Wq=AT, Wq_bytes=w, dx=AT, lddx=K, x=AT, ldx=K, dw=AT, lddw=K, dw_dtype=F32, dbias=AT, M=M, N=N, K=K, dtype=BF16, flags=0,
                workspace=AT, workspace_bytes=ws, stream=None)
    changes = [(dict(dy=None), EINVAL), (dict(Wq=None), EINVAL), (dict(Wq=AT + 1), EINVAL), (dict(x=None), EINVAL), (dict(dx=None, dw=None, dbias=None), EINVAL),
               (dict(format=2), EINVAL), (dict(dw_dtype=F16), EINVAL), (dict(dw_dtype=7), EINVAL), (dict(lddw=K - 1), EINVAL), (dict(lddw=0), EINVAL), (dict(N=0), EINVAL), (dict(M=-1), EINVAL), (dict(dtype=3), EINVAL),
               (dict(flags=1), EINVAL), (dict(workspace=None), EINVAL), (dict(workspace=AT + 8), EINVAL), (dict(workspace_bytes=ws - 1), ENOSPC), (dict(Wq_bytes=w - 1), ENOSPC)]
    if M > 1:
        changes += [(dict(lddy=N - 1), EINVAL), (dict(ldy=N - 1), EINVAL), (dict(lddx=K - 1), EINVAL), (dict(lddx=0), EINVAL), (dict(ldx=K - 1), EINVAL)]
    refused(L.nova_f8_linear_backward, call, changes)
    # no rows and sums that stay as they are; without dw and dbias there is nothing to clear
    assert L.nova_f8_linear_backward(*{**call, "M": 0, "flags": 8}.values()) == 0
    assert L.nova_f8_linear_backward(*{**call, "M": 0, "dw": None, "dbias": None}.values()) == 0


def test_dropout():
    L = nova.lib()
    call = dict(x=AT, ldx=40, residual=AT, ldr=40, y=AT, ldy=40, rows=5, columns=40, dtype=F16, p=0.5, seed=1, offset=2, device_offset=None, flags=0, stream=None)
    changes = [(dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(rows=-1), EINVAL), (dict(columns=-1), EINVAL), (dict(dtype=3), EINVAL), (dict(p=-0.1), EINVAL),
               (dict(p=1.0001), EINVAL), (dict(p=NAN), EINVAL), (dict(flags=4), EINVAL), (dict(flags=8), EINVAL), (dict(ldx=39), EINVAL), (dict(ldr=39), EINVAL),
               (dict(ldy=39), EINVAL), (dict(ldy=0), EINVAL), (dict(ldx=-40), EINVAL)]
    refused(L.nova_dropout, call, changes)
    for nothing in (dict(rows=0), dict(columns=0)):
        assert L.nova_dropout(*{**call, **nothing, "x": None, "y": None}.values()) == 0
    call = dict(dy=AT, lddy=40, gate=AT, ldg=40, dx=AT, lddx=40, rows=5, columns=40, dtype=F16, p=0.5, seed=1, offset=2, device_offset=None, stream=None)
    refused(L.nova_dropout_backward, call, [(dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(rows=-1), EINVAL), (dict(dtype=-1), EINVAL), (dict(p=2.0), EINVAL),
                                            (dict(p=NAN), EINVAL), (dict(lddy=39), EINVAL), (dict(ldg=39), EINVAL), (dict(lddx=39), EINVAL), (dict(lddx=0), EINVAL)])
    assert L.nova_dropout_backward(*{**call, "rows": 0, "dy": None}.values()) == 0


def test_binding():
    x = torch.zeros(4, 8)
    for call in (lambda: nova.nova_f8_quantize(x, 1), lambda: nova.nova_f8_linear(x, torch.zeros(16, dtype=torch.uint8), 4, workspace=x), lambda: nova.nova_dropout(x, 0.5, 1),
                 lambda: nova.nova_dropout_backward(x, 0.5, 1), lambda: nova.nova_f8_pack(x.to(torch.float8_e4m3fn), x, 1),
                 lambda: nova.nova_f8_linear_backward(x, None, x, workspace=x)):
        with pytest.raises((ValueError, RuntimeError)):                             # (a CPU tensor, or no device to ask)
            call()
    with pytest.raises(TypeError):
        nova.nova_f8_quantize(x.int(), 1)
    with pytest.raises(TypeError):
        nova.nova_f8_pack(x, x, 1)
    with pytest.raises(ValueError):
        nova.nova_f8_linear_backward(x, None, None)


def test_plain_generator_gives_the_published_answers():
    for counter, key, words in (((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                                ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                                ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(w) for w in plain.philox(counter, key)) == words
