"""What the calls of 4-bit layers and of log probabilities refuse, before anything is launched: the C entry points with made-up addresses, which a refused call never
reads.  CPU only."""
import ctypes

import pytest
import torch

from paper_2512_18453_amd import nova

EINVAL, ENOSPC = -1, -5
F32, F16, BF16 = nova.NOVA_F32, nova.NOVA_F16, nova.NOVA_BF16
AT, BIG = 1 << 20, 1 << 40                                 # an aligned address; more bytes than any of these calls needs


def test_sizes():
    L = nova.lib()
    assert L.nova_q4_bytes(4096, 25088, 128, F16, 0) == 4096 * 25088 // 2 + 4096 * 196 * 2
    assert L.nova_q4_bytes(17, 130, 32, F32, 0) == 2 * 2 * 1024 + 2 * 8 * 16 * 4
    assert L.nova_q4_bytes(17, 130, 32, F32, 1) == 9 * 1 * 1024 + 5 * 128 * 4
    for bad in ((0, 1, 32, F16, 0), (1, 0, 32, F16, 0), ((1 << 24) + 1, 1, 32, F16, 0), (1, (1 << 24) + 1, 32, F16, 0), (1, 1, 16, F16, 0), (1, 1, 256, F16, 0),
                (1, 1, 0, F16, 0), (1, 1, 32, 3, 0), (1, 1, 32, -1, 0), (1, 1, 32, F16, 2), (1, 1, 32, F16, -1)):
        assert L.nova_q4_bytes(*bad) == 0, bad
        assert L.nova_q4_linear_workspace_bytes(4, *bad) == 0, bad
    assert L.nova_q4_linear_workspace_bytes(-1, 4, 4, 32, F16, 0) == 0
    for bad in ((-1, 5, 0, F16), (1, 0, 0, F16), (1, 5, -1, F16), (1, 5, 65, F16), (1, 5, 0, 7)):
        assert L.nova_logprobs_workspace_bytes(*bad) == 0, bad


def test_lay_out():
    L = nova.lib()
    need = L.nova_q4_bytes(20, 40, 32, F16, 0)
    quantize = dict(w=AT, N=20, K=40, group=32, dtype=F16, direction=0, Wq=AT, Wq_bytes=need, stream=None)
    for change, code in ((dict(w=None), EINVAL), (dict(Wq=None), EINVAL), (dict(Wq=AT + 8), EINVAL), (dict(group=48), EINVAL), (dict(dtype=9), EINVAL),
                         (dict(direction=3), EINVAL), (dict(N=0), EINVAL), (dict(Wq_bytes=need - 1), ENOSPC)):
        assert L.nova_q4_quantize(*{**quantize, **change}.values()) == code, change
    pack = dict(codes=AT, scales=AT, N=20, K=40, group=32, dtype=F16, direction=0, Wq=AT, Wq_bytes=need, stream=None)
    for change, code in ((dict(codes=None), EINVAL), (dict(scales=None), EINVAL), (dict(Wq=None), EINVAL), (dict(K=0), EINVAL), (dict(Wq_bytes=need - 1), ENOSPC)):
        assert L.nova_q4_pack(*{**pack, **change}.values()) == code, change
    unpack = dict(Wq=AT, Wq_bytes=need, N=20, K=40, group=32, dtype=F16, direction=0, codes=AT, scales=None, stream=None)
    for change, code in ((dict(Wq=None), EINVAL), (dict(Wq=AT + 4), EINVAL), (dict(codes=None), EINVAL), (dict(Wq_bytes=need - 1), ENOSPC)):
        assert L.nova_q4_unpack(*{**unpack, **change}.values()) == code, change


@pytest.mark.parametrize("M", [1, 3, 40, 500])
def test_products(M):
    L = nova.lib()
    N, K = 20, 40
    need, ws = L.nova_q4_bytes(N, K, 32, BF16, 0), L.nova_q4_linear_workspace_bytes(M, N, K, 32, BF16, 0)
    linear = dict(x=AT, ldx=K, Wq=AT, Wq_bytes=need, bias=None, y=AT, ldy=N, M=M, N=N, K=K, group=32, dtype=BF16, flags=0, workspace=AT, workspace_bytes=BIG,
                  stream=None)
    changes = [(dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(Wq=None), EINVAL), (dict(Wq=AT + 1), EINVAL), (dict(M=-1), EINVAL), (dict(flags=2), EINVAL),
               (dict(flags=4), EINVAL), (dict(group=100), EINVAL), (dict(dtype=3), EINVAL), (dict(Wq_bytes=need - 1), ENOSPC)]
    if M > 1:
        changes += [(dict(ldx=K - 1), EINVAL), (dict(ldx=-K), EINVAL), (dict(ldy=N - 1), EINVAL), (dict(ldy=0), EINVAL)]
    if ws:
        changes += [(dict(workspace=None), EINVAL), (dict(workspace=AT + 4), EINVAL), (dict(workspace_bytes=ws - 1), ENOSPC)]
    for change, code in changes:
        assert L.nova_q4_linear(*{**linear, **change}.values()) == code, change
    assert L.nova_q4_linear(*{**linear, "M": 0, "x": None, "y": None}.values()) == 0            # nothing to do
    need, ws = L.nova_q4_bytes(N, K, 32, BF16, 1), L.nova_q4_linear_workspace_bytes(M, N, K, 32, BF16, 1)
    back = dict(dy=AT, lddy=N, y=None, ldy=0, Wq=AT, Wq_bytes=need, dx=AT, lddx=K, M=M, N=N, K=K, group=32, dtype=BF16, workspace=AT, workspace_bytes=BIG, stream=None)
    changes = [(dict(dy=None), EINVAL), (dict(dx=None), EINVAL), (dict(Wq=None), EINVAL), (dict(N=0), EINVAL), (dict(Wq_bytes=need - 1), ENOSPC)]
    if M > 1:
        changes += [(dict(lddy=N - 1), EINVAL), (dict(y=AT, ldy=N - 1), EINVAL), (dict(lddx=0), EINVAL)]
    if ws:
        changes += [(dict(workspace=None), EINVAL), (dict(workspace_bytes=ws - 1), ENOSPC)]
    for change, code in changes:
        assert L.nova_q4_linear_backward(*{**back, **change}.values()) == code, change
    assert L.nova_q4_linear_backward(*{**back, "M": 0, "dy": None}.values()) == 0


@pytest.mark.parametrize("rows,V", [(1, 200000), (4, 100), (3000, 5000)])
def test_logprobs(rows, V):
    L = nova.lib()
    ws = L.nova_logprobs_workspace_bytes(rows, V, 5, F16)
    call = dict(logits=AT, stride=V, targets=AT, mask=None, mask_stride=0, rows=rows, V=V, scale=1.0, top=5, dtype=F16, logprob=AT, entropy=AT, stats=AT,
                top_logprobs=AT, top_ids=AT, workspace=AT, workspace_bytes=BIG, stream=None)
    changes = [(dict(logits=None), EINVAL), (dict(stats=None), EINVAL), (dict(targets=None), EINVAL), (dict(top_ids=None), EINVAL), (dict(top_logprobs=None), EINVAL),
               (dict(top=65), EINVAL), (dict(top=-1), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL), (dict(scale=float("nan")), EINVAL),
               (dict(scale=float("inf")), EINVAL), (dict(V=0), EINVAL), (dict(rows=-1), EINVAL), (dict(dtype=3), EINVAL)]
    if rows > 1:
        changes += [(dict(stride=V - 1), EINVAL), (dict(mask=AT, mask_stride=V - 1), EINVAL)]
    if ws:
        changes += [(dict(workspace=None), EINVAL), (dict(workspace=AT + 8), EINVAL), (dict(workspace_bytes=ws - 1), ENOSPC)]
    for change, code in changes:
        assert L.nova_logprobs(*{**call, **change}.values()) == code, change
    assert L.nova_logprobs(*{**call, "rows": 0, "logits": None}.values()) == 0
    back = dict(logits=AT, stride=V, stats=AT, targets=AT, g_logprob=AT, entropy=AT, g_entropy=AT, mask=None, mask_stride=0, rows=rows, V=V, scale=1.0, dtype=F16,
                dlogits=AT, dstride=V, stream=None)
    changes = [(dict(logits=None), EINVAL), (dict(stats=None), EINVAL), (dict(targets=None), EINVAL), (dict(entropy=None), EINVAL), (dict(dlogits=None), EINVAL),
               (dict(scale=0.0), EINVAL), (dict(V=0), EINVAL), (dict(dtype=-2), EINVAL)]
    if rows > 1:
        changes += [(dict(stride=V - 1), EINVAL), (dict(dstride=V - 1), EINVAL), (dict(dstride=0), EINVAL), (dict(mask=AT, mask_stride=1), EINVAL)]
    for change, code in changes:
        assert L.nova_logprobs_backward(*{**back, **change}.values()) == code, change
    assert L.nova_logprobs_backward(*{**back, "rows": 0, "logits": None}.values()) == 0


def test_convolutions_do_not_take_bfloat16():
    L = nova.lib()
    assert L.nova_filter_bytes(8, 8, 4, 3, BF16) == 0
    assert L.nova_relu_maxpool2x2(ctypes.c_void_p(AT), ctypes.c_void_p(AT), 1, 1, 2, 2, BF16, None) == EINVAL


def test_binding():
    x = torch.zeros((2, 40))
    with pytest.raises(ValueError):
        nova.nova_q4_linear(x, torch.zeros(10, dtype=torch.uint8), 20, 32)                      # not on the device
    with pytest.raises(TypeError):
        nova.nova_q4_linear(x.double(), torch.zeros(10, dtype=torch.uint8), 20, 32)
    with pytest.raises(TypeError):
        nova.nova_logprobs(x.long())


@pytest.mark.parametrize("direction", [0, 1])
def test_no_rows_need_no_workspace(direction):
    # (the host divides by the number of tiles, of which there are none)
    for N, K in ((1, 1), (20, 40), (4096, 25088)):
        assert nova.lib().nova_q4_linear_workspace_bytes(0, N, K, 32, F16, direction) == 0
    assert nova.lib().nova_logprobs_workspace_bytes(0, 200000, 5, F16) == 0


def test_binding_wants_matrices():
    with pytest.raises(ValueError):
        nova._rows(torch.zeros(40), (1, 40), torch.float32, "x")
    with pytest.raises(ValueError):
        nova._rows(torch.zeros((40, 2)).T, (2, 40), torch.float32, "x")


def test_largest_scale():
    # (its product with log2 e has to be a number)
    call = [AT, 10, None, None, 0, 2, 10, 1.1e38, 0, F16, None, None, AT, None, None, None, 0, None]
    assert nova.lib().nova_logprobs(*call) == EINVAL
    back = [AT, 10, AT, None, None, None, None, None, 0, 2, 10, 1.1e38, F16, AT, 10, None]
    assert nova.lib().nova_logprobs_backward(*back) == EINVAL
