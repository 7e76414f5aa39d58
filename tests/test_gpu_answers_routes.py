"""Which kernels the calls of 4-bit layers and of log probabilities launch: every variant of the kernels is reached, by the sizes its rule names, and gives
the definition's results there (tolerances as in test_gpu_q4.py and test_gpu_logprobs.py)."""
import pytest
import torch

from launches import launches
from paper_2512_18453_amd import nova
from test_gpu_logprobs import check
from test_gpu_logprobs import make as make_logits
from test_gpu_q4 import BF16, BWD, DEV, F16, F32, FWD, close, make

pytestmark = pytest.mark.gpu
CODE = {F32: 0, F16: 1, BF16: 2}


def run(M, N, K, group, dtype, direction):
    gen, codes, scales, W = make(N, K, group, dtype)
    Wq = nova.nova_q4_pack(codes, scales, group, direction)
    x = torch.randn((M, K if direction == FWD else N), device=DEV, generator=gen).to(dtype)
    y = torch.full((M, N if direction == FWD else K), float("nan"), dtype=dtype, device=DEV)
    ws = torch.full((nova.nova_q4_linear_workspace_bytes(M, N, K, group, dtype, direction),), 0xFF, dtype=torch.uint8, device=DEV)

    def call():
        if direction == FWD:
            nova.nova_q4_linear(x, Wq, N, group, y=y, workspace=ws)
        else:
            nova.nova_q4_linear_backward(x, Wq, K, group, dx=y, workspace=ws)
    call()
    operand = W.T if direction == FWD else W
    close(y, x.double() @ operand, x.double().abs() @ operand.abs(), K if direction == FWD else N, 2.0 ** -15 if direction == BWD and dtype != F32 else 0.0)
    return [name.replace("nova::", "").replace(" ", "") for name, _, _ in launches(call)], ws.numel()


@pytest.mark.parametrize("M,N,K,group,dtype,quads", [(1, 500, 1000, 128, F16, 1), (4, 700, 3000, 32, F32, 1), (5, 130, 2500, 64, BF16, 2), (8, 4096, 2048, 128, F16, 2),
                                                     (9, 300, 2100, 32, F16, 4), (16, 1000, 4096, 64, BF16, 4), (3, 9000, 300, 128, BF16, 1), (2, 40000, 130, 64, F16, 1), (8, 1000, 4097, 128, F16, 2),
                                                     (6, 300, 700, 32, BF16, 2)])
def test_few_rows(M, N, K, group, dtype, quads):
    names, workspace = run(M, N, K, group, dtype, FWD)
    assert names == [f"q4_few_rows_kernel<{CODE[dtype]},{group},{quads}>"] and workspace == 0


@pytest.mark.parametrize("M,N,K,group,dtype,direction,tile", [
    (12, 30000, 500, 128, F16, FWD, "1,2,2"), (7, 200, 600, 32, F32, FWD, "1,2,2"), (20, 300, 400, 64, BF16, FWD, "2,2,4"),
    (50, 260, 390, 128, F32, FWD, "2,2,2"), (70, 500, 900, 32, F16, FWD, "4,2,2"), (1010, 8150, 400, 128, BF16, FWD, "4,4,2"),
    (1020, 8190, 1300, 128, F16, FWD, "4,4,2"), (8, 5000, 3001, 64, F16, FWD, "1,2,2"), (1100, 2300, 300, 64, F16, FWD, "4,2,2"),
    (3, 300, 500, 128, F16, BWD, "1,2,2"), (16, 300, 500, 64, BF16, BWD, "1,1,2"), (30, 900, 2000, 128, BF16, BWD, "2,2,4"),
    (40, 500, 700, 32, F16, BWD, "2,1,4"), (20, 500, 700, 32, BF16, BWD, "2,1,4"), (90, 500, 700, 128, F16, BWD, "4,2,2"), (90, 500, 700, 64, BF16, BWD, "4,1,2"),
    (90, 500, 700, 32, F32, BWD, "1,1,2"), (90, 500, 700, 64, F32, BWD, "2,1,2")])
def test_tiles(M, N, K, group, dtype, direction, tile):
    names, workspace = run(M, N, K, group, dtype, direction)
    assert names[0] == f"q4_tile_kernel<{CODE[dtype]},{direction},{group},Tile<{tile}>>"
    assert names[1:] == ([f"q4_join_kernel<{CODE[dtype]}>"] if workspace else [])


def test_reduction_is_cut_where_tiles_are_few():
    for dtype in (F32, F16, BF16):
        names, workspace = run(33, 300, 5000, 128, dtype, FWD)
        assert names[1:] == [f"q4_join_kernel<{CODE[dtype]}>"] and workspace % (33 * 300 * 4) == 0 and workspace >= 2 * 33 * 300 * 4
        names, workspace = run(33, 5000, 300, 128, dtype, BWD)
        assert names[1:] == [f"q4_join_kernel<{CODE[dtype]}>"] and workspace % (33 * 300 * 4) == 0 and workspace >= 2 * 33 * 300 * 4


@pytest.mark.parametrize("R,V,top,masked,waves,slices", [(5, 2048, 3, False, 1, 1), (5, 2049, 3, True, 4, 1), (1, 200000, 20, True, 4, 25), (1024, 9000, 0, False, 4, 1),
                                                         (3, 1100000, 7, False, 4, 45), (2, 700, 0, True, 1, 1)])
def test_logprobs(R, V, top, masked, waves, slices):
    gen, x, targets = make_logits(R, V, BF16)
    mask = None
    if masked:
        mask = torch.rand((R, V), device=DEV, generator=gen) < 0.7
        mask[torch.arange(R, device=DEV), targets] = True
    check(x, targets, mask, 0.9, top)
    L, ws = nova.lib(), torch.empty(nova.nova_logprobs_workspace_bytes(R, V, top, BF16), dtype=torch.uint8, device=DEV)
    out = nova.nova_logprobs(x, targets, mask=mask, top=top, workspace=ws)
    found = launches(lambda: nova._check(L.nova_logprobs(
        x.data_ptr(), V, targets.data_ptr(), None if mask is None else mask.data_ptr(), V, R, V, 1.0, top, nova.NOVA_BF16, out.logprob.data_ptr(), out.entropy.data_ptr(),
        out.stats.data_ptr(), out.top_logprobs.data_ptr(), out.top_ids.data_ptr(), ws.data_ptr(), ws.numel(), nova._stream()), "nova_logprobs"))
    assert found[0] == (f"logprobs_kernel<2, {int(masked)}, {int(top > 0)}, {waves}>", R * slices, 64 * waves)
    assert [name for name, _, _ in found[1:]] == ([f"logprobs_join_kernel<2, {int(masked)}>"] if slices > 1 else [])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("V", [1500, 30000, 200000])
def test_alternatives_beyond_the_list(V, dtype):
    # more logits reach the bound than the list holds: all of a row equal, all of it equal but for the last entries, rows with little allowed
    x = torch.full((4, V), 1.5, device=DEV, dtype=dtype)
    x[1, -10:] = 3.0
    x[2] = torch.arange(V, device=DEV) % 5
    targets = torch.full((4,), V - 1, device=DEV)
    mask = torch.ones((4, V), dtype=torch.bool, device=DEV)
    mask[3] = torch.arange(V, device=DEV) % 97 == (V - 1) % 97
    for top in (1, 8, 64):
        check(x, targets, mask, 1.0, top)
