"""Numbers of rows up to the largest that the calls of 4-bit layers and of log probabilities take: what their workspace queries, which the calls begin with, say
there.  CPU only."""
import pytest

from paper_2512_18453_amd import nova

F32, F16, BF16 = nova.NOVA_F32, nova.NOVA_F16, nova.NOVA_BF16
LARGEST = 2 ** 31 - 1


@pytest.mark.parametrize("V", [1, 5, 2048, 2049, 200000, LARGEST])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_many_rows_of_logits_are_not_cut(V, dtype):
    # (more rows than the chip has room for: one workgroup takes a whole row, and nothing has to be joined)
    for rows in (1024, 1 << 22, LARGEST - 1023, LARGEST - 1022, LARGEST - 1, LARGEST):
        assert nova.lib().nova_logprobs_workspace_bytes(rows, V, 5, dtype) == 0, rows


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("N,K,direction", [(1, 1 << 24, 0), (16, 1 << 24, 0), (1 << 24, 1, 1)])
def test_sums_of_many_rows_are_not_cut(N, K, direction, dtype):
    # (the rows fill the chip many times over, so pieces of the sum would only be written and read)
    for M in (1 << 30, LARGEST - 100, LARGEST - 32, LARGEST - 15, LARGEST):
        for group in (32, 128):
            assert nova.lib().nova_q4_linear_workspace_bytes(M, N, K, group, dtype, direction) == 0, (M, group)
