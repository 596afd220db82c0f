"""What linear_attn_workspace_bytes answers for batches without sequences (no GPU)."""
import pytest
import torch

import paper_2504_20490_amd as A

none = lambda: A.LinearBatch(torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("rows", [0, 10, 1 << 20])
def test_no_sequence_takes_none(rows, backward):
    """Rows behind the last sequence may be all there is."""
    assert A.linear_attn_workspace_bytes(none(), rows, 4, 2, 64, backward=backward) == 0
    if rows == 0:
        assert A.linear_attn_workspace_bytes(A.LinearBatch(), rows, 4, 2, 64, backward=backward) == 0


@pytest.mark.parametrize("counts", [(10, 4, 2, 60), (10, 3, 2, 64), (0, 4, 0, 64), (1 << 26, 4, 2, 64), (10, 4, 2, 0)])
def test_counts_that_make_no_sense_are_refused_all_the_same(counts):
    for batch in (none(), A.LinearBatch(), A.LinearBatch(torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(A.HspmdError) as e:
            A.linear_attn_workspace_bytes(batch, *counts)
        assert e.value.status == 1 and str(e.value).strip()
