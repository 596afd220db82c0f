"""What linear_attn_workspace_bytes answers for batches without sequences, and for gradients without those of the decays (no GPU)."""
import ctypes

import pytest
import torch

import paper_2504_20490_amd as A
from paper_2504_20490_amd import binding as B

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


@pytest.mark.parametrize("rows,hint,d", [(32768, 10000, 128), (32768, 10000, 104), (3000, 3000, 64), (255, 255, 128), (256, 256, 8)])
def test_decays_that_are_not_wanted_take_no_states(rows, hint, d):
    """Two states for every 256 rows and KV head, and the bound that the call itself sets."""
    batch, size = A.LinearBatch(torch.zeros(8, dtype=torch.int32), hint), lambda **c: A.linear_attn_workspace_bytes(batch, rows, 8, 4, d, backward=True, **c)
    state = -(-d // 16) * 16 * -(-d // 32) * 32
    assert size() - size(decays=False) == 2 * 4 * (rows // 256) * 4 * state
    assert A.linear_attn_workspace_bytes(batch, rows, 8, 4, d, decays=False) == A.linear_attn_workspace_bytes(batch, rows, 8, 4, d)

    def call(d_log_decay, n):
        P = 1 << 20            # a pointer that is never followed: the workspace is too small
        args = B._LinearBatchArgs(P, None, None, 7, rows, hint, 8, 4, d)
        return A.load_library().hspmd_linear_attn_bwd(ctypes.byref(args), P, P, P, P, P, 8 * d, 4 * d, 4, 0.0, None, None, P, P, P, 0, d_log_decay, None, P, n, None)
    assert call(1 << 20, size() - 1) == 3 and call(None, size(decays=False) - 1) == 3
    if rows >= 256:
        assert call(1 << 20, size(decays=False)) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,f32", [(4, 4, 128, False), (8, 2, 64, True), (3, 3, 104, False)])
def test_gradients_without_the_decays_in_their_own_workspace(hq, hkv, d, f32):
    from linear_util import Case, check_backward
    case = Case([700, 33, 0, 1129], hq, hkv, d, 70, False, True).to_device()
    batch = case.batch(A)
    size = A.linear_attn_workspace_bytes(batch, case.rows, hq, hkv, d, backward=True, decays=False)
    ws = torch.full((size + 4096,), 90, dtype=torch.uint8, device="cuda")
    out = case.run_backward(A, f32=f32, decays=False, workspace=ws[:size])
    check_backward(case, out, f32)
    assert (ws[size:] == 90).all()
