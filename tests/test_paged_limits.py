"""Sizes at the limits of the calls around the paged cache (no GPU): what the binding and the library say to them."""
import pytest
import torch

import paper_2504_20490_amd as A


def pool(h=2, size=16, d=64, pages=3):
    return [torch.zeros(pages, h, size, d, dtype=torch.bfloat16) for _ in range(2)]


def batch(seqs=2, width=8, max_rows=0):
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return A.KVBatch(i(seqs + 1), i(seqs), i(seqs, width), max_rows)


@pytest.mark.parametrize("rows,heads", [(12, 3), (12, 0), (12, -2), (-1, 4), ((1 << 25) + 1, 2), ((1 << 19) + 1, 64), (0, 3)])
def test_the_workspace_of_a_refused_batch_is_an_error(rows, heads):
    with pytest.raises(A.HspmdError) as e:
        A.attn_paged_workspace_bytes(A.KVCache(*pool()), batch(), rows, heads)
    assert e.value.status == 1 and ("total_rows" in str(e.value) or "local_q_heads" in str(e.value))


def test_the_workspace_of_an_unsupported_head_dim_is_an_error():
    with pytest.raises(A.HspmdError) as e:
        A.attn_paged_workspace_bytes(A.KVCache(*pool(d=60)), batch(), 12, 4)
    assert e.value.status == 2 and "head_dim" in str(e.value)


def test_a_batch_with_nothing_to_do_takes_no_workspace():
    cache = A.KVCache(*pool())
    assert A.attn_paged_workspace_bytes(cache, batch(), 0, 4) == 0 and A.attn_paged_workspace_bytes(cache, batch(seqs=0), 5, 4) == 0
    assert A.attn_paged_workspace_bytes(cache, batch(), 5, 4) > 0
