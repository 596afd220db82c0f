"""Sizes at the limits of the calls around the paged cache (no GPU): what the binding and the library say to them."""
import ctypes
import random

import pytest
import torch

import paper_2504_20490_amd as A
from paper_2504_20490_amd import binding


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


def test_the_stated_limits_are_the_ones_that_hold():
    """The largest sizes that the header names are taken, the next ones are not."""
    lib, cache = A.load_library(), A.KVCache(*pool())
    size = lambda heads=2, **change: lib.hspmd_attn_paged_workspace_bytes(cache._ref, ctypes.byref(with_(**change)), heads)

    def with_(num_seqs=2, total_rows=5):
        b = batch()._with_rows(total_rows)._obj
        b.num_seqs = num_seqs
        return b

    assert size(total_rows=1 << 24) > 0 and size(total_rows=(1 << 24) + 1) == 0               # 2^25 rows x heads
    assert size(num_seqs=1 << 25) > 0 and size(num_seqs=(1 << 25) + 1) == 0
    assert size(heads=(1 << 25) // 5 // 2 * 2) > 0 and size(heads=((1 << 25) // 5 // 2 + 1) * 2) == 0
    one = A.KVCache(*pool(h=1))
    rows = lambda n: lib.hspmd_attn_paged_workspace_bytes(one._ref, batch()._with_rows(n), 1)
    assert rows(1 << 25) > 0 and rows((1 << 25) + 1) == 0
    P = 1 << 20                                             # never followed
    rope = binding._RopeAxesArgs(P, 100, 1, P, 1 << 26, None)
    for d, hq, hkv, tokens in ((8, 65537, 0, 5), (8, 1, 65537, 5), (8, 1, 1, (1 << 25) + 1), (8, -1, 0, 5)):
        assert lib.hspmd_rope_axes_qk(ctypes.byref(rope), P, P, 1 << 20, 1 << 20, P, P, 1 << 20, 1 << 20, tokens, hq, hkv, d, 0, 0, None) == 1
        assert b"65536" in lib.hspmd_last_error() or b"2^25" in lib.hspmd_last_error()
    for heads in (0, 65537):
        assert lib.hspmd_kv_cache_write(cache._ref, batch()._with_rows(5), P, P, 128, ctypes.byref(rope), P, P, 1 << 23, 1 << 23, heads, None) == 1
        assert b"65536" in lib.hspmd_last_error()
    cache._args.local_kv_heads, cache._args.page_stride = 65537, 1 << 40
    assert size(heads=65537) == 0 and b"65536" in lib.hspmd_last_error()



def test_the_workspace_for_one_cache_never_shrinks_with_the_batch():
    """A buffer for the largest batch serves every smaller one: each of the four sizes alone, at every step, over caches of several shapes."""
    rng = random.Random(3)
    lib = A.load_library()
    pointer = 1 << 20
    for _ in range(300):
        h, d, size = rng.choice([1, 2, 3, 8]), rng.choice([8, 64, 72, 128]), rng.choice([16, 64, 1024])
        cache = binding._KVCacheArgs(pointer, pointer, None, None, h * size * d, 0, 10, size, h, d, A.CACHE_BF16)
        at = dict(num_seqs=rng.choice([1, 2, 30, 192, 5000]), table_width=rng.choice([0, 1, 3, 200, 8192]), total_rows=rng.choice([1, 2, 3, 17, 300, 5000]),
                  group=rng.choice([1, 2, 5, 16, 17, 64]))

        def bytes_(num_seqs, table_width, total_rows, group, max_rows=0):
            batch = binding._KVBatchArgs(pointer, pointer, pointer, num_seqs, table_width, total_rows, max_rows)
            return lib.hspmd_attn_paged_workspace_bytes(ctypes.byref(cache), ctypes.byref(batch), group * h)

        for name, value in at.items():
            last = 0
            for more in sorted([value + i for i in range(20)] + [value * 2, value * 7 + 11, value * 40 + 1]):
                changed = dict(at, **{name: more})
                if changed["total_rows"] * changed["group"] * h > 1 << 25:
                    break
                now = bytes_(**changed)
                assert now >= last, (name, more, at, h, d, size)
                last = now
        assert bytes_(**at) == bytes_(**at, max_rows=1) == bytes_(**at, max_rows=10 ** 6)


def test_counts_that_do_not_fit_32_bits_are_refused_not_cut():
    """2^32 + 12 rows are not 12."""
    cache, wide = A.KVCache(*pool()), 1 << 32
    rows = lambda n, h: torch.zeros(1, 1, 1, dtype=torch.bfloat16).expand(n, h, 64)
    table = torch.zeros(10, 32, 2)

    def refused(f, *args, **kw):
        with pytest.raises(A.HspmdError) as e:
            f(*args, **kw)
        assert e.value.status == 1 and "32 bits" in str(e.value)

    for n in (wide + 12, 1 << 31, -wide + 12):
        refused(A.attn_paged_workspace_bytes, cache, batch(), n, 4)
        refused(A.attn_paged_workspace_bytes, cache, batch(), 12, n)
        refused(batch, max_rows=n)
        refused(A.RopeAxes, table, n)
    for x, q in ((rows(wide + 5, 2), rows(wide + 5, 4)), (rows(wide + 5, 2), rows(5, wide + 4))):
        refused(A.kv_cache_read, cache, batch(), x, x)
        refused(A.kv_cache_write, cache, batch(), x, x)
        refused(A.attn_paged_fwd, cache, batch(), q, q, None, table)
        refused(A.rope_axes_qk, A.RopeAxes(table, 10), q, None, q, None)
    meta = lambda *s: torch.empty(*s, dtype=torch.int32, device="meta")
    refused(A.KVBatch, meta(2), meta(1), meta(1, 1 << 31))
