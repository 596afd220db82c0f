"""The paged cache on the GPU: the attention of new rows over it, the write, the read back, and all of them together, against the fp64
oracle."""
import math

import numpy as np
import pytest

from oracle import paged
from paged_util import BF16_HALF_STEP, E4M3_HALF_STEP, Batch, attend, bf16

pytestmark = pytest.mark.gpu

# What the attention may be off by, row by row.  O: the result's own rounding (half a bf16 step of the value) and that of every weight
# (half a step of P_j, so at most half a step of sum_j P_j |v_j|), fp32 sums and exponentials beside them less than 1e-4 of that sum.
# LSE: fp32 scores of at most 128 products, 2^-24 each against sum |q k|, and a logarithm and sum of fp32: 1e-4 is many times that.
LSE_ABS = 1e-4


def check_attention(b, hq, o, lse, q64, scale, k=None, v=None):
    k, v = b.k if k is None else k, b.v if v is None else v
    with np.errstate(invalid="ignore"):
        ref_o, ref_lse = paged.attention(q64, k, v, b.cu, b.kv, b.table, b.size, scale)
        mass, _ = paged.attention(q64, k, np.abs(v), b.cu, b.kv, b.table, b.size, scale)
    got = o.float().cpu().numpy().astype(np.float64)
    n = b.cu[-1]
    assert np.isnan(got[n:]).all()                                   # rows behind the last sequence: as they were
    ref_o, mass, got = ref_o[:n], mass[:n], got[:n]
    plain = np.isfinite(ref_o)
    assert np.array_equal(np.isnan(got), np.isnan(ref_o)) and np.array_equal(got[np.isinf(ref_o)], ref_o[np.isinf(ref_o)])
    tol = BF16_HALF_STEP * np.abs(ref_o[plain]) + (BF16_HALF_STEP + 1e-4) * mass[plain] + 1e-30
    worst = (np.abs(got[plain] - ref_o[plain]) / tol).max(initial=0.0)
    assert worst <= 1.0, worst
    if lse is not None:
        gl, ref_lse = lse.cpu().numpy().astype(np.float64), ref_lse[:, :n]
        assert np.isnan(gl[:, n:]).all()
        gl = gl[:, :n]
        fine = np.isfinite(ref_lse)
        assert np.array_equal(np.isinf(gl), np.isinf(ref_lse)) and np.array_equal(np.isnan(gl), np.isnan(ref_lse))
        worst = np.abs(gl[fine] - ref_lse[fine]).max(initial=0.0)
        assert worst <= LSE_ABS, worst


def rows_of_q(b, hq):
    import torch
    q64 = bf16(b.rng.standard_normal((b.T, hq, b.d)))
    return q64, torch.from_numpy(q64).to(torch.bfloat16).cuda()


def run_attention(rows, kv, hq, hkv, d, page_size, e4m3, seed=1, lse=True, scale=0.0, **more):
    import torch
    import paper_2504_20490_amd as A
    b = Batch(rows, kv, hkv, d, page_size, e4m3, seed, **more)
    b.device(A, interleaved=seed % 2 == 1)
    q64, q = rows_of_q(b, hq)
    o, l = attend(A, b, q, lse, scale)
    torch.cuda.synchronize()
    check_attention(b, hq, o, l, q64, scale or 1.0 / math.sqrt(d))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows,kv,hq,hkv,d,page_size", [
    ([1], [1], 1, 1, 128, 16),
    ([1], [1058], 5, 5, 128, 16),
    ([1, 1, 1], [31, 33, 640], 8, 2, 64, 16),
    ([1] * 5, [16, 17, 300, 2, 129], 16, 1, 104, 32),
    ([3, 1, 0, 7, 2], [40, 500, 20, 7, 129], 6, 3, 128, 64),
    ([0, 4, 1], [0, 2, 0], 4, 2, 64, 16),                 # fewer keys than rows: rows without a place; a row and no key at all
    ([2, 5], [300, 4000], 24, 2, 40, 256),                # 12 query heads per KV head: rows of a token fall into two tiles
    ([1, 1], [5000, 70], 2, 2, 8, 1024),
    ([1] * 70, list(range(1, 71)), 4, 4, 128, 16),        # more sequences than lanes
    ([1] * 300, [1 + 7 * i % 50 for i in range(300)], 1, 1, 64, 16),   # more than threads
])
def test_few_rows(rows, kv, hq, hkv, d, page_size, e4m3):
    run_attention(rows, kv, hq, hkv, d, page_size, e4m3, extra_rows=3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows,kv,hq,hkv,d,page_size", [
    ([130], [130], 2, 2, 128, 16),                        # a whole prompt
    ([200, 1, 33], [1000, 777, 40], 4, 2, 128, 16),       # chunks and a single token
    ([17, 64, 111], [17, 64, 111], 2, 2, 64, 16),
    ([40, 9], [2000, 65], 16, 2, 104, 32),
    ([100], [90], 4, 1, 64, 64),                          # the first ten rows have no place
    ([300], [1300], 3, 3, 80, 256),
    ([33, 0, 1, 140], [33, 50, 700, 2140], 10, 2, 40, 16),
    ([65], [4200], 8, 1, 96, 16),                         # few row tiles, many keys: shared out
])
def test_many_rows(rows, kv, hq, hkv, d, page_size, e4m3):
    run_attention(rows, kv, hq, hkv, d, page_size, e4m3, seed=2, extra_rows=2)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows,kv", [
    ([i % 3 for i in range(300)], [9000 if i == 100 else 2 + i * 13 % 200 for i in range(300)]),           # one long: shared out
    ([25 + i // 10 if i % 25 == 7 else i % 4 for i in range(250)], [2500 + i if i in (57, 111) else 60 + i % 50 for i in range(250)]),
    ([1] * 192, [5 + i for i in range(192)]),             # the most whose sums every workgroup makes
    ([1] * 193, [5 + i for i in range(193)]),             # the fewest that are planned
    ([0] * 1030 + [3] + [0] * 70, [7] * 1030 + [3000] + [1] * 70),
    ([0] * 200, [9] * 200),
])
def test_shares_planned_by_a_launch_in_front(rows, kv, e4m3):
    run_attention(rows, kv, 4, 2, 64, 16, e4m3, seed=18, extra_rows=3)


def test_replays_of_a_planned_batch():
    """More sequences than the workgroups sum over by themselves: a captured call follows the lengths, from a workspace that holds anything."""
    import torch
    import paper_2504_20490_amd as A
    rng = np.random.default_rng(19)
    seqs, width, hkv, hq, d, size, T = 230, 40, 1, 3, 64, 16, 600
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    cu, lens, table = ints(seqs + 1), ints(seqs), ints(seqs, width)
    pool = torch.from_numpy(rng.standard_normal((2, 500, hkv, size, d))).to(torch.bfloat16).cuda()
    cache, batch = A.KVCache(pool[0], pool[1]), A.KVBatch(cu, lens, table)
    q = torch.from_numpy(rng.standard_normal((T, hq, d))).to(torch.bfloat16).cuda()
    bytes_ = A.attn_paged_workspace_bytes(cache, batch, T, hq)
    got, want = ([torch.empty_like(q), torch.empty(hq, T, device="cuda"), torch.zeros(bytes_, dtype=torch.uint8, device="cuda")] for _ in range(2))
    call = lambda x: A.attn_paged_fwd(cache, batch, q, *x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(got)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(got)
    for most in (1, 3, 12, 0):
        rows = rng.integers(0, most + 1, seqs)
        rows[np.cumsum(rows) > T] = 0
        cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(rows)])).int())
        lens.copy_(torch.from_numpy(rng.integers(0, width * size, seqs)).int())
        table.copy_(torch.from_numpy(rng.integers(0, 500, (seqs, width))).int())
        for x in (got, want):
            x[0].fill_(float("nan")), x[1].fill_(float("nan")), x[2].fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        call(want)
        torch.cuda.synchronize()
        n = int(rows.sum())
        assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[1][:, :n], want[1][:, :n])
        assert not torch.isnan(got[0][:n].float()).any() and torch.isnan(got[0][n:].float()).all() and torch.isnan(got[1][:, n:]).all()


@pytest.mark.parametrize("max_rows", [0, 1, 5])
@pytest.mark.parametrize("rows,kv", [([70, 1, 9], [400, 300, 9]), ([90], [500])])
def test_a_wrong_hint_changes_no_result(rows, kv, max_rows):
    import torch
    import paper_2504_20490_amd as A
    b = Batch(rows, kv, 2, 128, 16, seed=14)
    b.device(A)
    b.batch = A.KVBatch(b.cu_dev, b.kv_dev, b.table_dev, max_rows)
    q64, q = rows_of_q(b, 6)
    o, lse = attend(A, b, q)
    torch.cuda.synchronize()
    check_attention(b, 6, o, lse, q64, 1.0 / math.sqrt(128))


def test_rows_in_front_of_the_first_sequence_are_left_alone():
    import torch
    import paper_2504_20490_amd as A
    b = Batch([2, 40], [3000, 300], 2, 64, 16, seed=15, extra_rows=5)
    b.device(A)
    _, q = rows_of_q(b, 4)
    want, want_lse = attend(A, b, q)
    shifted = torch.cat([q[-3:], q[:-3]])
    b.cu_dev += 3
    got, got_lse = attend(A, b, shifted)
    torch.cuda.synchronize()
    assert torch.equal(got[3:45], want[:42]) and torch.equal(got_lse[:, 3:45], want_lse[:, :42])
    assert torch.isnan(got[:3].float()).all() and torch.isnan(got[45:].float()).all() and torch.isnan(got_lse[:, :3]).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("seqs,rows,kv", [(40, 1, 20000), (9, 17, 40000)])
def test_more_pages_than_are_kept_at_a_time(seqs, rows, kv, e4m3):
    """So many heads that no keys are shared out, and a workgroup walks more pages than it keeps the numbers of (512 and 2048).  64 pages
    take turns in all of them."""
    import torch
    import paper_2504_20490_amd as A
    heads, d, size, distinct = 64, 8, 16, 64
    b = Batch([distinct * size], [distinct * size], heads, d, size, e4m3, seed=16, extra_pages=0, extra_width=0)
    cache, _ = b.device(A)
    table = np.resize(b.table[0], (seqs, -(-kv // size)))
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).int().cuda()
    b.cache, T = cache, seqs * rows
    b.batch = A.KVBatch(i32(np.arange(seqs + 1) * rows), i32(np.full(seqs, kv)), i32(table), rows)
    q64 = bf16(b.rng.standard_normal((T, heads, d)))
    o, lse = attend(A, b, torch.from_numpy(q64).to(torch.bfloat16).cuda())
    torch.cuda.synchronize()
    k, v = (paged.gather(pool, b.table[0], distinct * size, size) for pool in (b.k, b.v))
    where = np.argsort(b.table[0])[table]                                          # [seqs, pages]: which of the 64
    key = (where[:, :, None] * size + np.arange(size)).reshape(seqs, -1)[:, :kv]   # [seqs, kv]
    seq, pos = np.repeat(np.arange(seqs), rows), kv - rows + np.tile(np.arange(rows), seqs)
    for h in range(0, heads, 7):
        s = np.take_along_axis(q64[:, h] @ k[:, h].T / math.sqrt(d), key[seq], 1)  # [T, kv]
        s[np.arange(kv)[None] > pos[:, None]] = -np.inf
        top = s.max(-1, keepdims=True)
        w = np.exp(s - top)
        total = w.sum(-1, keepdims=True)
        per_key = np.stack([np.bincount(key[seq[t]], w[t] / total[t], distinct * size) for t in range(T)])
        ref, mass = per_key @ v[:, h], per_key @ np.abs(v[:, h])
        got = o[:, h].double().cpu().numpy()
        assert (np.abs(got - ref) <= BF16_HALF_STEP * np.abs(ref) + (BF16_HALF_STEP + 1e-4) * mass).all()
        assert (np.abs(lse[h].double().cpu().numpy() - (top + np.log(total))[:, 0]) <= LSE_ABS).all()


def test_thousands_of_sequences():
    """The rows' sequences are found among many; writes, reads and attends to 5000 of 0 to 3 rows."""
    import torch
    import paper_2504_20490_amd as A
    rng = np.random.default_rng(17)
    seqs, hkv, d, size = 5000, 1, 16, 16
    rows = rng.integers(0, 4, seqs)
    kv = rows + rng.integers(0, 20, seqs)
    cu = np.concatenate([[0], np.cumsum(rows)])
    T = int(cu[-1])
    table = np.stack([2 * np.arange(seqs), 2 * np.arange(seqs) + 1], 1)
    i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).int().cuda()
    pool = torch.from_numpy(rng.standard_normal((2, 2 * seqs, hkv, size, d))).to(torch.bfloat16).cuda()
    cache = A.KVCache(pool[0], pool[1])
    batch = A.KVBatch(i32(cu), i32(kv), i32(table), 3)
    x = torch.from_numpy(rng.standard_normal((T, 2, hkv, d))).to(torch.bfloat16).cuda()
    k, v = x[:, 0], x[:, 1]
    A.kv_cache_write(cache, batch, k, v)
    back = torch.empty(2, T, hkv, d, dtype=torch.bfloat16, device="cuda")
    A.kv_cache_read(cache, batch, back[0], back[1])
    q = torch.from_numpy(rng.standard_normal((T, 2, d))).to(torch.bfloat16).cuda()
    o, lse = torch.empty_like(q), torch.empty(2, T, device="cuda")
    ws = torch.empty(A.attn_paged_workspace_bytes(cache, batch, T, 2), dtype=torch.uint8, device="cuda")
    A.attn_paged_fwd(cache, batch, q, o, lse, ws)
    torch.cuda.synchronize()
    assert torch.equal(back[0], k) and torch.equal(back[1], v)
    keys, values = (p.double().cpu().numpy().reshape(seqs, 2 * size, d) for p in pool)       # (one head: a sequence's pages are neighbours)
    seq = np.repeat(np.arange(seqs), rows)
    pos = kv[seq] - rows[seq] + np.arange(T) - cu[seq]
    for h in range(2):
        s = np.einsum("td,tkd->tk", q[:, h].double().cpu().numpy(), keys[seq]) / 4.0
        s[np.arange(2 * size)[None] > pos[:, None]] = -np.inf
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        ref, mass = np.einsum("tk,tkd->td", w, values[seq]), np.einsum("tk,tkd->td", w, np.abs(values[seq]))
        assert (np.abs(o[:, h].double().cpu().numpy() - ref) <= BF16_HALF_STEP * np.abs(ref) + (BF16_HALF_STEP + 1e-4) * mass).all()


@pytest.mark.parametrize("scale", [0.01, 3.0])
def test_other_scales_and_no_lse(scale):
    run_attention([1, 40], [100, 300], 4, 2, 128, 16, False, seed=4, lse=False, scale=scale)
    run_attention([1, 40], [100, 300], 4, 2, 128, 16, True, seed=5, scale=scale)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [[1, 3, 1], [1, 150, 20]])
def test_pages_that_do_not_exist(rows, e4m3):
    """Rows that would see a key of such a page are NaN, the others right; neighbouring sequences as well."""
    import torch
    import paper_2504_20490_amd as A
    kv = [600, 400, 90]
    b = Batch(rows, kv, 2, 128, 16, e4m3, seed=7)
    b.table[0, 3] = b.num_pages                            # one past the last
    b.table[1, 22] = -5                                    # positions 352 .. 367: the later rows of the second sequence
    b.device(A)
    q64, q = rows_of_q(b, 4)
    o, lse = attend(A, b, q)
    torch.cuda.synchronize()
    check_attention(b, 4, o, lse, q64, 1.0 / math.sqrt(128))
    assert torch.isnan(o[0].float()).all() and not torch.isnan(o[b.cu[2]:].float()).any()


def test_lengths_and_rows_beyond_the_table_are_clamped():
    """kv_lens above what the page table holds, cu_rows above the tensors' rows and falling: nothing faults; the good sequence is right."""
    import torch
    import paper_2504_20490_amd as A
    b = Batch([1, 1, 1], [40, 64, 33], 2, 64, 16, seed=8, extra_width=0)
    b.device(A)
    q64, q = rows_of_q(b, 4)
    want, _ = attend(A, b, q)
    b.kv_dev[0] = 1 << 30                                  # the table holds 64 tokens a sequence; its third page onward is -1
    got, _ = attend(A, b, q)
    torch.cuda.synchronize()
    assert torch.equal(got[1:], want[1:]) and torch.isnan(got[0].float()).all()
    b.cu_dev.copy_(torch.tensor([0, 5, 2, 1 << 30], dtype=torch.int32))
    attend(A, b, q)
    b.cu_dev.copy_(torch.tensor([-7, 1, -1 << 31, 3], dtype=torch.int32))
    b.kv_dev.copy_(torch.tensor([-3, 64, 33], dtype=torch.int32))
    attend(A, b, q)
    k = torch.empty(b.T, 2, 64, dtype=torch.bfloat16, device="cuda")
    A.kv_cache_read(b.cache, b.batch, k, torch.empty_like(k))
    torch.cuda.synchronize()


def test_rows_cut_off_by_the_tensors_stand_at_the_same_positions_in_every_call():
    """cu_rows names more rows than the tensors have: the sequence has those that there are, its last ones, in write, read and attention."""
    import torch
    import paper_2504_20490_amd as A
    b = Batch([3, 10], [20, 40], 2, 64, 16, seed=22)
    b.device(A)
    _, q = rows_of_q(b, 4)
    x = torch.randn(b.T, 2, 64, device="cuda").bfloat16()
    A.kv_cache_write(b.cache, b.batch, x, -x)
    want, want_lse = attend(A, b, q)
    before = [t.clone() for t in b.cache.tensors]
    b.cu_dev[2] = 100
    A.kv_cache_write(b.cache, b.batch, x, -x)
    got, got_lse = attend(A, b, q)
    k, v = torch.empty_like(x), torch.empty_like(x)
    A.kv_cache_read(b.cache, b.batch, k, v)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_lse, want_lse) and torch.equal(k, x) and torch.equal(v, -x)
    for old, new in zip(before, b.cache.tensors):
        assert torch.equal(old.view(torch.int16), new.view(torch.int16))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [[6], [140]])
def test_infinities_and_nan_where_a_row_does_not_see_them(rows, e4m3):
    """A later row's key and value hold NaN and infinities: the rows before do not see them."""
    import torch
    import paper_2504_20490_amd as A
    n, kv = rows[0], 500
    b = Batch(rows, [kv], 2, 128, 16, e4m3, seed=9)
    for back, value in ((2, np.nan), (4, np.inf), (n // 2 + 2, -np.inf)):      # positions kv - back
        p = kv - back
        page, slot = b.table[0, p // 16], p % 16
        if e4m3:                                                               # (no infinities in 8 bits)
            b.v_code[page, :, slot, 5], b.k_code[page, :, slot, 7] = 127, 255
            b.v[page, :, slot, 5] = b.k[page, :, slot, 7] = np.nan
        else:
            b.v[page, :, slot, 5], b.k[page, 0, slot, 7] = value, np.nan
    b.device(A)
    q64, q = rows_of_q(b, 4)
    o, lse = attend(A, b, q)
    torch.cuda.synchronize()
    check_attention(b, 4, o, lse, q64, 1.0 / math.sqrt(128))


def test_results_do_not_change_from_run_to_run_nor_with_the_workspace():
    import torch
    import paper_2504_20490_amd as A
    b = Batch([1, 1, 200], [9000, 300, 2500], 2, 128, 16, seed=10)
    b.device(A)
    _, q = rows_of_q(b, 8)
    bytes_ = A.attn_paged_workspace_bytes(b.cache, b.batch, b.T, 8)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((bytes_,), fill, dtype=torch.uint8, device="cuda")
        for _ in range(3):
            o, lse = attend(A, b, q, workspace=ws)
            if first is None:
                first = (o, lse)
            assert torch.equal(o.view(torch.int16), first[0].view(torch.int16)) and torch.equal(lse, first[1])
    with pytest.raises(A.HspmdError) as e:
        attend(A, b, q, workspace=torch.empty(bytes_ - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3


# ------------------------------------------------------------------------------------------------ write and read
def write_case(rows, kv, hq, hkv, d, page_size, e4m3, rope, seed, axes=None, in_place=False):
    """Runs one write on a batch whose new rows' places hold NaN before; returns what the checks need."""
    import torch
    import paper_2504_20490_amd as A
    b = Batch(rows, kv, hkv, d, page_size, e4m3, seed, extra_rows=2)
    b.device(A, interleaved=seed % 2 == 0)
    fused = bf16(b.rng.standard_normal((b.T, hq + 2 * hkv, d)) * 3)
    dev = torch.from_numpy(fused).to(torch.bfloat16).cuda()
    q, k, v = dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]
    own = np.zeros(b.T, dtype=np.int64)
    for row, _, p, _, _ in paged.places(b.cu, b.kv, b.table, b.size, b.num_pages):
        own[row] = p
    placed = own >= 0                                       # (a row without a place stands at no position: its q becomes NaN)
    positions, pair_axis, args = own[None], [0] * (d // 2), {}
    if axes:
        positions = b.rng.integers(0, 50, (axes, b.T))
        pair_axis = [i * axes // (d // 2) for i in range(d // 2)]
    if rope:
        top = int(max(positions.max(), max(kv))) + 1
        table = torch.empty(top, d // 2, 2, device="cuda")
        A.rope_table(table, top, d)
        pos = torch.from_numpy(positions).int().cuda() if axes else None
        q_out = q if in_place else torch.full((b.T, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        args = dict(rope=A.RopeAxes(table, top, pos, pair_axis if axes else None), q=q, q_out=q_out)
    before = [None if t is None else t.clone() for t in b.cache.tensors]
    A.kv_cache_write(b.cache, b.batch, k, v, **args)
    torch.cuda.synchronize()
    where = np.ones(b.T, dtype=bool) if axes else placed
    turned = (lambda x: np.where(where[:, None, None], paged.turn_axes(x, positions, pair_axis), np.nan)) if rope else (lambda x: x)
    want = {"q": turned(fused[:, :hq]), "k": turned(fused[:, hq:hq + hkv]), "v": fused[:, hq + hkv:]}
    return b, before, want, fused, args.get("q_out")


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rope,axes", [(False, None), (True, None), (True, 3)])
@pytest.mark.parametrize("rows,kv,hq,hkv,d,page_size", [
    ([1], [1], 1, 1, 8, 16),
    ([1, 1, 1], [31, 33, 640], 8, 2, 128, 16),
    ([3, 0, 70], [40, 20, 70], 6, 3, 104, 32),
    ([4, 2], [2, 5], 4, 2, 64, 64),                       # two rows without a place
    ([1] * 80, list(range(1, 81)), 5, 5, 40, 16),
    ([5, 9], [300, 9], 2, 1, 96, 256),
])
def test_write(rows, kv, hq, hkv, d, page_size, rope, axes, e4m3):
    import torch
    b, before, want, fused, q_out = write_case(rows, kv, hq, hkv, d, page_size, e4m3, rope, 11 + d // 8, axes)
    # q: one rounding to bf16; the rotation in fp32 (two products and a sum, rounded: 3 * 2^-24 of |lo| + |hi|, and the table's own 2^-24)
    slack = 2.0 ** -21 * np.abs(fused).max()
    if rope:
        got = q_out.float().cpu().numpy()
        n = b.cu[-1]
        assert np.isnan(got[n:]).all()
        nowhere = np.isnan(want["q"][:n])
        assert np.array_equal(np.isnan(got[:n]), nowhere)
        assert ((np.abs(got[:n] - want["q"][:n]) <= BF16_HALF_STEP * np.abs(want["q"][:n]) + slack) | nowhere).all()
    after = [None if t is None else t for t in b.cache.tensors]
    written = np.zeros((b.num_pages, b.size), dtype=bool)
    for row, _, p, page, slot in paged.places(b.cu, b.kv, b.table, b.size, b.num_pages):
        if page >= 0:
            written[page, slot] = True
            for i, name in enumerate("kv"):
                x = want[name][row]
                if not e4m3:
                    got = after[i][page, :, slot].float().cpu().numpy()
                    assert (np.abs(got - x) <= BF16_HALF_STEP * np.abs(x) + (slack if rope and name == "k" else 0)).all()
                    continue
                codes, byte = after[i].view(torch.uint8)[page, :, slot].cpu().numpy(), after[2 + i][page, :, slot].cpu().numpy()
                ref_codes, ref_byte = paged.quantise(x)
                assert (codes[:, d:] == 0).all()
                if not rope or name == "v":
                    assert np.array_equal(codes[:, :d], ref_codes) and np.array_equal(byte, ref_byte)
                else:
                    top = np.abs(x).max(-1)                  # (at a border the fp32 rotation may fall on the other side)
                    border = np.abs(np.log2(top / 448.0) - np.round(np.log2(top / 448.0))) < 1e-5
                    assert (border | (byte == ref_byte)).all()
                    unit = 2.0 ** (byte.astype(np.float64) - 127)[:, None]
                    # normal numbers half a step, below 2^-6 half a step of 2^-9
                    assert (np.abs(paged.dequantise(codes[:, :d], byte) - x) <= E4M3_HALF_STEP * np.abs(x) + 2.0 ** -10 * unit + slack).all()
    for x, y in zip(before, after):                          # every other slot: bit for bit as it was
        if x is not None:
            bits = lambda t: t.contiguous().view(torch.uint8).cpu().numpy().reshape(b.num_pages, hkv, b.size, -1)
            keep = np.broadcast_to(~written[:, None, :, None], bits(x).shape)
            assert np.array_equal(bits(x)[keep], bits(y)[keep])


def test_write_turns_q_in_place():
    b, _, want, fused, q_out = write_case([3, 20], [50, 20], 4, 2, 128, 16, True, True, 21, None, in_place=True)
    got = q_out.float().cpu().numpy()[:23]
    assert (np.abs(got - want["q"][:23]) <= BF16_HALF_STEP * np.abs(want["q"][:23]) + 2.0 ** -21 * np.abs(fused).max()).all()


def test_write_of_special_values():
    """Zeros, infinities, NaN, the smallest and largest numbers, maxima at and around a power of two."""
    import torch
    import paper_2504_20490_amd as A
    b = Batch([8], [8], 1, 16, 16, True, seed=3)
    b.device(A)
    x = np.zeros((8, 1, 16))
    x[1, 0, :4] = [np.inf, -2.0, np.nan, 448.0]
    x[2] = np.nan
    x[3, 0, :3] = [2.0 ** -126, -2.0 ** -120, 2.0 ** -112]
    x[4, 0, :3] = [3.3895313892515355e38, -1.0, 2.0 ** 100]           # the largest bf16 number
    x[5, 0, :4] = [448.0, 447.0 - 447.0 % 2, 1.0, 2.0 ** -9]
    x[6, 0, :3] = [450.0, 224.0, 226.0]                               # just above a border: the next scale
    x[7, 0] = np.linspace(-1.0, 1.0, 16)
    x = bf16(x)
    k = torch.from_numpy(x).to(torch.bfloat16).cuda()
    A.kv_cache_write(b.cache, b.batch, k, k)
    torch.cuda.synchronize()
    page = b.table[0, 0]
    codes, byte = paged.quantise(x)
    for i in (0, 1):
        got = b.cache.tensors[i].view(torch.uint8)[page, :, :8].cpu().numpy().transpose(1, 0, 2)
        assert np.array_equal(b.cache.tensors[2 + i][page, :, :8].cpu().numpy().T, byte)
        same = (got == codes) | ((got & 127 == 127) & (codes & 127 == 127)) | ((got & 127 == 0) & (codes & 127 == 0))
        assert same.all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows,kv,hkv,d,page_size", [
    ([1], [1], 1, 8, 16), ([17, 64, 111], [17, 64, 111], 2, 64, 16), ([3, 0, 70, 2], [40, 20, 700, 2], 3, 104, 32),
    ([4, 2], [2, 5], 2, 128, 64), ([1] * 70, [9] * 70, 5, 40, 16), ([300], [1300], 1, 80, 256)])
def test_read(rows, kv, hkv, d, page_size, e4m3):
    import torch
    import paper_2504_20490_amd as A
    b = Batch(rows, kv, hkv, d, page_size, e4m3, 5 + d, extra_rows=2)
    if rows == [3, 0, 70, 2]:
        b.table[2, 20] = -1                                   # positions 640 .. 671
    b.device(A, interleaved=d % 16 == 0)
    both = torch.full((b.T, 2 * hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    A.kv_cache_read(b.cache, b.batch, both[:, :hkv], both[:, hkv:])
    torch.cuda.synchronize()
    got = both.float().cpu().numpy()
    assert (got[b.cu[-1]:] == 7.0).all()
    for row, _, p, page, slot in paged.places(b.cu, b.kv, b.table, b.size, b.num_pages):
        for x, pool in ((got[row, :hkv], b.k), (got[row, hkv:], b.v)):
            want = np.zeros_like(x) if p < 0 else np.full_like(x, np.nan) if page < 0 else pool[page, :, slot]
            assert np.array_equal(x, want, equal_nan=True), (row, p)


def test_write_skips_pages_that_do_not_exist():
    import torch
    import paper_2504_20490_amd as A
    b = Batch([20], [36], 2, 64, 16, False, seed=6)
    b.table[0, 1] = b.num_pages + 3
    b.device(A)
    before = [t.clone() for t in b.cache.tensors[:2]]
    x = torch.ones(20, 2, 64, dtype=torch.bfloat16, device="cuda")
    A.kv_cache_write(b.cache, b.batch, x, x)
    torch.cuda.synchronize()
    last = b.table[0, 2]
    for old, new in zip(before, b.cache.tensors):
        assert (new[last, :, :4] == 1).all()
        new[last, :, :4] = old[last, :, :4]
        assert torch.equal(new.view(torch.int16), old.view(torch.int16))


# ------------------------------------------------------------------------------------------------ together
def generate(A, cache_dtype, hq, hkv, d, prompts, steps, page_size, chunk, seed):
    """Prompts in chunks, then single tokens: write with rotation, attend, step by step.  Returns per sequence the unrotated q, k, v and the
    attention's results."""
    import torch
    rng = np.random.default_rng(seed)
    total = [p + steps for p in prompts]
    x = [bf16(rng.standard_normal((n, hq + 2 * hkv, d))) for n in total]
    width = -(-max(total) // page_size)
    pages = rng.permutation(width * len(prompts)).reshape(len(prompts), width)
    row = d if cache_dtype == torch.bfloat16 else A.kv_cache_row(d, A.CACHE_E4M3)
    shape = (pages.size, hkv, page_size, row)
    pools = [torch.full(shape, 255, dtype=torch.uint8, device="cuda").view(cache_dtype) if cache_dtype != torch.bfloat16
             else torch.full(shape, float("nan"), dtype=cache_dtype, device="cuda") for _ in range(2)]
    scales = [torch.full(shape[:3], 255, dtype=torch.uint8, device="cuda") for _ in range(2)] if cache_dtype != torch.bfloat16 else [None, None]
    cache = A.KVCache(*pools, *scales, head_dim=d)
    table = torch.empty(max(total), d // 2, 2, device="cuda")
    A.rope_table(table, max(total), d)
    rope = A.RopeAxes(table, max(total))
    page_dev = torch.from_numpy(pages).int().cuda()
    done, out = [0] * len(prompts), [[] for _ in prompts]
    while any(a < b for a, b in zip(done, total)):
        rows = [min(chunk, p - a) if a < p else min(1, n - a) for a, p, n in zip(done, prompts, total)]
        lens = [a + r for a, r in zip(done, rows)]
        cu = np.concatenate([[0], np.cumsum(rows)])
        ints = lambda y: torch.tensor(y, dtype=torch.int32, device="cuda")
        batch = A.KVBatch(ints(cu), ints(lens), page_dev, max(rows))
        packed = torch.from_numpy(np.concatenate([y[a:b] for y, a, b in zip(x, done, lens)])).to(torch.bfloat16).cuda()
        q, k, v = packed[:, :hq], packed[:, hq:hq + hkv], packed[:, hq + hkv:]
        q_rot = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        A.kv_cache_write(cache, batch, k, v, rope=rope, q=q, q_out=q_rot)
        o, lse = torch.empty_like(q_rot), torch.empty(hq, q.shape[0], device="cuda")
        ws = torch.empty(A.attn_paged_workspace_bytes(cache, batch, q.shape[0], hq), dtype=torch.uint8, device="cuda")
        A.attn_paged_fwd(cache, batch, q_rot, o, lse, ws)
        for s, r in enumerate(rows):
            out[s].append(o[cu[s]:cu[s + 1]])
        done = lens
    torch.cuda.synchronize()
    return x, [torch.cat(y) for y in out], cache, page_dev, total, rope


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (3, 3, 104), (8, 1, 64)])
def test_generation_matches_whole_sequence_attention(hq, hkv, d, e4m3):
    """A chunked prompt and single tokens, through the cache, against rotation and causal attention over whole sequences in 64 bits; and
    the cache read back gives the library's own packed attention the same results."""
    import torch
    import paper_2504_20490_amd as A
    prompts, steps = [37, 1, 150], 6
    x, outs, cache, pages, total, rope = generate(A, torch.float8_e4m3fn if e4m3 else torch.bfloat16, hq, hkv, d, prompts, steps, 16, 48, 31)
    ints = lambda y: torch.tensor(y, dtype=torch.int32, device="cuda")
    cu, _, T = A.build_cu_seqlens(total)
    k, v = (torch.empty(T, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    A.kv_cache_read(cache, A.KVBatch(ints(cu), ints(total), pages, max(total)), k, v)
    plan = A.Plan(cu, hq, hkv, d)
    q = torch.from_numpy(np.concatenate([y[:, :hq] for y in x])).to(torch.bfloat16).cuda()
    q_rot, k_same = torch.empty_like(q), torch.empty_like(k)
    A.rope_qk(plan, q, k, q_rot, k_same, rope.table, max(total))
    o, lse = torch.empty_like(q), torch.empty(hq, T, device="cuda")
    A.attn_varlen_fwd(plan, q_rot, k, v, o, lse)
    torch.cuda.synchronize()
    for s, n in enumerate(total):
        pos = np.arange(n)[None]
        turn = lambda y: paged.turn_axes(y, pos, [0] * (d // 2))
        qs, ks, vs = turn(x[s][:, :hq]), turn(x[s][:, hq:hq + hkv]), x[s][:, hq + hkv:]
        got = outs[s].float().cpu().numpy().astype(np.float64)
        packed = o[cu[s]:cu[s + 1]].float().cpu().numpy()
        kr, vr = (t[cu[s]:cu[s + 1]].float().cpu().numpy().astype(np.float64) for t in (k, v))
        # what the cache holds is what was written: bf16 half a step, e4m3 half a step of its own
        step = E4M3_HALF_STEP if e4m3 else BF16_HALF_STEP
        floor = 2.0 ** -10 * 2.0 ** -5 if e4m3 else 0.0      # (rows of magnitude below 8: scales of 2^-5 at most)
        for a, want in ((kr, ks), (vr, vs)):
            assert (np.abs(a - want) <= step * np.abs(want) + floor + 2.0 ** -20).all()
        # the attention against the same formulas in 64 bits on the cache's values and the rotated, rounded q
        one = lambda y: y.reshape(1, n, y.shape[1], d).transpose(0, 2, 1, 3)
        ref, _ = paged.attention(bf16(qs), one(kr), one(vr), [0, n], [n], [[0]], n, 1 / math.sqrt(d))
        mass, _ = paged.attention(bf16(qs), one(kr), one(np.abs(vr)), [0, n], [n], [[0]], n, 1 / math.sqrt(d))
        # (q: the fp32 rotation may round the other way where it falls on a border, a bf16 step of single elements: 1e-3 of the mass)
        tol = BF16_HALF_STEP * np.abs(ref) + (BF16_HALF_STEP + 1e-3) * mass
        assert (np.abs(got - ref) <= tol).all() and (np.abs(packed - ref) <= tol).all()


def test_graph_replays_follow_the_lengths_on_the_device():
    """Write, attention and read captured once and replayed with other lengths, pages and values, eager work in between; the batch is
    padded: sequences without rows, rows without sequence."""
    import torch
    import paper_2504_20490_amd as A
    hq, hkv, d, size, seqs, rows_most = 8, 2, 128, 16, 6, 12
    rng = np.random.default_rng(3)
    width = 64
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    cu, lens, table = ints(seqs + 1), ints(seqs), ints(seqs, width)
    new = lambda: torch.from_numpy(rng.standard_normal((rows_most, hq + 2 * hkv, d))).to(torch.bfloat16).cuda()
    packed = new()
    tab = torch.empty(size * width, d // 2, 2, device="cuda")
    A.rope_table(tab, size * width, d)
    rope = A.RopeAxes(tab, size * width)
    pool = [torch.from_numpy(rng.standard_normal((seqs * width, hkv, size, d))).to(torch.bfloat16).cuda() for _ in range(2)]
    batch = A.KVBatch(cu, lens, table, 0)

    def buffers():
        cache = A.KVCache(*[p.clone() for p in pool])
        ws = torch.empty(A.attn_paged_workspace_bytes(cache, batch, rows_most, hq), dtype=torch.uint8, device="cuda")
        e = lambda h: torch.zeros(rows_most, h, d, dtype=torch.bfloat16, device="cuda")
        return dict(cache=cache, ws=ws, q=e(hq), o=e(hq), lse=torch.zeros(hq, rows_most, device="cuda"), k=e(hkv), v=e(hkv))

    def calls(x):
        q, k, v = packed[:, :hq], packed[:, hq:hq + hkv], packed[:, hq + hkv:]
        A.kv_cache_write(x["cache"], batch, k, v, rope=rope, q=q, q_out=x["q"])
        A.attn_paged_fwd(x["cache"], batch, x["q"], x["o"], x["lse"], x["ws"])
        A.kv_cache_read(x["cache"], batch, x["k"], x["v"])

    captured, eager = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls(captured)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(captured)
    for replay in range(4):
        rows = [[1] * 6, [1, 0, 3, 0, 2, 1], [12, 0, 0, 0, 0, 0], [0] * 6][replay]
        n = [int(rng.integers(r, size * width)) if r else 0 for r in rows]
        cu.copy_(torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32))
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        table.copy_(torch.from_numpy(rng.permutation(seqs * width).reshape(seqs, width)).int())
        packed.copy_(new())
        for x in (captured, eager):
            for name in ("q", "o", "lse", "k", "v"):
                x[name].fill_(float("nan"))
            x["ws"].fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        calls(eager)
        torch.cuda.synchronize()
        for name in ("q", "o", "lse", "k", "v"):
            bits = lambda t: t.view(torch.int32 if t.element_size() == 4 else torch.int16)
            assert torch.equal(bits(captured[name]), bits(eager[name])), (replay, name)
            valid = sum(rows)
            done = captured[name][:, :valid] if name == "lse" else captured[name][:valid]
            rest = captured[name][:, valid:] if name == "lse" else captured[name][valid:]
            assert not torch.isnan(done.float()).any() and torch.isnan(rest.float()).all()
        for a, c in zip(captured["cache"].tensors[:2], eager["cache"].tensors[:2]):
            assert torch.equal(a.view(torch.int16), c.view(torch.int16))


def test_two_streams_with_workspaces_of_their_own():
    import torch
    import paper_2504_20490_amd as A
    work = []
    for seed in (41, 42):
        b = Batch([1, 60], [3000, 900], 2, 128, 16, seed=seed)
        b.device(A)
        _, q = rows_of_q(b, 8)
        want = attend(A, b, q)
        ws = torch.empty(A.attn_paged_workspace_bytes(b.cache, b.batch, b.T, 8), dtype=torch.uint8, device="cuda")
        work.append((b, q, want, ws, torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for b, q, _, ws, stream in work:
            with torch.cuda.stream(stream):
                got.append(attend(A, b, q, workspace=ws))
    torch.cuda.synchronize()
    for i, (o, lse) in enumerate(got):
        want = work[i % 2][2]
        assert torch.equal(o.view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse, want[1])


@pytest.mark.parametrize("e4m3", [False, True])
def test_pool_beyond_32_bit_offsets(e4m3):
    """Pages at the far end of a pool of more than 2^32 bytes, of k and of v each."""
    import torch
    import paper_2504_20490_amd as A
    hkv, d, size = 8, 128, 64
    dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
    per_page = hkv * size * d * dtype.itemsize
    pages = (1 << 32) // per_page + 100
    b = Batch([1, 70], [200, 150], hkv, d, size, e4m3, seed=12)
    pools = [torch.empty(pages, hkv, size, d, dtype=torch.uint8 if e4m3 else dtype, device="cuda") for _ in range(2)]
    scales = [torch.empty(pages, hkv, size, dtype=torch.uint8, device="cuda") for _ in range(2)] if e4m3 else [None, None]
    small, _ = b.device(A)
    first = pages - b.num_pages
    for big, x in zip(pools + scales, small.tensors):
        if x is not None:
            big[first:] = x.view(big.dtype) if e4m3 else x
    q64, q = rows_of_q(b, 8)
    want = attend(A, b, q)
    table = torch.where(b.table_dev >= 0, b.table_dev + first, b.table_dev)
    b.cache = A.KVCache(*[p.view(dtype) for p in pools], *scales, head_dim=d)
    b.batch = A.KVBatch(b.cu_dev, b.kv_dev, table, 70)
    got = attend(A, b, q)
    k, k_want = (torch.empty(b.T, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    v, v_want = torch.empty_like(k), torch.empty_like(k)
    A.kv_cache_read(b.cache, b.batch, k, v)
    A.kv_cache_read(small, A.KVBatch(b.cu_dev, b.kv_dev, b.table_dev, 70), k_want, v_want)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(k, k_want) and torch.equal(v, v_want)
    A.kv_cache_write(b.cache, b.batch, v, k)
    A.kv_cache_read(b.cache, b.batch, k_want, v_want)
    torch.cuda.synchronize()
    assert torch.equal(k_want, v) and torch.equal(v_want, k)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d", range(8, 129, 8))
def test_every_head_dim(d, e4m3):
    test_write([2, 40], [40, 41], 4, 2, d, 16, True, None, e4m3)
    test_read([2, 40], [40, 41], 3, d, 16, e4m3)
    run_attention([1, 45], [100, 150], 4, 2, d, 16, e4m3, seed=23, extra_rows=1)
