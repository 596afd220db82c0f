"""The attention over the paged cache where a token's query heads outnumber a tile's rows or a wave's, and where one long sequence meets many
short rows in one call; the largest numbers of the 8-bit cache.  Oracle and tolerances are those of test_gpu_paged."""
import numpy as np
import pytest

from oracle import paged
from paged_util import BF16_HALF_STEP, Batch, attend, bf16
from test_gpu_paged import LSE_ABS, check_attention, rows_of_q, run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("group", [17, 32, 33, 40, 136, 300])
@pytest.mark.parametrize("rows,kv,kv_heads,d", [
    ([1], [300], 1, 128),
    ([1, 1, 1], [31, 129, 640], 2, 64),
    ([3, 0, 2], [200, 70, 65], 1, 104),                   # a token in two tiles, a tile of two tokens
    ([1, 30, 1], [500, 90, 7], 1, 64),
    ([1], [9000], 1, 64),                                 # keys shared out
    ([5, 1], [3, 0], 1, 40),                              # rows without a place, and no key at all
])
def test_groups_above_a_tile_of_few_rows(rows, kv, kv_heads, d, group, e4m3):
    """17: the fewest that single tokens leave the kernel for few rows with; 32, 33, 40: whole waves without a row; 136, 300: a token in several tiles."""
    run_attention(rows, kv, group * kv_heads, kv_heads, d, 16, e4m3, seed=24 + group % 2, extra_rows=2)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("group", [17, 40, 136])
def test_hidden_infinities_and_nan_with_large_groups(group, e4m3):
    """The last token's key and value, and the one's in the middle, are not finite: the tokens before do not see them."""
    import torch
    import paper_2504_20490_amd as A
    kv = 200
    b = Batch([4], [kv], 1, 128, 16, e4m3, seed=26)
    for back, value in ((1, np.nan), (3, np.inf)):
        page, slot = b.table[0, (kv - back) // 16], (kv - back) % 16
        if e4m3:
            b.v_code[page, :, slot, 5], b.k_code[page, :, slot, 7] = 127, 255
            b.v[page, :, slot, 5] = b.k[page, :, slot, 7] = np.nan
        else:
            b.v[page, :, slot, 5] = value
    b.device(A)
    q64, q = rows_of_q(b, group)
    o, lse = attend(A, b, q)
    torch.cuda.synchronize()
    check_attention(b, group, o, lse, q64, 1.0 / np.sqrt(128))
    assert torch.isfinite(o[0].float()).all() and not torch.isfinite(o[3].float()).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows,kv,hq,hkv", [([1, 700], [20000, 700], 8, 2), ([70, 1, 40, 1], [90, 9000, 40, 30000], 40, 1)])
def test_one_long_sequence_among_many_rows(rows, kv, hq, hkv, e4m3):
    """More than 4096 (row, head) pairs, a few of which have results of many chunks to join."""
    run_attention(rows, kv, hq, hkv, 64, 16, e4m3, seed=27, extra_rows=3)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows,kv,hq,hkv,d", [([1, 1, 1], [2, 5, 40], 8, 2, 128), ([3, 2], [6, 300], 5, 1, 64), ([1], [3000], 4, 1, 104), ([2, 60], [9, 60], 4, 1, 64)])
def test_few_rows_are_off_by_their_own_rounding_alone(rows, kv, hq, hkv, d, e4m3):
    """Weights go into their product as their upper 8 bits and a rest (below 2^-7 of the weight) rounded to 8: O is off by half a bf16 step of its value, and
    by 2^-8 of 2^-7 and what fp32 scores and sums leave (1e-4, as in test_gpu_paged) of sum_j P_j |v_j|."""
    import torch
    import paper_2504_20490_amd as A
    b = Batch(rows, kv, hkv, d, 16, e4m3, seed=29)
    b.device(A)
    q64, q = rows_of_q(b, hq)
    o, _ = attend(A, b, q)
    torch.cuda.synchronize()
    n = b.cu[1] if max(rows) * hq // hkv > 16 else b.T                             # (the other sequence is for the kernel for many rows)
    ref, _ = paged.attention(q64, b.k, b.v, b.cu, b.kv, b.table, b.size, d ** -0.5)
    mass, _ = paged.attention(q64, b.k, np.abs(b.v), b.cu, b.kv, b.table, b.size, d ** -0.5)
    off = np.abs(o.double().cpu().numpy() - ref)[:n]
    assert (off <= BF16_HALF_STEP * np.abs(ref[:n]) + (2.0 ** -15 + 1e-4) * mass[:n]).all()


@pytest.mark.parametrize("rows", [[1], [7], [90]])
def test_infinite_values_make_infinite_results(rows):
    """An infinity of a value that a row sees stands in that column of its result, with the value's sign, whatever its weight (one key: 1)."""
    import torch
    import paper_2504_20490_amd as A
    b = Batch([1] + rows, [1, 120], 2, 64, 16, False, seed=31)
    for s, p, col, value in ((0, 0, 3, np.inf), (0, 0, 4, -np.inf), *((1, p, p % 61, (-1) ** p * np.inf) for p in range(0, 120, 3))):
        b.v[b.table[s, p // 16], :, p % 16, col] = value
    b.device(A)
    q64, q = rows_of_q(b, 4)
    o, lse = attend(A, b, q)
    torch.cuda.synchronize()
    o, k = o.double().cpu().numpy(), 0
    for s, (n, kv) in enumerate(zip(b.rows, b.kv)):
        for r in range(n):
            seen = b.v[b.table[s, np.arange(kv - n + r + 1) // 16], :, np.arange(kv - n + r + 1) % 16]          # [keys, heads, d]
            for h in range(4):
                v = seen[:, h // 2]
                up, down = np.isposinf(v).any(0), np.isneginf(v).any(0)
                got = o[k, h]
                assert np.isposinf(got[up & ~down]).all() and np.isneginf(got[down & ~up]).all() and np.isnan(got[up & down]).all()
                assert np.isfinite(got[~up & ~down]).all()
            k += 1
    assert k == len(o) and not torch.isnan(lse).any()


def test_the_largest_numbers_of_the_8_bit_cache():
    """Values up to where 8 bits round to 2^128, which is no number of bf16: those read back as infinities, everything below as it is stored."""
    import torch
    import paper_2504_20490_amd as A
    b = Batch([6], [6], 1, 16, 16, True, seed=28)
    b.device(A)
    top = 2.0 ** 127
    x = np.zeros((6, 1, 16))
    for row, first in enumerate((1.75, 1.7578125, 1.9296875, 1.9375, 1.9921875, 0.875)):
        x[row, 0] = np.array([first] + [1.0, -0.5, 2.0 ** -9] * 5) * top
        x[row, 0, 7] = -first * top
    k = torch.from_numpy(x).to(torch.bfloat16).cuda()
    assert (k.double().cpu().numpy() == x).all()
    A.kv_cache_write(b.cache, b.batch, k, -k)
    back = torch.empty(2, 6, 1, 16, dtype=torch.bfloat16, device="cuda")
    A.kv_cache_read(b.cache, b.batch, back[0], back[1])
    torch.cuda.synchronize()
    codes, byte = paged.quantise(x)
    want = paged.dequantise(codes, byte)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.sign(want) * np.inf, want)
    assert np.isinf(want[3:5, 0, [0, 7]]).all() and np.isinf(want).sum() == 4
    got = back.double().cpu().numpy()
    assert np.array_equal(got[0], want) and np.array_equal(got[1], -want)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [1, 40])
def test_lengths_next_to_two_to_the_31(rows, e4m3):
    """The longest sequence that there can be, one page of 1024 tokens over and over: every row sees whole rounds of it, the last one's keys up to
    its own beside them."""
    import torch
    import paper_2504_20490_amd as A
    size, d, width = 1024, 16, 1 << 21
    kv = (1 << 31) - 2 * size + 5
    b = Batch([size], [size], 1, d, size, e4m3, seed=30, extra_pages=0, extra_width=0)
    b.device(A)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    b.batch = A.KVBatch(i32(0, rows), i32(kv), torch.zeros(1, width, dtype=torch.int32, device="cuda"), rows)
    q64 = bf16(b.rng.standard_normal((rows, 2, d)))
    q64[:, 0] = 0.0                                                                 # (all weights 1: the sums count the keys)
    o, lse = attend(A, b, torch.from_numpy(q64).to(torch.bfloat16).cuda())
    back = torch.empty(2, rows, 1, d, dtype=torch.bfloat16, device="cuda")
    A.kv_cache_read(b.cache, b.batch, back[0], back[1])
    torch.cuda.synchronize()
    k, v = b.k[b.table[0, 0], 0], b.v[b.table[0, 0], 0]
    pos = kv - rows + np.arange(rows)
    assert np.array_equal(back[0, :, 0].double().cpu().numpy(), k[pos % size]) and np.array_equal(back[1, :, 0].double().cpu().numpy(), v[pos % size])
    times = (pos[:, None] + size - np.arange(size)) // size                        # how often a row sees each key
    s = np.einsum("thd,kd->htk", q64, k) / np.sqrt(d)
    top = s.max(-1, keepdims=True)
    w = times * np.exp(s - top)
    total = w.sum(-1, keepdims=True)
    ref, mass = w / total @ v, w / total @ np.abs(v)
    got = o.double().cpu().numpy().transpose(1, 0, 2)
    # A share of at most 2^22 keys is summed up tile by tile (32 keys, or 64): at most 2^16 sums one after the other, rounded by 2^-24 of them each, in O and
    # in the weights; 2^-7 of the mass together.  Weights of 1 are summed up exactly in a share, and in at most 2048 shares to 2^-13.
    assert (np.abs(got - ref) <= BF16_HALF_STEP * np.abs(ref) + (BF16_HALF_STEP + 2.0 ** -7 + 1e-4) * mass).all()
    off = np.abs(lse.double().cpu().numpy() - (top + np.log(total))[..., 0])
    assert (off[0] <= 2.0 ** -13 + 1e-5).all() and (off[1] <= 2.0 ** -8 + LSE_ABS).all()


def test_as_many_rows_as_there_can_be():
    """2^25 tokens through the axes rotation, the write and the read, and as many sequences of one token through the attention."""
    import torch
    import paper_2504_20490_amd as A
    T, d = 1 << 25, 8
    i32 = lambda x: x.to(torch.int32).cuda()
    x = torch.randn(T, 1, d, device="cuda").bfloat16()
    pool = torch.zeros(2, T // 1024, 1, 1024, d, dtype=torch.bfloat16, device="cuda")
    cache = A.KVCache(pool[0], pool[1])
    pages = i32(torch.randperm(T // 1024))[None]
    batch = A.KVBatch(i32(torch.tensor([0, T])), i32(torch.tensor([T])), pages)
    A.kv_cache_write(cache, batch, x, -x)
    back = torch.empty(2, T, 1, d, dtype=torch.bfloat16, device="cuda")
    A.kv_cache_read(cache, batch, back[0], back[1])
    assert torch.equal(back[0], x) and torch.equal(back[1], -x) and torch.equal(pool[0, pages[0].long()].view(T, 1, d), x)
    table = torch.empty(4, d // 2, 2, device="cuda")
    A.rope_table(table, 4, d)
    turned, again = torch.empty_like(x), torch.empty_like(x)
    rope = A.RopeAxes(table, 4, i32(torch.arange(T) % 4))
    A.rope_axes_qk(rope, x, None, turned, None)
    part = A.RopeAxes(table, 4, i32(torch.arange(T - 1000, T) % 4))
    A.rope_axes_qk(part, x[-1000:], None, again[-1000:], None)
    assert torch.equal(turned[-1000:], again[-1000:]) and torch.equal(turned[::4], x[::4])
    # sequence s: one token, in slot 0 of a page of 16 (of 2^21): O is its value
    cache = A.KVCache(pool[0].view(-1, 1, 16, d), pool[1].view(-1, 1, 16, d))
    table = i32(torch.arange(T) % (T // 16))[:, None]
    batch = A.KVBatch(i32(torch.arange(T + 1)), torch.ones(T, dtype=torch.int32, device="cuda"), table, 1)
    o, lse = torch.empty_like(x), torch.empty(1, T, device="cuda")
    A.attn_paged_fwd(cache, batch, x, o, lse, torch.empty(A.attn_paged_workspace_bytes(cache, batch, T, 1), dtype=torch.uint8, device="cuda"))
    first = pool.view(2, -1, 16, d)[:, :, 0]
    assert torch.equal(o[:, 0], first[1][table[:, 0].long()])
    score = (x[:, 0].float() * first[0][table[:, 0].long()].float()).sum(-1) / d ** 0.5
    assert (lse[0] - score).abs().max() <= 1e-4
