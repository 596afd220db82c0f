"""Refusals of the calls around the paged cache (no GPU): nothing here may reach a launch."""
import ctypes

import pytest
import torch

import paper_2504_20490_amd as A
from paper_2504_20490_amd import binding as B

P = 1 << 20            # a pointer that is never followed
BF16, E4M3 = A.CACHE_BF16, A.CACHE_E4M3


def rope(**change):
    a = B._RopeAxesArgs(P, 100, 3, P, 1000, bytes([0, 1, 2, 0] * 16))
    for k, v in change.items():
        setattr(a, k, v)
    return a


def cache(dtype=BF16, d=64, **change):
    row = A.kv_cache_row(d, dtype) or d
    a = B._KVCacheArgs(P, P, P, P, 2 * 16 * row, 2 * 16, 10, 16, 2, d, dtype)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def batch(**change):
    a = B._KVBatchArgs(P, P, P, 4, 8, 12, 3)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def axes(r=None, q=P, k=P, qs=256, ks=128, qo=P, ko=P, T=12, hq=4, hkv=2, d=64, dtype=0, qos=None, kos=None):
    return A.load_library().hspmd_rope_axes_qk(None if r is None else ctypes.byref(r), q, k, qs, ks, qo, ko, qos or qs, kos or ks, T, hq, hkv, d,
                                               dtype, 0, None)


def write(c, b, k=P, v=P, ks=128, r=None, q=None, qo=None, qs=256, hq=4):
    by = lambda x: None if x is None else ctypes.byref(x)
    return A.load_library().hspmd_kv_cache_write(by(c), by(b), k, v, ks, by(r), q, qo, qs, qs, hq, None)


def read(c, b, k=P, v=P, ks=128):
    return A.load_library().hspmd_kv_cache_read(ctypes.byref(c), ctypes.byref(b), k, v, ks, None)


def attend(c, b, q=P, qs=256, hq=4, scale=0.0, o=P, lse=P, ws=P, n=1 << 40):
    return A.load_library().hspmd_attn_paged_fwd(ctypes.byref(c), ctypes.byref(b), q, qs, hq, scale, o, lse, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(r=None), 1), (dict(r=rope(table=None)), 1), (dict(r=rope(table=P + 4)), 1), (dict(r=rope(table_positions=-1)), 1),
    (dict(r=rope(num_axes=0)), 1), (dict(r=rope(num_axes=5)), 1), (dict(r=rope(positions=None)), 1), (dict(r=rope(positions=P + 2)), 1),
    (dict(r=rope(positions_stride=11)), 1), (dict(r=rope(num_axes=2)), 1), (dict(q=None), 1), (dict(qo=None), 1), (dict(k=None), 1), (dict(ko=None), 1),
    (dict(q=P + 8), 1), (dict(k=P + 2), 1), (dict(qs=248), 1), (dict(qs=260), 1), (dict(ks=120), 1), (dict(T=-1), 1), (dict(T=(1 << 25) + 1), 1),
    (dict(qos=264), 1), (dict(kos=136), 1), (dict(hq=0), 1), (dict(hkv=-1), 1), (dict(d=60), 2), (dict(d=136), 2), (dict(d=0), 2), (dict(dtype=2), 2)])
def test_rope_axes_refusals(change, status):
    args = dict(r=rope())
    args.update(change)
    assert axes(**args) == status
    assert A.load_library().hspmd_last_error()


def test_nothing_to_do_is_fine():
    assert axes(rope(), T=0) == 0 and axes(None, q=None, k=None, T=0) == 0
    for b in (batch(total_rows=0), batch(num_seqs=0)):
        assert write(cache(), b, None, None) == 0 and read(cache(), b, None, None) == 0
        assert attend(cache(), b, None, o=None, ws=None, n=0) == 0
        assert A.load_library().hspmd_attn_paged_workspace_bytes(ctypes.byref(cache()), ctypes.byref(b), 4) == 0


CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(k=P + 8), 1), (dict(page_stride=2 * 16 * 64 - 8), 1), (dict(page_stride=2 * 16 * 64 + 4), 1),
          (dict(num_pages=0), 1), (dict(num_pages=-3), 1), (dict(page_size=8), 1), (dict(page_size=2048), 1), (dict(page_size=24), 1),
          (dict(local_kv_heads=0), 1), (dict(head_dim=63), 2), (dict(head_dim=0), 2), (dict(head_dim=136), 2), (dict(dtype=2), 2), (dict(dtype=-1), 2)]
SCALES = [(dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(v_scale=P + 1), 1), (dict(scale_page_stride=28), 1), (dict(scale_page_stride=34), 1),
          (dict(page_stride=2 * 16 * 64 + 8), 1)]
BATCHES = [(dict(cu_rows=None), 1), (dict(kv_lens=None), 1), (dict(page_table=None), 1), (dict(cu_rows=P + 1), 1), (dict(num_seqs=-1), 1), (dict(num_seqs=(1 << 25) + 1), 1),
           (dict(table_width=-1), 1), (dict(total_rows=-1), 1), (dict(total_rows=(1 << 25) + 1), 1), (dict(max_rows=-1), 1)]


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("c,b,status", [(cache(**x), batch(), s) for x, s in CACHES] + [(cache(E4M3, **x), batch(), s) for x, s in SCALES]
                         + [(cache(), batch(**x), s) for x, s in BATCHES])
def test_cache_and_batch_refusals(call, c, b, status):
    assert call(c, b) == status


@pytest.mark.parametrize("call,change,status", [
    (write, dict(k=None), 1), (write, dict(v=None), 1), (write, dict(k=P + 8), 1), (write, dict(ks=120), 1), (write, dict(ks=132), 1),
    (write, dict(q=P), 1), (write, dict(q=P, qo=P), 1), (write, dict(q=P, r=rope()), 1), (write, dict(q=P, qo=P, r=rope(), hq=0), 1),
    (write, dict(q=P, qo=P, r=rope(), qs=128), 1), (write, dict(q=P + 4, qo=P, r=rope()), 1), (write, dict(r=rope(table=None)), 1),
    (write, dict(r=rope(num_axes=2)), 1), (write, dict(r=rope(positions_stride=11)), 1),
    (read, dict(k=None), 1), (read, dict(v=P + 2), 1), (read, dict(ks=64), 1),
    (attend, dict(q=None), 1), (attend, dict(o=None), 1), (attend, dict(ws=None), 1), (attend, dict(q=P + 4), 1), (attend, dict(o=P + 8), 1),
    (attend, dict(ws=P + 8), 1), (attend, dict(lse=P + 2), 1), (attend, dict(qs=248), 1), (attend, dict(hq=3), 1), (attend, dict(hq=0), 1),
    (attend, dict(hq=-2), 1), (attend, dict(scale=float("nan")), 1), (attend, dict(scale=float("inf")), 1), (attend, dict(scale=1e-30), 1),
    (attend, dict(n=16), 3), (attend, dict(n=0), 3)])
def test_call_refusals(call, change, status):
    assert call(cache(), batch(), **change) == status
    assert A.load_library().hspmd_last_error()


def test_null_structs():
    lib = A.load_library()
    assert lib.hspmd_kv_cache_write(None, ctypes.byref(batch()), P, P, 128, None, None, None, 0, 0, 0, None) == 1
    assert lib.hspmd_kv_cache_read(ctypes.byref(cache()), None, P, P, 128, None) == 1
    assert lib.hspmd_attn_paged_workspace_bytes(None, None, 4) == 0


def test_rows_times_heads_are_bounded():
    assert attend(cache(), batch(total_rows=1 << 24)) == 1


def test_cache_row():
    assert [A.kv_cache_row(d, BF16) for d in (8, 104, 128)] == [8, 104, 128]
    assert [A.kv_cache_row(d, E4M3) for d in (8, 40, 104, 128)] == [16, 48, 112, 128]
    assert A.kv_cache_row(100, BF16) == A.kv_cache_row(64, 2) == A.kv_cache_row(136, E4M3) == 0


def test_workspace_grows_with_everything():
    size = lambda hq=4, **c: A.load_library().hspmd_attn_paged_workspace_bytes(ctypes.byref(cache()), ctypes.byref(batch(**c)), hq)
    base = size()
    assert base > 0
    for more in (dict(num_seqs=40), dict(table_width=4000), dict(total_rows=3000), dict(hq=32)):
        assert size(**more) >= base
    assert size(max_rows=0) == size(max_rows=1) == size(max_rows=1000)      # (the hint never changes it)


# ------------------------------------------------------------------------------------------------ the binding's own checks
def tensors(e4m3=False, pages=3, h=2, size=16, d=64):
    k = torch.zeros(pages, h, size, d, dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    return [k, k.clone()] + ([torch.zeros(pages, h, size, dtype=torch.uint8) for _ in range(2)] if e4m3 else [])


def refused(f, *args, **kw):
    with pytest.raises(A.HspmdError) as e:
        f(*args, **kw)
    assert e.value.status in (1, 2)


def test_pool_shapes_and_types():
    A.KVCache(*tensors())
    A.KVCache(*tensors(True))
    A.KVCache(*tensors(True, d=112), head_dim=104)
    both = torch.zeros(3, 2, 2, 16, 64, dtype=torch.bfloat16)
    assert A.KVCache(both[:, 0], both[:, 1])._args.page_stride == 2 * 2 * 16 * 64
    k, v = tensors()
    k8, v8, ks, vs = tensors(True)
    refused(A.KVCache, k.float(), v.float())
    refused(A.KVCache, k, v8)
    refused(A.KVCache, k, v[:, :1])
    refused(A.KVCache, k, v, ks, vs)
    refused(A.KVCache, k8, v8)
    refused(A.KVCache, k8, v8, ks, None)
    refused(A.KVCache, k8, v8, ks.int(), vs)
    refused(A.KVCache, k8, v8, ks[:, :1], vs)
    refused(A.KVCache, k.transpose(1, 2).contiguous().transpose(1, 2), v)
    refused(A.KVCache, both[:, 0], v)                       # two page strides
    refused(A.KVCache, k, v, head_dim=56)
    refused(A.KVCache, k8, v8, ks, vs, head_dim=40)


def test_batch_shapes_and_types():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    A.KVBatch(i(4), i(3), i(3, 7))
    refused(A.KVBatch, i(3), i(3), i(3, 7))
    refused(A.KVBatch, i(4), i(3), i(2, 7))
    refused(A.KVBatch, i(4), i(3), i(21))
    refused(A.KVBatch, i(4).long(), i(3), i(3, 7))
    refused(A.KVBatch, i(4), i(3), i(3, 14)[:, ::2])


def test_tensors_of_the_wrong_shape_type_or_place():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    c, b = A.KVCache(*tensors()), A.KVBatch(i(2), i(1), i(1, 2))
    x = lambda h, d=64, t=torch.bfloat16: torch.zeros(5, h, d, dtype=t)
    table = torch.zeros(10, 32, 2)
    r = A.RopeAxes(table, 10)
    refused(A.kv_cache_write, c, b, x(2), x(2))                           # not on a GPU
    refused(A.kv_cache_read, c, b, x(2), x(2))
    refused(A.kv_cache_write, c, b, x(3), x(3))
    refused(A.kv_cache_write, c, b, x(2, 32), x(2))
    refused(A.kv_cache_write, c, b, x(2), x(2, 64, torch.float16))
    refused(A.kv_cache_write, c, b, x(2), x(4)[:, :2])                     # two strides
    refused(A.kv_cache_write, c, b, x(4)[:, ::2], x(4)[:, ::2])
    refused(A.kv_cache_write, c, b, x(2), x(2), rope=r, q=x(4))
    refused(A.kv_cache_read, c, b, x(2), x(2)[:4])
    refused(A.attn_paged_fwd, c, b, x(4), x(4).transpose(0, 1), None, i(4))
    refused(A.attn_paged_fwd, c, b, x(4), x(4), torch.zeros(5, 4), i(4))
    refused(A.attn_paged_fwd, c, b, x(4, 32), x(4, 32), None, i(4))
    refused(A.rope_axes_qk, r, x(4), x(2), x(4), x(2))
    refused(A.rope_axes_qk, r, x(4), x(2), x(4), None)
    refused(A.rope_axes_qk, r, x(4).half(), None, x(4).half(), None)
    refused(A.RopeAxes, table, 10, torch.zeros(3, 5))
    refused(A.RopeAxes, table.double(), 10)
    refused(A.RopeAxes, table, 10, None, [0, 300])
    refused(A.RopeAxes._check, A.RopeAxes(table, 10, i(5), [0] * 31), 64, 5)
    refused(A.RopeAxes._check, A.RopeAxes(table, 10, i(4)), 64, 5)
    refused(A.RopeAxes._check, A.RopeAxes(table, 11), 64, 5)
    refused(A.RopeAxes._check, A.RopeAxes(table, 10), 40, 5)              # a table of another head_dim
    A.RopeAxes(table, 10, i(5), [0] * 32)._check(64, 5)
