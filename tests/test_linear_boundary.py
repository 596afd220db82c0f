"""Refusals of the linear attention's calls (no GPU): nothing here may reach a launch."""
import ctypes

import pytest
import torch

import paper_2504_20490_amd as A
from paper_2504_20490_amd import binding as B

P = 1 << 20            # a pointer that is never followed
by = lambda x: None if x is None else ctypes.byref(x)


def batch(**change):
    a = B._LinearBatchArgs(P, P, P, 4, 12, 5, 4, 2, 64)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def states(**change):
    a = B._LinearStatesArgs(P, 2 * 64 * 64, 9)
    for k, v in change.items():
        setattr(a, k, v)
    return a


def fwd(b, q=P, k=P, v=P, g=P, qs=256, ks=128, gs=2, scale=0.0, initial=None, final=None, o=P, ws=P, n=1 << 40):
    return A.load_library().hspmd_linear_attn_fwd(by(b), q, k, v, g, qs, ks, gs, scale, by(initial), by(final), o, ws, n, None)


def bwd(b, q=P, k=P, v=P, g=P, do=P, qs=256, ks=128, gs=2, scale=0.0, initial=None, d_final=None, dq=P, dk=P, dv=P, dtype=0, dg=P, d_initial=None, ws=P,
        n=1 << 40):
    return A.load_library().hspmd_linear_attn_bwd(by(b), q, k, v, g, do, qs, ks, gs, scale, by(initial), d_final, dq, dk, dv, dtype, dg, d_initial, ws, n,
                                                  None)


def step(b, q=P, k=P, v=P, g=P, qs=256, ks=128, gs=2, scale=0.0, initial=None, final=None, o=P):
    b = None if b is None else b
    if b is not None and b.total_rows == 12 and b.num_seqs == 4:
        b.num_seqs = 12
    return A.load_library().hspmd_linear_attn_step(by(b), q, k, v, g, qs, ks, gs, scale, by(initial), by(final), o, None)


BATCHES = [(dict(num_seqs=-1), 1), (dict(total_rows=-1), 1), (dict(total_rows=(1 << 25) + 1), 1), (dict(max_rows=-1), 1), (dict(local_q_heads=0), 1),
           (dict(local_q_heads=3), 1), (dict(local_kv_heads=0), 1), (dict(local_kv_heads=1 << 17, local_q_heads=1 << 17), 1), (dict(head_dim=60), 2),
           (dict(head_dim=0), 2), (dict(head_dim=136), 2), (dict(total_rows=1 << 24), 1), (dict(num_seqs=(1 << 21) + 1, total_rows=(1 << 21) + 1), 1)]
ROWS = [(dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(g=None), 1), (dict(q=P + 8), 1), (dict(k=P + 2), 1), (dict(v=P + 4), 1), (dict(g=P + 2), 1),
        (dict(qs=248), 1), (dict(qs=260), 1), (dict(ks=120), 1), (dict(qs=(1 << 24) + 8), 1), (dict(ks=1 << 40), 1), (dict(gs=1), 1), (dict(gs=-2), 1),
        (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(scale=1e-30), 1)]
POOLS = [(dict(data=None), 1), (dict(data=P + 4), 1), (dict(num_slots=0), 1), (dict(num_slots=-2), 1), (dict(slot_stride=2 * 64 * 64 - 4), 1),
         (dict(slot_stride=2 * 64 * 64 + 2), 1)]


@pytest.mark.parametrize("call", [fwd, bwd, step])
@pytest.mark.parametrize("change,status", BATCHES)
def test_batches(call, change, status):
    assert call(batch(**change)) == status
    assert A.load_library().hspmd_last_error()


@pytest.mark.parametrize("call", [fwd, bwd, step])
@pytest.mark.parametrize("change,status", ROWS)
def test_rows(call, change, status):
    assert call(batch(), **change) == status


@pytest.mark.parametrize("call,which", [(fwd, "initial"), (fwd, "final"), (bwd, "initial"), (step, "initial"), (step, "final")])
@pytest.mark.parametrize("change,status", POOLS)
def test_pools(call, which, change, status):
    assert call(batch(), **{which: states(**change)}) == status


def test_a_pool_without_slots_has_to_hold_all_sequences():
    assert fwd(batch(initial_slots=None), initial=states(num_slots=3)) == 1
    assert fwd(batch(final_slots=None), final=states(num_slots=3)) == 1
    assert fwd(batch(initial_slots=P + 2), initial=states()) == 1


@pytest.mark.parametrize("call,change,status", [
    (fwd, dict(o=None), 1), (fwd, dict(o=P + 8), 1), (bwd, dict(do=None), 1), (bwd, dict(do=P + 8), 1), (bwd, dict(dq=None), 1), (bwd, dict(dk=P + 4), 1),
    (bwd, dict(dv=None), 1), (bwd, dict(dtype=2), 2), (bwd, dict(dtype=-1), 2), (bwd, dict(dg=P + 2), 1), (bwd, dict(d_final=P + 8), 1),
    (bwd, dict(d_initial=P + 4), 1), (bwd, dict(ws=None), 1), (bwd, dict(ws=P + 8), 1), (bwd, dict(n=100), 3), (step, dict(o=None), 1), (step, dict(o=P + 4), 1)])
def test_calls(call, change, status):
    assert call(batch(), **change) == status
    assert A.load_library().hspmd_last_error()


def test_long_sequences_take_a_workspace():
    long = dict(total_rows=100000, max_rows=90000, local_q_heads=2, local_kv_heads=2)
    assert fwd(batch(**long), qs=128, ws=None) == 1 and fwd(batch(**long), qs=128, n=1000) == 3
    size = lambda backward, **c: A.load_library().hspmd_linear_attn_workspace_bytes(ctypes.byref(batch(**c)), backward)
    assert size(0, **long) > 0 and size(1, **long) > 2 * size(0, **long)
    assert size(0) == 0 and size(1) > 0
    assert size(0, head_dim=60) == size(1, num_seqs=0) == 0


def test_cu_rows():
    for call in (fwd, bwd):
        assert call(batch(cu_rows=None)) == 1 and call(batch(cu_rows=P + 2)) == 1
    assert step(batch(total_rows=11)) == 1                   # a row per sequence


def test_null_batch():
    assert fwd(None) == 1 and bwd(None) == 1 and step(None) == 1
    assert A.load_library().hspmd_linear_attn_workspace_bytes(None, 0) == 0


def test_nothing_to_do_is_fine():
    none = dict(q=None, k=None, v=None, g=None)
    assert fwd(batch(num_seqs=0), **none, o=None, ws=None, n=0) == 0
    assert fwd(batch(total_rows=0), **none, o=None, ws=None, n=0) == 0
    assert bwd(batch(num_seqs=0), **none, do=None, dq=None, dk=None, dv=None, dg=None, ws=None, n=0) == 0
    assert step(batch(num_seqs=0, total_rows=0), **none, o=None) == 0


# ------------------------------------------------------------------------------------------------ the binding's own checks
def refused(f, *args, **kw):
    with pytest.raises(A.HspmdError) as e:
        f(*args, **kw)
    assert e.value.status in (1, 2)


def test_batch_shapes_and_types():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    assert A.LinearBatch(i(4), 7, i(3), i(3)).num_seqs == 3
    assert A.LinearBatch().num_seqs is None and A.LinearBatch(initial_slots=i(5)).num_seqs == 5
    refused(A.LinearBatch, i(4).long())
    refused(A.LinearBatch, i(0))
    refused(A.LinearBatch, i(2, 2))
    refused(A.LinearBatch, i(8)[::2])
    refused(A.LinearBatch, i(4), 0, i(4))
    refused(A.LinearBatch, i(4), 0, None, i(2))
    refused(A.LinearBatch, i(4), 1 << 40)
    refused(A.LinearBatch, None, 0, i(3), i(4))


def test_tensors_of_the_wrong_shape_type_or_place():
    b = A.LinearBatch(torch.zeros(2, dtype=torch.int32))
    x = lambda h, d=64, t=torch.bfloat16, T=5: torch.zeros(T, h, d, dtype=t)
    g, pool = torch.zeros(5, 2), torch.zeros(3, 2, 64, 64)
    good = dict(q=x(4), k=x(2), v=x(2), log_decay=g, o=x(4), workspace=None)
    call = lambda **c: A.linear_attn_fwd(b, **{**good, **c})
    refused(call)                                                            # not on a GPU
    for c in (dict(q=x(4)[0]), dict(q=x(4, t=torch.float16)), dict(q=x(4, T=4)), dict(k=x(2, 32)), dict(v=x(3)), dict(v=x(4)[:, :2]), dict(k=x(4)[:, ::2]),
              dict(log_decay=g.double()), dict(log_decay=g[:, :1]), dict(log_decay=torch.zeros(5)), dict(log_decay=torch.zeros(5, 4)[:, ::2]),
              dict(o=x(4).float()), dict(o=x(4).transpose(0, 1)), dict(o=x(8)[:, :4]), dict(initial=pool.double()), dict(initial=pool[:, :1]),
              dict(final=pool.transpose(2, 3)), dict(final=pool[0]), dict(workspace=torch.zeros(8, 2)[:, 0])):
        refused(call, **c)
    refused(A.linear_attn_fwd, A.LinearBatch(), **good)                      # no cu_rows
    back = dict(q=x(4), k=x(2), v=x(2), log_decay=g, d_o=x(4), dq=x(4), dk=x(2), dv=x(2), workspace=None)
    call = lambda **c: A.linear_attn_bwd(b, **{**back, **c})
    for c in (dict(dq=x(4).half()), dict(dk=x(2).float()), dict(d_o=x(2)), dict(d_log_decay=g[0]), dict(log_decay=g[0], d_log_decay=g), dict(d_final=pool),
              dict(d_initial=pool[:1].double()), dict(d_initial=pool[:1].transpose(2, 3))):
        refused(call, **c)
    refused(A.linear_attn_bwd, A.LinearBatch(), **back)
    del good["workspace"]
    refused(A.linear_attn_step, A.LinearBatch(), **good)
    refused(A.linear_attn_step, A.LinearBatch(), **{**good, "o": x(4, T=4)})


def test_workspace_refusals():
    b = A.LinearBatch(torch.zeros(2, dtype=torch.int32))
    assert A.linear_attn_workspace_bytes(b, 10, 4, 2, 64) == 0 < A.linear_attn_workspace_bytes(b, 10, 4, 2, 64, backward=True)
    refused(A.linear_attn_workspace_bytes, b, 10, 3, 2, 64)
    refused(A.linear_attn_workspace_bytes, b, 10, 4, 2, 60)
    refused(A.linear_attn_workspace_bytes, b, 1 << 40, 4, 2, 64)
