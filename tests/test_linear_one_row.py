"""Linear attention: decays that are fixed, given as a view with one row per token, where a pack shrinks to one row or none.  Such a view does not tell that its rows are
one: then the shape that is wanted of d_log_decay does."""
import pytest
import torch

import paper_2504_20490_amd as A

H, D = 2, 64


def tensors(T, device, hq=4):
    x = lambda h, t=torch.bfloat16: torch.randn(T, h, D, device=device).to(t)
    return dict(q=x(hq), k=x(H), v=x(H), d_o=x(hq), dq=x(hq, torch.float32), dk=x(H, torch.float32), dv=x(H, torch.float32))


@pytest.mark.parametrize("T,shape,fine", [(0, (H,), True), (0, (0, H), True), (1, (H,), True), (1, (1, H), True), (2, (H,), True), (2, (2, H), False),
                                          (1, (H + 1,), False), (1, (2, H), False), (1, (H, 1), False), (0, (1, H), False)])
def test_what_is_taken(T, shape, fine):
    """On the CPU every call is refused in the end: for its device where the shapes are right."""
    batch = A.LinearBatch(torch.zeros(2, dtype=torch.int32))
    decays = torch.full((H,), -0.1).expand(T, H)
    with pytest.raises(A.HspmdError) as e:
        A.linear_attn_bwd(batch, log_decay=decays, workspace=None, d_log_decay=torch.zeros(shape), **tensors(T, "cpu"))
    assert ("d_log_decay" in str(e.value)) != fine


def test_decays_by_token_are_not_summed():
    batch = A.LinearBatch(torch.zeros(2, dtype=torch.int32))
    with pytest.raises(A.HspmdError) as e:
        A.linear_attn_bwd(batch, log_decay=torch.zeros(3, H), workspace=None, d_log_decay=torch.zeros(H), **tensors(3, "cpu"))
    assert "d_log_decay" in str(e.value)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [0, 1, 2])
def test_one_call_for_packs_of_any_length(T):
    torch.manual_seed(T)
    t = tensors(T, "cuda")
    flat = torch.tensor([-0.3, -0.01], device="cuda")
    batch = A.LinearBatch(torch.tensor([0, T], dtype=torch.int32, device="cuda"), max_rows=T)
    pool, d_final = torch.randn(2, 1, H, D, D, device="cuda")
    ws = torch.empty(A.linear_attn_workspace_bytes(batch, T, 4, H, D, backward=True), dtype=torch.uint8, device="cuda")
    out = []
    for decays in (flat, flat.expand(T, H)):
        for name in ("dq", "dk", "dv"):
            t[name].fill_(float("nan"))
        dg = torch.full((H,), float("nan"), device="cuda")
        A.linear_attn_bwd(batch, log_decay=decays, workspace=ws, initial=pool, d_final=d_final, d_log_decay=dg, **t)
        out.append([t[name].clone() for name in ("dq", "dk", "dv")] + [dg])
    assert all(torch.equal(a, b) for a, b in zip(*out)) and torch.isfinite(out[0][3]).all()
    if T == 0:
        assert (out[0][3] == 0).all()
    if T == 1:        # by token: the same value
        by_token = torch.full((1, H), float("nan"), device="cuda")
        A.linear_attn_bwd(batch, log_decay=flat.expand(1, H), workspace=ws, initial=pool, d_final=d_final, d_log_decay=by_token, **t)
        assert torch.equal(by_token[0], out[0][3]) and (by_token != 0).all()
