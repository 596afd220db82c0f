"""Linear attention, calls that the documentation allows and that hardly anyone makes: offsets beyond 32 bits, many query heads on one KV head, two host threads,
row offsets that make no sense, gradients that are not wanted, accuracy of what goes out in fp32."""
import threading

import numpy as np
import pytest

from linear_util import Case, check, check_backward, check_forward, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2504_20490_amd as A
    A.load_library()
    return A


def test_rows_beyond_4_gib(A):
    """70000 rows, 32768 elements apart: the last ones start at 4.6e9 bytes."""
    import torch
    T, d, far = 70000, 64, 32768
    wide = torch.zeros(T * far, dtype=torch.bfloat16, device="cuda").view(T, far)
    wide[:, :3 * d] = torch.randn(T, 3 * d, device="cuda")
    q, k, v = (wide[:, i * d:(i + 1) * d].view(T, 1, d) for i in range(3))
    g = -torch.rand(T, 1, device="cuda") * 0.2
    batch = A.LinearBatch(torch.tensor([0, 5, T], dtype=torch.int32, device="cuda"), max_rows=T)
    outs = []
    for x in ((q, k, v), tuple(y.contiguous() for y in (q, k, v))):
        o, final = torch.full((T, 1, d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 1, d, d, device="cuda")
        ws = torch.empty(A.linear_attn_workspace_bytes(batch, T, 1, 1, d, backward=True), dtype=torch.uint8, device="cuda")
        A.linear_attn_fwd(batch, *x, g, o, ws, final=final)
        grads = [torch.empty(T, 1, d, device="cuda") for _ in range(3)]
        dg = torch.empty_like(g)
        A.linear_attn_bwd(batch, *x, g, o, *grads, ws, d_log_decay=dg)
        outs.append([o, final, *grads, dg])
    assert torch.isfinite(outs[0][0].float()).all()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_states_beyond_4_gib(A):
    """Slots of a pool of 70000 states of 64 KB."""
    import torch
    d, slots = 128, [69999, 3, 66000]
    pool = torch.empty(70000, 1, d, d, device="cuda")
    case = Case([1, 1, 1], 2, 1, d, 40, False, True).to_device()
    for i, s in enumerate(slots):
        pool[s] = case.tinitial[i]
    guard = pool[slots[0] - 1].clone()
    where = torch.tensor(slots, dtype=torch.int32, device="cuda")
    o = torch.empty_like(case.tq)
    A.linear_attn_step(A.LinearBatch(initial_slots=where, final_slots=where), case.tq, case.tk, case.tv, case.tg, o, initial=pool, final=pool)
    check_forward(case, o, pool[slots])
    assert torch.equal(torch.nan_to_num(pool[slots[0] - 1]), torch.nan_to_num(guard))
    for i, s in enumerate(slots):
        pool[s] = case.tinitial[i]
    A.linear_attn_fwd(A.LinearBatch(case.tcu, 1, where, where), case.tq, case.tk, case.tv, case.tg, o, None, initial=pool, final=pool)
    check_forward(case, o, pool[slots])


@pytest.mark.parametrize("hq,hkv,d", [(33, 1, 32), (34, 2, 128), (24, 24, 16)])
def test_many_heads(A, hq, hkv, d):
    case = Case([90, 400], hq, hkv, d, 41, False, True).to_device()
    check_forward(case, *case.run_forward(A))
    check_backward(case, case.run_backward(A))


def test_two_host_threads(A):
    import torch
    cases = [Case([700, 33], 2, 2, 64, 42, False, True).to_device(), Case([64, 300, 5], 4, 2, 104, 43, False, True).to_device()]
    want = [(c.run_forward(A), c.run_backward(A)) for c in cases]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    got[i] = (cases[i].run_forward(A), cases[i].run_backward(A))
                stream.synchronize()
        except Exception as e:          # (a thread's exception would be lost)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for (f0, b0), (f1, b1) in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(f0, f1)) and all(torch.equal(b0[n], b1[n]) for n in b0)


@pytest.mark.parametrize("cu", [[0, 500, 100000, 700], [0, -5, 300, 2 ** 31 - 1], [800, 400, 0, 0], [-2 ** 31, 900, 100, 950]])
def test_row_offsets_that_make_no_sense_stay_inside_the_tensors(A, cu):
    """Results are undefined; what lies around the tensors, and the rows that no sequence can reach, are not touched."""
    import torch
    T, d, H = 1000, 64, 2
    q, k, v, do = (torch.randn(T, H, d, device="cuda").bfloat16() for _ in range(4))
    g = -torch.rand(T, H, device="cuda")
    batch = A.LinearBatch(torch.tensor(cu, dtype=torch.int32, device="cuda"))
    guarded = lambda *shape, t=torch.float32: torch.full((shape[0] + 2, *shape[1:]), 7.0, dtype=t, device="cuda")
    o, dq, dk, dv = (guarded(T, H, d, t=torch.bfloat16) for _ in range(4))
    dg, final, first = guarded(T, H), guarded(3, H, d, d), guarded(3, H, d, d)
    need = A.linear_attn_workspace_bytes(batch, T, H, H, d, backward=True)
    ws = torch.full((need + 4096,), 90, dtype=torch.uint8, device="cuda")
    A.linear_attn_fwd(batch, q, k, v, g, o[1:-1], ws[:A.linear_attn_workspace_bytes(batch, T, H, H, d)], final=final[1:-1])
    A.linear_attn_bwd(batch, q, k, v, g, do, dq[1:-1], dk[1:-1], dv[1:-1], ws[:need], d_log_decay=dg[1:-1], d_initial=first[1:-1])
    torch.cuda.synchronize()
    for x in (o, dq, dk, dv, dg, final, first):
        assert (x[0] == 7).all() and (x[-1] == 7).all()
    assert (ws[need:] == 90).all()


def test_without_the_decays_gradient_the_others_are_the_same(A):
    import torch
    for fixed in (False, True):
        case = Case([700, 33], 4, 2, 64, 44, fixed, True).to_device()
        want, got = case.run_backward(A, f32=False), case.run_backward(A, f32=False, decays=False)
        assert all(torch.equal(want[n], got[n]) for n in got)


@pytest.mark.parametrize("hq,hkv,d,fixed", [(4, 4, 128, False), (8, 2, 64, False), (3, 3, 80, True)])
def test_what_goes_out_in_fp32_is_of_fp32(A, hq, hkv, d, fixed):
    """Relative to the result's 2-norm.  Terms have random signs, so errors and results grow with the same root of their number: an error of e per term leaves e of the
    result.  Per term: three roundings at 2^-24 (weight, product, part), the decays' exponents of up to 7 roundings of sums below 2^4 (7 * 2^-20 at worst, their root
    mean square an eighth of that), and chains of 64 + 128 sums, whose roundings at 2^-25 of the running sum add up as sqrt(192) of one: 2^-21.  Decay gradients cancel
    by up to four of these, a fixed decay's, the sum of all rows, by the root of their number more."""
    case = Case([900, 300, 70], hq, hkv, d, 45, fixed, True, rate=0.05).to_device()
    out, want = case.run_backward(A), case.backward()
    _, final = case.run_forward(A)
    out["final"], want["final"] = final, case.forward()[1]
    for name, x in out.items():
        got, ref = host(x), want[name]
        off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        most = 2.0 ** -20 * (4 if name == "dg" else 1) * (np.sqrt(case.T) if name == "dg" and fixed else 1)
        assert off <= most, (name, off, most)


@pytest.mark.parametrize("d,f32", [(64, True), (128, False), (128, True)])
def test_gradients_of_rows_that_a_bad_value_does_not_reach(A, d, f32):
    """From the formulas: dk_j and dv_j hold decays behind row j, q and d_o from it on, v_j and k_j; dq_i holds decays, k and v up to row i."""
    import torch
    case = Case([50, 400, 90], 4, 2, d, 46, False, True).to_device()
    clean = case.run_backward(A, f32=f32)
    bad, rows = 50 + 77, torch.arange(case.T, device="cuda")
    before, behind, inside = rows < bad, rows > bad, (rows >= 50) & (rows < 450)
    everywhere, own = torch.ones_like(before), rows != bad
    # what a bad value in each input leaves as it is: of dq, dk, dv
    for name, value, keeps in (("tg", float("nan"), (before, ~before, ~before)), ("tq", float("inf"), (everywhere, behind, behind)),
                               ("tdo", float("nan"), (own, behind, behind)), ("tk", float("-inf"), (before, everywhere, own)),
                               ("tv", float("nan"), (before, own, everywhere))):
        x = getattr(case, name)
        old = x.clone()
        x[bad] = value
        got = case.run_backward(A, f32=f32)
        x.copy_(old)
        for out, keep in zip(("dq", "dk", "dv"), keeps):
            assert torch.equal(got[out][keep | ~inside], clean[out][keep | ~inside]), (name, out)
        assert torch.equal(got["d_initial"][[0, 2]], clean["d_initial"][[0, 2]]), name


@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2)])
@pytest.mark.parametrize("d,f32", [(128, True), (128, False), (64, True), (104, True)])
def test_infinite_sources_keep_the_sign_of_their_weights(A, hq, hkv, d, f32):
    """One sequence of one group of 64 rows, an infinite value in one row of a tensor that sources are taken from: the formulas' signed infinities."""
    import torch
    case = Case([64], hq, hkv, d, 47, False, False).to_device()
    q, k, v, do = (host(getattr(case, n)) for n in ("tq", "tk", "tv", "tdo"))
    group = hq // hkv
    row, col, head = 45, 3, 1
    def column(name, out):
        x = getattr(case, name)
        old = x.clone()
        x[row, head, col] = float("inf")
        if out == "o":
            got = host(case.run_forward(A, final=False)[0])
        else:
            got = host(case.run_backward(A, f32=f32)[out])
        x.copy_(old)
        return got[:, :, col]
    def expect(got, sign, sees):          # (weights whose sign a rounding of 128 terms could turn are let be)
        clear = sees & (abs(sign) > 2.0 ** -10)
        assert clear.any() and (np.isposinf(got[clear]) == (sign[clear] > 0)).all() and np.isinf(got[clear]).all()
        assert np.isfinite(got[~sees]).all()
    rows = np.arange(64)
    for h in range(head * group, (head + 1) * group):      # o_i[col] = <q_i, k_row> v_row[col], dq_i[col] = <dO_i, v_row> k_row[col]
        expect(column("tv", "o")[:, h], q[:, h] @ k[row, head], rows >= row)
        expect(column("tk", "dq")[:, h], do[:, h] @ v[row, head], rows >= row)
    head = 1                                               # (a query head, whose KV head is head // group)
    expect(column("tq", "dk")[:, head // group], v[:, head // group] @ do[row, head], rows <= row)
    expect(column("tdo", "dv")[:, head // group], k[:, head // group] @ q[row, head], rows <= row)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("hq,hkv,d,fixed,states", [(2, 2, 128, False, False), (2, 2, 104, True, True), (8, 2, 128, False, True), (3, 1, 80, True, False),
                                                   (2, 2, 40, False, True), (6, 2, 24, True, False)])
def test_gradients_without_the_decays(A, hq, hkv, d, fixed, states, f32):
    import torch
    case = Case([700, 33, 0, 129], hq, hkv, d, 48, fixed, states).to_device()
    want, got = case.run_backward(A, f32=f32), case.run_backward(A, f32=f32, decays=False)
    assert "dg" not in got
    assert all(torch.equal(want[n], got[n]) for n in got)
    check_backward(case, want, f32)


def test_the_most_rows(A):
    """2^25 rows of one head; the last 3000, from a decay that forgets all on, are as they are alone."""
    import torch
    T, n, d = 1 << 25, 3000, 8
    case = Case([n], 1, 1, d, 49, False, False)
    case.g[0] = -np.inf
    case.to_device()
    q, k, v, do = (torch.zeros(T, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(4))
    g = torch.full((T, 1), -0.01, device="cuda")
    for whole, part in ((q, case.tq), (k, case.tk), (v, case.tv), (do, case.tdo), (g, case.tg)):
        if whole is not g:
            whole[:T - n] = 1.0
        whole[T - n:] = part
    batch = A.LinearBatch(torch.tensor([0, 7, T], dtype=torch.int32, device="cuda"))
    ws = torch.empty(A.linear_attn_workspace_bytes(batch, T, 1, 1, d, backward=True), dtype=torch.uint8, device="cuda")
    out = {"o": torch.empty_like(q), "dg": torch.empty_like(g), **{x: torch.empty(T, 1, d, device="cuda") for x in ("dq", "dk", "dv")}}
    A.linear_attn_fwd(batch, q, k, v, g, out["o"], ws)
    A.linear_attn_bwd(batch, q, k, v, g, do, out["dq"], out["dk"], out["dv"], ws, d_log_decay=out["dg"])
    # (a constant's steady state: 8 * 1 / (1 - e^-0.01) / sqrt(8); sums of 64 decays and states in fp32: as many roundings as rows are remembered)
    assert abs(out["o"][T - n - 1].float().mean().item() / (np.sqrt(8) / (1 - np.exp(-0.01))) - 1) < 2.0 ** -8
    check_forward(case, out["o"][T - n:], None)
    check_backward(case, {x: out[x][T - n:] for x in ("dq", "dk", "dv", "dg")})


@pytest.mark.parametrize("d", [8, 72])
def test_the_most_sequences(A, d):
    """2^22 sequences of one row: o = s <q, k> v and its gradients, row by row."""
    import torch
    T = 1 << 22
    q, k, v, do = (torch.randint(-2, 3, (T, 1, d), device="cuda").bfloat16() for _ in range(4))      # (sums of small whole numbers: exact in fp32)
    g = torch.full((T, 1), -0.5, device="cuda")
    batch = A.LinearBatch(torch.arange(T + 1, dtype=torch.int32, device="cuda"))
    ws = torch.empty(A.linear_attn_workspace_bytes(batch, T, 1, 1, d, backward=True), dtype=torch.uint8, device="cuda")
    o, step = torch.empty_like(q), torch.empty_like(q)
    A.linear_attn_fwd(batch, q, k, v, g, o, ws, scale=0.5)
    A.linear_attn_step(A.LinearBatch(), q, k, v, g, step, scale=0.5)
    want = 0.5 * (q.float() * k.float()).sum(-1, keepdim=True) * v.float()
    assert torch.equal(o, want.bfloat16()) and torch.equal(step, o)
    dq, dk, dv = (torch.empty(T, 1, d, device="cuda") for _ in range(3))
    dg = torch.empty_like(g)
    A.linear_attn_bwd(batch, q, k, v, g, do, dq, dk, dv, ws, d_log_decay=dg, scale=0.5)
    pair = 0.5 * (do.float() * v.float()).sum(-1, keepdim=True)
    assert torch.equal(dq, pair * k.float()) and torch.equal(dk, pair * q.float())
    assert torch.equal(dv, 0.5 * (q.float() * k.float()).sum(-1, keepdim=True) * do.float())
    assert (dg == 0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rate", [0.5, 2.0, 20.0, "in half of the rows all", "in half of the rows e^-80"])
def test_strong_decays_keep_fp32(A, rate, d):
    """As above: a weight's exponent is off by the roundings of sums of 64 rests of at most a half, 2^-20 each at worst."""
    case = Case([900, 300, 70], 2, 2, d, 50, False, True)
    rng = np.random.default_rng(51)
    shape = case.g.shape
    strong = {"in half of the rows all": -np.inf, "in half of the rows e^-80": -80.0}
    g = np.where(rng.random(shape) < 0.5, strong[rate], -0.05 * rng.random(shape)) if rate in strong else -rate * rng.exponential(1.0, shape)
    case.g = g.astype(np.float32).astype(np.float64)
    case.to_device()
    out, want = case.run_backward(A), case.backward()
    out["final"], want["final"] = case.run_forward(A)[1], case.forward()[1]
    for name, x in out.items():
        off = np.linalg.norm(host(x) - want[name]) / np.linalg.norm(want[name])
        assert off <= 2.0 ** -20 * (4 if name == "dg" else 1), (name, off)
