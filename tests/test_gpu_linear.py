"""Linear attention with a decay for each head through the C ABI against the fp64 oracle: chunked forward and backward, single steps."""
import numpy as np
import pytest

from linear_util import BF16_HALF_STEP, TERMS, Case, check, check_backward, check_forward, host
from oracle import linear

pytestmark = pytest.mark.gpu

SHAPES = [
    # lengths, query heads, KV heads, head_dim, fixed decays, states
    ([1], 1, 1, 8, False, False), ([0, 1, 2], 2, 2, 64, False, True), ([63, 64, 65], 3, 3, 128, False, True), ([17, 64, 111], 2, 2, 64, True, False),
    ([300, 0, 129, 1, 700], 4, 2, 104, False, True), ([128], 8, 1, 40, True, True), ([1500, 3, 800], 2, 1, 72, False, True),
    ([257], 5, 5, 24, False, False), ([256, 256], 6, 2, 32, True, True), ([2049], 1, 1, 128, False, False), ([640, 70], 4, 4, 96, True, True),
    ([0, 0, 5, 0], 3, 1, 80, False, True), ([1031], 9, 3, 16, False, True), ([513, 2, 300], 10, 2, 128, True, False),
]


@pytest.fixture(scope="module")
def A():
    import paper_2504_20490_amd as A
    A.load_library()
    return A


def slots_of(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("lengths,hq,hkv,d,fixed,states", SHAPES)
def test_forward(A, lengths, hq, hkv, d, fixed, states):
    case = Case(lengths, hq, hkv, d, 1, fixed, states).to_device()
    check_forward(case, *case.run_forward(A))


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("lengths,hq,hkv,d,fixed,states", SHAPES)
def test_backward(A, lengths, hq, hkv, d, fixed, states, f32):
    case = Case(lengths, hq, hkv, d, 2, fixed, states).to_device()
    check_backward(case, case.run_backward(A, f32=f32), f32)


@pytest.mark.parametrize("rate", [0.0, 1e-4, 3.0, 40.0])
def test_decays_from_none_to_all(A, rate):
    case = Case([200, 70], 2, 2, 64, 3, False, True, rate=rate).to_device()
    check_forward(case, *case.run_forward(A))
    check_backward(case, case.run_backward(A))


def test_a_decay_of_minus_infinity_forgets_all(A):
    case = Case([200, 600], 2, 2, 64, 4, False, True)
    for t in (0, 63, 64, 100, 101, 130, 500):
        case.g[t, 0] = -np.inf
    case.g[300:364] = -np.inf
    case.g[20, 1] = -1e30
    case.to_device()
    with np.errstate(invalid="ignore"):
        check_forward(case, *case.run_forward(A))
        out = case.run_backward(A)
        check_backward(case, out)


@pytest.mark.parametrize("fixed", [False, True])
def test_views_into_one_projection_and_wide_decays(A, fixed):
    case = Case([90, 310], 4, 2, 72, 5, fixed, True, extra_rows=7).to_device(fused=True, decay_stride=None if fixed else 5)
    check_forward(case, *case.run_forward(A))
    check_backward(case, case.run_backward(A, f32=False), False)


def test_a_broadcast_view_of_the_decays_is_a_fixed_decay(A):
    import torch
    case = Case([90, 310], 4, 2, 72, 6, True, True).to_device()
    want = case.run_backward(A)
    flat, case.tg = case.tg, case.tg.expand(case.rows, case.hkv)
    got = case.run_backward(A)
    for name in want:
        assert torch.equal(want[name], got[name]), name
    case.tg = flat.expand(case.rows, case.hkv).contiguous()
    case.fixed = False                                     # as one decay per token: the gradients of the tokens add up to it
    per_token = case.run_backward(A)["dg"]
    case.fixed = True
    check(host(per_token).sum(0), host(want["dg"]), np.abs(host(per_token)).sum(0), what="sum of the tokens' gradients")


@pytest.mark.parametrize("hint", [0, 1, 300, 100000])
def test_the_most_rows_is_a_hint_only(A, hint):
    case = Case([700, 5, 1300], 2, 2, 64, 7, False, True).to_device()
    check_forward(case, *case.run_forward(A, case.batch(A, hint)))
    check_backward(case, case.run_backward(A, case.batch(A, hint)))


@pytest.mark.parametrize("lengths", [[40, 3], [1000, 40, 3]])
def test_states_go_where_the_slots_say(A, lengths):
    """Named slots, no state (negative), slots outside the pool, in place, and the other slots left alone."""
    import torch
    n = len(lengths)
    case = Case(lengths, 4, 2, 40, 8, False, True).to_device()
    stride = case.hkv * case.d * case.d + 12
    pool = torch.empty((n + 4) * stride, device="cuda").normal_().as_strided((n + 4, case.hkv, case.d, case.d), (stride, case.d ** 2, case.d, 1))
    before = pool.clone()
    where = list(range(n + 1, 1, -1))
    for i, s in enumerate(where):
        pool[s] = case.tinitial[i]
    o = torch.empty_like(case.tq)
    batch = case.batch(A, initial_slots=slots_of(where), final_slots=slots_of(where))
    A.linear_attn_fwd(batch, case.tq, case.tk, case.tv, case.tg, o, case.workspace(A, batch, False), initial=pool, final=pool)
    check_forward(case, o, pool[where])
    rest = [i for i in range(n + 4) if i not in where]
    assert torch.equal(pool[rest], before[rest])
    # the last sequence: no initial state, no place for the final one; the first: slots that do not exist
    initial = slots_of([n + 4] + where[1:-1] + [-1])
    final = slots_of([n + 4] + where[1:-1] + [-7])
    for i, s in enumerate(where):
        pool[s] = case.tinitial[i]
    before = pool.clone()
    batch = case.batch(A, initial_slots=initial, final_slots=final)
    A.linear_attn_fwd(batch, case.tq, case.tk, case.tv, case.tg, o, case.workspace(A, batch, False), initial=pool, final=pool)
    assert torch.isnan(o[:lengths[0]].float()).all()
    kept = case.initial.copy()
    case.initial[-1] = 0.0
    want, want_final = case.forward()
    most, _ = case.forward(absolute=True)
    check(host(o)[lengths[0]:], want[lengths[0]:], most[lengths[0]:], BF16_HALF_STEP, "o")
    changed = where[1:-1]
    same = [i for i in range(n + 4) if i not in changed]
    assert torch.equal(pool[same], before[same])
    case.initial = kept


def test_sequences_may_start_from_one_state(A):
    """A shared prefix: one slot for all; the gradients come by sequence."""
    import torch
    case = Case([70, 130, 300], 2, 2, 64, 9, False, True)
    case.initial[:] = case.initial[:1]
    case.to_device()
    batch = case.batch(A, initial_slots=slots_of([1, 1, 1]))
    pool = torch.stack([torch.full_like(case.tinitial[0], float("nan")), case.tinitial[0]])
    case.tinitial = pool
    check_forward(case, *case.run_forward(A, batch))
    check_backward(case, case.run_backward(A, batch))


@pytest.mark.parametrize("d", [64, 128])
def test_later_rows_change_nothing_whatever_they_hold(A, d):
    """Infinities and NaN in a row: the rows before it in its sequence, and the other sequences, keep every bit."""
    import torch
    case = Case([50, 400, 90], 4, 2, d, 10, False, True).to_device()
    clean, clean_final = case.run_forward(A)
    grads = case.run_backward(A)
    bad = 50 + 77                                          # in the second sequence's second group of 64 rows
    for name, value in (("tv", float("inf")), ("tv", float("nan")), ("tk", float("inf")), ("tq", float("nan")), ("tg", float("nan"))):
        x = getattr(case, name)
        old = x.clone()
        x[bad, :1] = value
        if name != "tg":
            x[bad + 2, :1, 3] = -value
        o, final = case.run_forward(A)
        x.copy_(old)
        rows = [i for i in range(case.T) if i < bad or i >= 450]
        assert torch.equal(o[rows], clean[rows]), name
        assert torch.equal(final[[0, 2]], clean_final[[0, 2]]), name
        assert torch.equal(o[:, 2:], clean[:, 2:]) or name in ("tg",) and torch.equal(o[:, 2:], clean[:, 2:]), name   # (the other KV head)
        if name != "tq":
            assert not torch.isfinite(o[bad, :2].float()).all()
    # backwards it is the rows behind that are not to change, and those of the other sequences
    old = case.tdo.clone()
    case.tdo[bad, :2] = float("nan")
    got = case.run_backward(A)
    case.tdo.copy_(old)
    behind = [i for i in range(case.T) if i < 50 or i > bad]
    for name in ("dk", "dv", "dq"):
        assert torch.equal(got[name][behind], grads[name][behind]), name
    assert torch.equal(got["d_initial"][[0, 2]], grads["d_initial"][[0, 2]])
    old = case.tv.clone()
    case.tv[bad, :1] = float("inf")
    got = case.run_backward(A)
    case.tv.copy_(old)
    before = [i for i in range(case.T) if i < bad or i >= 450]
    assert torch.equal(got["dq"][before], grads["dq"][before])


def test_an_infinite_value_in_a_row_stays_in_its_columns(A):
    import torch
    case = Case([100], 1, 1, 64, 11).to_device()
    clean, _ = case.run_forward(A)
    case.tv[30, 0, 5] = float("inf")
    o, _ = case.run_forward(A)
    other = [c for c in range(64) if c != 5]
    assert torch.equal(o[:, :, other], clean[:, :, other]) and torch.equal(o[:30], clean[:30])
    assert not torch.isfinite(o[30:, :, 5].float()).any()


def test_gradients_are_adjoint_to_the_forward(A):
    """o is linear in q, and in k, and in v: <o(x), do> = <d x, x> for any x put in the place of one of them."""
    case = Case([300, 45], 4, 2, 64, 12).to_device()
    grads = case.run_backward(A)
    rng = np.random.default_rng(1)
    do = case.do
    for name, grad in (("tq", "dq"), ("tk", "dk"), ("tv", "dv")):
        import torch
        old = getattr(case, name)
        x = torch.from_numpy(rng.standard_normal(tuple(old.shape)).astype(np.float32)).bfloat16().cuda()
        setattr(case, name, x)
        o, _ = case.run_forward(A, final=False)
        setattr(case, name, old)
        left, right = (host(o) * do).sum(), (host(grads[grad]) * host(x)).sum()
        # o is rounded to bf16, half a step of each term, signs as they come
        room = 4 * BF16_HALF_STEP * np.sqrt(((host(o) * do) ** 2).sum()) + TERMS * (np.abs(host(grads[grad])) * np.abs(host(x))).sum()
        assert abs(left - right) <= room, (name, left, right, room)


def test_the_decays_gradient_is_a_difference(A):
    """Central differences of <final state, R>, which is fp32."""
    import torch
    case = Case([100, 150], 2, 2, 32, 13, False, True)
    case.do[:] = 0.0
    case.to_device()
    grad = host(case.run_backward(A)["dg"])
    R, most = case.d_final, case.forward(absolute=True)[1]
    h = 0.125
    for t, c in ((0, 0), (63, 1), (64, 0), (99, 1), (100, 0), (180, 1), (249, 0)):
        ends = []
        old = case.tg.clone()
        for sign in (1, -1):
            case.tg[t, c] = old[t, c] + sign * h
            _, final = case.run_forward(A)
            ends.append((host(final) * R).sum())
        case.tg.copy_(old)
        # the state depends on one decay as a + b e^g: the difference is exactly 2 b e^g sinh h.  Each end is off by TERMS of its terms
        b = 0 if t < 100 else 1
        room = TERMS * (most[b, c] * np.abs(R[b, c])).sum() / np.sinh(h) * np.exp(h)
        assert abs((ends[0] - ends[1]) / (2 * np.sinh(h)) - grad[t, c]) <= room + TERMS * abs(grad[t, c]), (t, c)


# ---------------------------------------------------------------------------------------------------------------- steps
def step_case(n, hq, hkv, d, seed, fixed=False):
    return Case([1] * n, hq, hkv, d, seed, fixed, True)


@pytest.mark.parametrize("n,hq,hkv,d,fixed", [(1, 1, 1, 8, False), (1, 5, 5, 128, False), (3, 6, 2, 104, True), (40, 4, 4, 64, False), (2, 18, 2, 72, False),
                                              (300, 4, 2, 24, True), (7, 9, 1, 120, False), (130, 4, 4, 128, True), (5, 3, 3, 40, False), (600, 1, 1, 96, False)])
def test_step(A, n, hq, hkv, d, fixed):
    import torch
    case = step_case(n, hq, hkv, d, 20, fixed).to_device(fused=True)
    o = torch.full((n, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    final = torch.full_like(case.tinitial, float("nan"))
    A.linear_attn_step(A.LinearBatch(), case.tq, case.tk, case.tv, case.tg, o, initial=case.tinitial, final=final)
    check_forward(case, o, final)
    # fp32 throughout: a product and a sum, the decay's exponent and exponential
    want, most = case.forward()[1], case.forward(absolute=True)[1]
    assert (np.abs(host(final) - want) <= 2.0 ** -22 * most).all()


def test_steps_in_place_without_states_and_with_slots_that_do_not_exist(A):
    import torch
    case = step_case(5, 4, 2, 64, 21).to_device()
    pool = torch.randn(9, 2, 64, 64, device="cuda")
    where = [7, 3, -1, 9, 0]
    for i in (0, 1, 4):
        pool[where[i]] = case.tinitial[i]
    before = pool.clone()
    o = torch.empty_like(case.tq)
    batch = A.LinearBatch(initial_slots=slots_of(where), final_slots=slots_of(where))
    A.linear_attn_step(batch, case.tq, case.tk, case.tv, case.tg, o, initial=pool, final=pool)
    assert torch.isnan(o[3].float()).all()
    case.initial[2] = 0.0
    want, want_final = case.forward()
    most, most_final = case.forward(absolute=True)
    for i in (0, 1, 2, 4):
        check(host(o)[i], want[i], most[i], BF16_HALF_STEP, f"o of row {i}")
    for i in (0, 1, 4):
        check(pool[where[i]], want_final[i], most_final[i], what=f"state {i}")
    same = [i for i in range(9) if i not in (7, 3, 0)]
    assert torch.equal(pool[same], before[same])
    A.linear_attn_step(A.LinearBatch(), case.tq, case.tk, case.tv, case.tg, o)         # no states at all: every row alone
    case.initial[:] = 0.0
    check(o, case.forward()[0], case.forward(absolute=True)[0], BF16_HALF_STEP, "o without states")


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (3, 3, 104)])
def test_a_prompt_and_steps_behind_it_are_one_sequence(A, hq, hkv, d):
    """Chunked prompts of several lengths into the pool, a second chunk of one of them, steps of all: as one forward over everything."""
    import torch
    lengths, steps, more = [70, 300, 1], 5, 130
    whole = Case([n + steps + (more if i == 1 else 0) for i, n in enumerate(lengths)], hq, hkv, d, 22, False, False).to_device()
    pool, slots = torch.full((6, hkv, d, d), float("nan"), device="cuda"), [4, 0, 2]
    o = torch.full_like(whole.tq, float("nan"))
    starts = whole.cu[:-1]

    def pack(spans, slots, first):
        rows = torch.cat([torch.arange(a, e) for a, e in spans]).cuda()
        cu = torch.tensor(np.concatenate([[0], np.cumsum([e - a for a, e in spans])]), dtype=torch.int32, device="cuda")
        batch = A.LinearBatch(cu, initial_slots=slots_of([-1] * len(spans) if first else slots), final_slots=slots_of(slots))
        q, k, v, g = (x[rows].contiguous() for x in (whole.tq, whole.tk, whole.tv, whole.tg))
        out = torch.empty_like(q)
        size = A.linear_attn_workspace_bytes(batch, len(rows), hq, hkv, d)
        A.linear_attn_fwd(batch, q, k, v, g, out, torch.empty(size, dtype=torch.uint8, device="cuda"), initial=pool, final=pool)
        o[rows] = out

    pack([(a, a + n) for a, n in zip(starts, lengths)], slots, True)
    pack([(starts[1] + 300, starts[1] + 300 + more)], [0], False)
    at = [a + n + (more if i == 1 else 0) for i, (a, n) in enumerate(zip(starts, lengths))]
    batch = A.LinearBatch(initial_slots=slots_of(slots), final_slots=slots_of(slots))
    for i in range(steps):
        rows = torch.tensor([a + i for a in at]).cuda()
        out = torch.empty(3, hq, d, dtype=torch.bfloat16, device="cuda")
        A.linear_attn_step(batch, whole.tq[rows], whole.tk[rows], whole.tv[rows], whole.tg[rows], out, initial=pool, final=pool)
        o[rows] = out
    check_forward(whole, o, pool[slots])


# ---------------------------------------------------------------------------------------------------------------- how the calls run
def test_two_runs_are_the_same_bits_whatever_the_workspace_held(A):
    import torch
    case = Case([900, 33, 400], 4, 2, 128, 30, False, True).to_device()
    first, second = case.run_backward(A), case.run_backward(A, workspace=torch.zeros(1 << 26, dtype=torch.uint8, device="cuda"))
    for name in first:
        assert torch.equal(first[name], second[name]), name
    for a, b in zip(case.run_forward(A), case.run_forward(A)):
        assert torch.equal(a, b)


def test_captured_calls_replay_with_the_lengths_and_slots_they_find(A):
    import torch
    cases = [Case(n, 4, 2, 64, 31 + i, False, True) for i, n in enumerate(([700, 40, 60], [1, 799, 0], [300, 300, 150]))]
    rows = 800
    q, k, v, do = (torch.empty(rows, h, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2, 4))
    g, initial, d_final = torch.empty(rows, 2, device="cuda"), torch.empty(3, 2, 64, 64, device="cuda"), torch.empty(3, 2, 64, 64, device="cuda")
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    batch = A.LinearBatch(cu)
    o, final = torch.empty_like(q), torch.empty_like(initial)
    out = {"dq": torch.empty(rows, 4, 64, device="cuda"), "dk": torch.empty(rows, 2, 64, device="cuda"), "dv": torch.empty(rows, 2, 64, device="cuda"),
           "dg": torch.empty(rows, 2, device="cuda"), "d_initial": torch.empty_like(initial)}
    ws = [torch.empty(A.linear_attn_workspace_bytes(batch, rows, 4, 2, 64, backward=b), dtype=torch.uint8, device="cuda") for b in (False, True)]

    def both():
        A.linear_attn_fwd(batch, q, k, v, g, o, ws[0], initial=initial, final=final)
        A.linear_attn_bwd(batch, q, k, v, g, do, out["dq"], out["dk"], out["dv"], ws[1], initial=initial, d_final=d_final, d_log_decay=out["dg"],
                          d_initial=out["d_initial"])

    def fill(case):
        for to, x in ((q, case.tq), (k, case.tk), (v, case.tv), (do, case.tdo), (g, case.tg)):
            to[:case.T] = x
        initial.copy_(case.tinitial), d_final.copy_(case.td_final), cu.copy_(case.tcu)
        for x in (o, final, *out.values()):
            x.fill_(float("nan"))

    for case in cases:
        case.to_device()
    fill(cases[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in (0, 1, 2, 1, 0):
        case = cases[i]
        fill(case)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(host(o)[:case.T], case.forward()[0], case.forward(absolute=True)[0], BF16_HALF_STEP, f"o, replay of pack {i}")
        assert torch.isnan(o[case.T:].float()).all()
        want = {name: x.clone() for name, x in out.items()}
        both()
        for name in out:
            assert torch.equal(out[name][:case.T] if name != "d_initial" else out[name], want[name][:case.T] if name != "d_initial" else want[name]), name


def test_a_captured_step_replays_on_its_own_states(A):
    import torch
    case = Case([6, 6], 2, 2, 64, 33, False, True).to_device()
    pool = case.tinitial.clone()
    q, k, v, g, o = (torch.empty_like(x[:2]) for x in (case.tq, case.tk, case.tv, case.tg, case.tq))
    batch = A.LinearBatch()
    graph = torch.cuda.CUDAGraph()
    A.linear_attn_step(batch, case.tq[:2], case.tk[:2], case.tv[:2], case.tg[:2], o, initial=pool.clone(), final=pool.clone())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        A.linear_attn_step(batch, q, k, v, g, o, initial=pool, final=pool)
    got = torch.empty_like(case.tq)
    for i in range(6):
        rows = [i, 6 + i]
        for to, x in ((q, case.tq), (k, case.tk), (v, case.tv), (g, case.tg)):
            to.copy_(x[rows])
        graph.replay()
        got[rows] = o
    check_forward(case, got, pool)


def test_another_stream(A):
    import torch
    case = Case([900, 33], 2, 2, 64, 34, False, True).to_device()
    want, want_final = case.run_forward(A)
    grads = case.run_backward(A)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    ws = [case.workspace(A, case.batch(A), b) for b in (False, True)]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        o, final = case.run_forward(A, workspace=ws[0])
        got = case.run_backward(A, workspace=ws[1])
    stream.synchronize()
    assert torch.equal(o, want) and torch.equal(final, want_final)
    assert all(torch.equal(got[name], grads[name]) for name in grads)


def test_nothing_to_do(A):
    import torch
    empty = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    none = torch.empty(0, 2, device="cuda")
    states = torch.randn(3, 2, 64, 64, device="cuda")
    # no sequence
    batch = A.LinearBatch(torch.zeros(1, dtype=torch.int32, device="cuda"))
    A.linear_attn_fwd(batch, empty, empty, empty, none, empty, None)
    dg = torch.full((2,), float("nan"), device="cuda")
    A.linear_attn_bwd(batch, empty, empty, empty, torch.zeros(2, device="cuda"), empty, empty, empty, empty, None, d_log_decay=dg)
    assert (dg == 0).all()
    A.linear_attn_step(A.LinearBatch(), empty, empty, empty, none, empty)
    # sequences without rows: the states pass, both ways
    batch = A.LinearBatch(torch.zeros(4, dtype=torch.int32, device="cuda"))
    final = torch.full_like(states, float("nan"))
    A.linear_attn_fwd(batch, empty, empty, empty, none, empty, None, initial=states, final=final)
    assert torch.equal(final, states)
    d_initial = torch.full_like(states, float("nan"))
    dg.fill_(float("nan"))
    ws = torch.empty(A.linear_attn_workspace_bytes(batch, 0, 2, 2, 64, backward=True), dtype=torch.uint8, device="cuda")
    A.linear_attn_bwd(batch, empty, empty, empty, torch.zeros(2, device="cuda"), empty, empty, empty, empty, ws, initial=states, d_final=states,
                      d_log_decay=dg, d_initial=d_initial)
    assert torch.equal(d_initial, states) and (dg == 0).all()


def test_many_short_sequences_among_a_long_one(A):
    rng = np.random.default_rng(5)
    lengths = list(rng.integers(0, 4, 150)) + [900] + list(rng.integers(0, 4, 150))
    case = Case(lengths, 2, 1, 32, 35, False, True).to_device()
    check_forward(case, *case.run_forward(A))
    check_backward(case, case.run_backward(A))
