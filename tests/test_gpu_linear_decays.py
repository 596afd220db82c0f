"""Linear attention: the decays' gradients along long sequences that no workgroup cuts, against the fp64 oracle, every 64 rows by what they themselves are summed
from, and a fixed decay's by the norm of its rows'."""
import numpy as np
import pytest

from linear_util import TERMS, Case, host

pytestmark = pytest.mark.gpu

NEAR = 4        # groups of 64 rows that what lies across one may be carried over


@pytest.fixture(scope="module")
def A():
    import paper_2504_20490_amd as A
    A.load_library()
    return A


def uncut(case, A):
    """Hints that no sequence has more than one row: then none is cut."""
    return case.batch(A, 1)


def room(case, most):
    """[groups, KV heads] of one sequence: what the gradients of 64 rows may be off by.  They are sums of the pairs with a row among them, and of what lies across them,
    which is no more than the rows' own gradients: `local`, by magnitudes.  What lies across may come out of differences that begin up to NEAR groups
    away on the side where the terms are smaller."""
    n, group = case.T, case.hq // case.hkv
    pairs = (np.abs(case.q[:n]) * most["dq"]).sum(-1).reshape(n, case.hkv, group).sum(-1) + (np.abs(case.k[:n]) * most["dk"]).sum(-1)
    per_row = most["dg"].reshape(-1, case.hkv)
    starts = range(0, n, 64)
    local = np.stack([pairs[a:a + 64].sum(0) + per_row[a:a + 64].max(0) for a in starts])
    behind = np.stack([local[i:i + NEAR + 1].max(0) for i in range(len(local))])
    before = np.stack([local[max(i - NEAR, 0):i + 1].max(0) for i in range(len(local))])
    return TERMS * np.minimum(behind, before)


@pytest.mark.parametrize("large", ["none", "last", "first", "middle", "values"])
@pytest.mark.parametrize("n,hq,hkv,d,rate,states", [(4096, 2, 2, 32, 0.15, False), (3000, 4, 2, 64, 0.05, True), (1500, 1, 1, 128, 0.15, False),
                                                    (2100, 2, 1, 104, 0.5, True)])
def test_large_gradients_elsewhere_leave_no_trace(A, n, hq, hkv, d, rate, states, large):
    """64 rows of d_o, or of v, 2^40 times the others: rows that their decays separate from these keep gradients as accurate as without."""
    case = Case([n], hq, hkv, d, 60, False, states, rate=rate)
    case.g = -np.full_like(case.g, np.float32(rate)).astype(np.float64) if large != "none" else case.g
    rows = {"none": slice(0, 0), "last": slice(n - 64, n), "first": slice(0, 64), "middle": slice(n // 2, n // 2 + 64), "values": slice(n // 2, n // 2 + 64)}[large]
    (case.v if large == "values" else case.do)[rows] *= 2.0 ** 40
    case.to_device()
    got, want = host(case.run_backward(A, uncut(case, A))["dg"]), case.backward()["dg"]
    off = np.abs(got - want)
    may = np.repeat(room(case, case.backward(absolute=True)), 64, axis=0)[:n]
    worst = np.unravel_index(np.argmax(off / may), off.shape)
    assert np.isfinite(got).all() and off[worst] <= may[worst], (worst, got[worst], want[worst], off[worst] / may[worst])


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("rate", [0.003, 0.03, 0.1, 0.3, 1.0])
@pytest.mark.parametrize("n,hq,hkv,d,states", [(8192, 2, 2, 32, False), (4000, 2, 1, 64, True), (2500, 1, 1, 128, False)])
def test_a_fixed_decays_gradient_over_a_long_sequence(A, n, hq, hkv, d, states, rate, f32):
    """A row's gradient is off by 2^-20 of its terms, which cancel by up to four: 2^-18 of the rows' 2-norm.  Rows share the error of what lies across 64 of them, and
    groups of 64 that of a difference carried over NEAR of them: the errors of 256 rows add up, those of different 256 as the root of their number, so the
    sum is off by sqrt(256) times that."""
    case = Case([n], hq, hkv, d, 61, True, states)
    case.g = np.full(hkv, -np.float32(rate)).astype(np.float64)
    case.to_device()
    got = host(case.run_backward(A, uncut(case, A), f32=f32)["dg"])
    case.fixed = False                           # (the gradients row by row)
    rows = case.backward()["dg"]
    off, may = np.abs(got - rows.sum(0)), 16 * 2.0 ** -18 * np.linalg.norm(rows, axis=0)
    assert (off <= may).all(), (off / may).tolist()


@pytest.mark.parametrize("rate", [0.3, 0.6, 1.0, 2.5])
@pytest.mark.parametrize("n,hq,hkv,d", [(8192, 2, 2, 32), (4000, 2, 1, 64), (2500, 1, 1, 128)])
def test_a_fixed_strong_decays_gradient(A, n, hq, hkv, d, rate):
    """With the same decay in every row, a weight's error is the same for all pairs as far apart, and pairs are counted into a row's gradient and out of it again: both
    times with one weight's bits, so that its error counts no more than the pair does.  What is left are the roundings of sums, 2^-21 (chains of 64 + 128),
    of four of them: 2^-20 of the rows' 2-norm, and sqrt(256) times that of their sum, as above."""
    case = Case([n], hq, hkv, d, 62, True, False)
    case.g = np.full(hkv, -np.float32(rate)).astype(np.float64)
    case.to_device()
    got = host(case.run_backward(A, uncut(case, A))["dg"])
    case.fixed = False
    rows = case.backward()["dg"]
    off, may = np.abs(got - rows.sum(0)), 16 * 2.0 ** -20 * np.linalg.norm(rows, axis=0)
    assert (off <= may).all(), (off / may).tolist()


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("hq,hkv,d", [(24, 24, 128), (24, 24, 64), (16, 4, 128), (12, 12, 104), (20, 20, 80)])
def test_packs_that_fill_the_device_are_run_to_run_the_same(A, hq, hkv, d, f32):
    """Many heads on segments of many groups of 64 rows: the same bits three times, and as uncut sequences.  Each of the two is off by 2^-20 of
    its terms, which cancel by up to four, 2^-18 of the norm of 64 rows' and their neighbours', in its own way, as states pass in other roundings: the two differ by
    up to twice that."""
    import torch
    torch.manual_seed(63)
    lengths = [1851, 4713, 898, 8207, 450]
    n = sum(lengths)
    q, do = (torch.randn(n, hq, d, device="cuda").bfloat16() for _ in range(2))
    k, v = (torch.randn(n, hkv, d, device="cuda").bfloat16() for _ in range(2))
    rate = 0.5 * 2.0 ** (-8.0 * torch.arange(hkv, device="cuda") / hkv)
    g = -rate * torch.exp(0.5 * torch.randn(n, hkv, device="cuda"))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")

    def run(hint):
        batch = A.LinearBatch(cu, max_rows=hint)
        ws = torch.full((A.linear_attn_workspace_bytes(batch, n, hq, hkv, d, backward=True),), 255, dtype=torch.uint8, device="cuda")
        t = torch.float32 if f32 else torch.bfloat16
        out = [torch.empty(n, h, d, dtype=t, device="cuda") for h in (hq, hkv, hkv)] + [torch.empty(n, hkv, device="cuda")]
        A.linear_attn_bwd(batch, q, k, v, g, do, *out[:3], ws, d_log_decay=out[3])
        return out

    first = run(max(lengths))
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(first, run(max(lengths))))
    uncut = run(1)[3].double()
    off = (first[3].double() - uncut)
    groups = lambda x: torch.nn.functional.pad(x * x, (0, 0, 0, -n % 64)).view(-1, 64, hkv).sum(1)
    size = groups(uncut)
    near = torch.stack([size, size.roll(1, 0), size.roll(-1, 0)]).max(0).values      # (groups of the packed rows, not of the sequences)
    assert (groups(off) <= (2 * 2.0 ** -18) ** 2 * near).all(), (groups(off) / near).max().sqrt().item()
