"""Pins of the linear attention's oracle, independent of its own code: the sum over pairs, closed forms, finite differences."""
import numpy as np
import pytest

from oracle import linear


def case(lengths, hq, hkv, d, seed, fixed=False):
    rng = np.random.default_rng(seed)
    T = sum(lengths)
    q, do = rng.standard_normal((2, T, hq, d))
    k, v = rng.standard_normal((2, T, hkv, d))
    g = -rng.exponential(0.3, (hkv,) if fixed else (T, hkv))
    initial, d_final = rng.standard_normal((2, len(lengths), hkv, d, d))
    return q, k, v, g, do, initial, d_final


@pytest.mark.parametrize("hq,hkv", [(2, 2), (6, 2)])
def test_forward_is_the_sum_over_pairs(hq, hkv):
    lengths, d, scale = [5, 0, 9, 1], 6, 0.3
    q, k, v, g, _, initial, _ = case(lengths, hq, hkv, d, 1)
    o, final = linear.forward(q, k, v, g, lengths, scale, initial)
    t0 = 0
    for b, n in enumerate(lengths):
        for h in range(hq):
            c = h // (hq // hkv)
            run = np.concatenate([[0.0], np.cumsum(g[t0:t0 + n, c])])
            for t in range(n):
                want = np.exp(run[t + 1]) * (q[t0 + t, h] @ initial[b, c])
                for j in range(t + 1):
                    want = want + np.exp(run[t + 1] - run[j + 1]) * (q[t0 + t, h] @ k[t0 + j, c]) * v[t0 + j, c]
                np.testing.assert_allclose(o[t0 + t, h], scale * want, rtol=1e-12, atol=1e-12)
        t0 += n
    np.testing.assert_array_equal(final[1], initial[1])        # no tokens: the state passes


def test_without_decay_it_is_a_running_sum_and_with_all_of_it_only_the_own_token():
    q, k, v, _, _, _, _ = case([7], 1, 1, 4, 2)
    o, final = linear.forward(q, k, v, np.zeros(1), [7], 1.0)
    np.testing.assert_allclose(final[0, 0], k[:, 0].T @ v[:, 0], rtol=1e-12)
    np.testing.assert_allclose(o[6, 0], q[6, 0] @ (k[:, 0].T @ v[:, 0]), rtol=1e-12)
    o, _ = linear.forward(q, k, v, np.full(1, -np.inf), [7], 1.0)
    np.testing.assert_allclose(o[:, 0], (q[:, 0] * k[:, 0]).sum(1)[:, None] * v[:, 0], rtol=1e-12)


def test_pieces_with_the_state_handed_on_are_the_whole():
    q, k, v, g, _, initial, _ = case([12], 4, 2, 5, 3)
    o, final = linear.forward(q, k, v, g, [12], 0.5, initial)
    o1, s1 = linear.forward(q[:7], k[:7], v[:7], g[:7], [7], 0.5, initial)
    o2, s2 = linear.forward(q[7:], k[7:], v[7:], g[7:], [5], 0.5, s1)
    np.testing.assert_allclose(np.concatenate([o1, o2]), o, rtol=1e-12)
    np.testing.assert_allclose(s2, final, rtol=1e-12)


@pytest.mark.parametrize("fixed", [False, True])
def test_gradients_are_finite_differences(fixed):
    lengths, scale = [4, 1, 3], 0.7
    q, k, v, g, do, initial, d_final = case(lengths, 4, 2, 3, 4, fixed)
    grads = linear.backward(q, k, v, g, do, lengths, scale, initial, d_final)
    if fixed:
        grads["dg"] = grads["dg"].sum(0)

    def loss():
        o, final = linear.forward(q, k, v, g, lengths, scale, initial)
        return (o * do).sum() + (final * d_final).sum()

    h = 1e-6
    for x, name in ((q, "dq"), (k, "dk"), (v, "dv"), (g, "dg"), (initial, "d_initial")):
        for at in np.ndindex(x.shape):
            old = x[at]
            x[at] = old + h
            up = loss()
            x[at] = old - h
            down = loss()
            x[at] = old
            assert abs((up - down) / (2 * h) - grads[name][at]) < 1e-6 * (1 + abs(grads[name][at])), (name, at)
