"""Pins of the paged-cache oracle that do not rest on its own code."""
import numpy as np
import pytest
import torch

from oracle import attn_fwd, paged, rope


def test_e4m3_table_and_rounding_are_the_formats():
    codes = np.arange(256, dtype=np.uint8)
    values = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(paged.E4M3, values, equal_nan=True)
    x = np.concatenate([np.random.default_rng(0).uniform(-448, 448, 4000), values[np.isfinite(values)], np.geomspace(2.0 ** -12, 448, 500),
                        (values[:126] + values[1:127]) / 2]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(paged.to_e4m3(x.astype(np.float64)), want)


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.1, 1), (224.0, -1), (1.0, -8), (0.0, -100), (1e-40, -100), (1.75, -8), (1.7500001, -7)])
def test_exponents(top, e):
    assert paged.exponent_of(top) == e


def test_quantised_rows_are_within_half_a_step():
    x = np.random.default_rng(1).standard_normal((50, 3, 40)) * 10.0 ** np.random.default_rng(2).uniform(-5, 5, (50, 3, 1))
    codes, byte = paged.quantise(x)
    unit = 2.0 ** (byte.astype(np.float64) - 127)[..., None]
    assert (np.abs(paged.dequantise(codes, byte) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * unit) * (1 + 1e-12)).all()
    assert (np.abs(x).max(-1) <= 448 * unit[..., 0]).all() and (np.abs(x).max(-1) > 224 * unit[..., 0]).all()


def test_one_axis_is_the_rope_oracle():
    x, pos = np.random.default_rng(3).standard_normal((9, 2, 24)), np.arange(9) * 3
    for inverse, f in ((False, rope.rope), (True, rope.rope_transposed)):
        assert np.allclose(paged.turn_axes(x, pos[None], [0] * 12, inverse=inverse), f(x, pos), atol=1e-12, rtol=0)


def test_axes_turn_their_own_pairs():
    x = np.random.default_rng(4).standard_normal((6, 1, 8))
    pos = np.array([[1] * 6, [0] * 6])
    y = paged.turn_axes(x, pos, [0, 1, 0, 1])
    keep = [1, 3, 5, 7]
    assert np.array_equal(y[..., keep], x[..., keep]) and not np.allclose(y[..., [0, 2]], x[..., [0, 2]])


@pytest.mark.parametrize("size", [1, 4, 16])
def test_attention_over_pages_is_the_packed_oracle(size):
    rng = np.random.default_rng(5)
    lengths, hq, hkv, d = [7, 1, 19], 4, 2, 8
    q, k, v = (rng.standard_normal((27, h, d)) for h in (hq, hkv, hkv))
    ref_o, ref_lse = attn_fwd(q, k, v, lengths, 0.3)
    width = -(-19 // size)
    table = rng.permutation(width * 3).reshape(3, width)
    pools = [np.full((width * 3, hkv, size, d), np.nan) for _ in range(2)]
    cu = np.concatenate([[0], np.cumsum(lengths)])
    for s, n in enumerate(lengths):
        for p in range(n):
            for pool, x in zip(pools, (k, v)):
                pool[table[s, p // size], :, p % size] = x[cu[s] + p]
    for new in ([7, 1, 19], [1, 1, 1], [3, 0, 10]):
        rows = np.concatenate([np.arange(cu[s + 1] - n, cu[s + 1]) for s, n in enumerate(new)])
        o, lse = paged.attention(q[rows], *pools, np.concatenate([[0], np.cumsum(new)]), lengths, table, size, 0.3)
        assert np.allclose(o, ref_o[rows], atol=1e-12) and np.allclose(lse, ref_lse[:, rows], atol=1e-12)


def test_rows_without_a_place():
    pool = np.ones((1, 1, 4, 2))
    o, lse = paged.attention(np.ones((3, 1, 2)), pool, pool, [0, 3], [1], [[0]], 4, 1.0)
    assert (o[:2] == 0).all() and np.isinf(lse[0, :2]).all() and np.allclose(o[2], 1.0) and np.isclose(lse[0, 2], 2.0)
