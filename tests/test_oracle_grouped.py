"""The oracle of the attention layers past the fixed windows, by other means:
against the windows' attention oracle, differences of its own forward, and
properties that the definitions give."""
import numpy as np
import pytest

from oracle import attention, grouped


def test_equals_the_window_oracle_where_both_apply():
    rng = np.random.default_rng(0)
    qkv, do = rng.standard_normal((2, 32, 3, 3, 64)), rng.standard_normal((2, 32, 3, 64))
    q, k, v = (qkv[:, :, i] for i in range(3))
    out, lse, _ = grouped.forward(q, k, v)
    r_out, r_lse = attention.forward(qkv)
    np.testing.assert_allclose(out, r_out, atol=1e-12)
    np.testing.assert_allclose(lse, r_lse, atol=1e-12)
    g, _ = grouped.backward(q, k, v, do)
    r = attention.backward(qkv, do)
    for i in range(3):
        np.testing.assert_allclose(g[i], r[:, :, i], atol=1e-12)


@pytest.mark.parametrize("n_q,n_k,causal,lengths", [(5, 7, True, None), (6, 4, True, [4, 2]),
                                                    (3, 6, False, [0, 5])])
def test_gradients_against_differences(n_q, n_k, causal, lengths):
    rng = np.random.default_rng(n_q)
    q = rng.standard_normal((2, n_q, 4, 8))
    k, v = rng.standard_normal((2, n_k, 2, 8)), rng.standard_normal((2, n_k, 2, 8))
    do = rng.standard_normal(q.shape)
    g, _ = grouped.backward(q, k, v, do, causal, lengths)
    ops = [q, k, v]
    h = 1e-5
    for i, t in enumerate(ops):
        d = rng.standard_normal(t.shape)
        f = [(grouped.forward(*ops[:i], t + s * d, *ops[i + 1:], causal, lengths)[0] * do).sum()
             for s in (h, -h)]
        # the third derivatives are of order 10: h^2 / 6 of them, rounding 1e-16 / h
        assert abs((f[0] - f[1]) / (2 * h) - (g[i] * d).sum()) < 1e-7


def test_rotary_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 1, 16))
    freqs = 100.0 ** (-np.arange(8) / 8)
    for half in (True, False):
        dots = [(grouped.rotary(q, [[p + 5]], freqs, half)
                 * grouped.rotary(k, [[p]], freqs, half)).sum() for p in (0, 3, 1000)]
        np.testing.assert_allclose(dots, dots[0], atol=1e-12)
        y = grouped.rotary(q, [[7]], freqs, half, scale=1.5)
        np.testing.assert_allclose(grouped.rotary(y, [[7]], freqs, half, 1 / 1.5, inverse=True), q,
                                   atol=1e-12)


def test_e4m3_grid_and_scales():
    grid = sorted({m * 2.0 ** e for e in range(-9, 6) for m in range(8, 16)}
                  | {m * 2.0 ** -9 for m in range(8)} | {448.0})
    grid = [v for v in grid if v <= 448]
    np.testing.assert_array_equal(grouped.e4m3(np.array(grid)), grid)
    assert grouped.e4m3(17.0) == 16.0 and grouped.e4m3(19.0) == 20.0       # ties to even
    assert grouped.e4m3(-1000.0) == -448.0 and np.isnan(grouped.e4m3(np.nan))
    for amax in (448.0, 448.0001, 1.0, 1e-30, 3e38, 0.0):
        s = grouped.needed_scale(np.array([amax]))
        assert amax <= 448 * s and (s == 2.0 ** -118 or amax > 224 * s)


def test_a_grown_block_is_held_as_if_appended_at_once():
    """A power of two costs no significant bit: but for values below 2^-6 units."""
    rng = np.random.default_rng(2)
    x = rng.uniform(1, 2, (40, 1, 8)) * np.array([1.0] * 20 + [30.0] * 20)[:, None, None]
    a, b = grouped.Cache(64, 1, 8), grouped.Cache(64, 1, 8)
    a.append(x, 0)
    for t in range(40):
        b.append(x[t:t + 1], t)
    np.testing.assert_array_equal(a.held, b.held)
