"""Pins of the oracle of the history operators: closed forms and differences, on the CPU."""
import numpy as np
import pytest

from oracle import history_operators as ho


def _inputs(B=2, T=7, H=2, d=4, seed=0):
    g = np.random.default_rng(seed)
    x = [g.standard_normal((B, T, H, d)) for _ in range(4)]
    return (*x, g.standard_normal((B, H, d, d)), g.standard_normal((B, H, d, d)), np.array([-0.1, -1.3]))


def test_recurrence_equals_the_sum_over_pairs():
    q, k, v, _, s0, _, ld = _inputs()
    o, last = ho.linear_attention(q, k, v, ld, 0.7, s0, lengths=[7, 4])
    for b, n in ((0, 7), (1, 4)):
        for h in range(2):
            for t in range(n):
                want = np.exp(ld[h] * (t + 1)) * (q[b, t, h] @ s0[b, h])
                for s in range(t + 1):
                    want = want + np.exp(ld[h] * (t - s)) * (q[b, t, h] @ k[b, s, h]) * v[b, s, h]
                assert np.allclose(o[b, t, h], 0.7 * want, atol=1e-12)
            assert np.all(o[b, n:, h] == 0)
    assert np.allclose(last[0, 0], np.exp(-0.1 * 7) * s0[0, 0] + sum(np.exp(-0.1 * (6 - s)) * np.outer(k[0, s, 0], v[0, s, 0]) for s in range(7)))


@pytest.mark.parametrize("which", range(4))
def test_gradients_against_differences(which):
    q, k, v, do, s0, ds, ld = _inputs()
    lengths = [7, 5]
    args = [q, k, v, s0]

    def loss():
        o, last = ho.linear_attention(args[0], args[1], args[2], ld, 0.6, args[3], lengths)
        return (o * do).sum() + (last * ds).sum()
    grad = ho.linear_attention_backward(q, k, v, ld, 0.6, do, s0, ds, lengths)[which]
    g = np.random.default_rng(which)
    for _ in range(12):
        at = tuple(g.integers(0, n) for n in args[which].shape)
        keep, eps = args[which][at], 1e-5
        args[which][at] = keep + eps
        up = loss()
        args[which][at] = keep - eps
        down = loss()
        args[which][at] = keep
        assert abs((up - down) / (2 * eps) - grad[at]) < 1e-7


def test_rounding_to_e4m3_is_to_the_nearest_of_all_values():
    values = np.array(sorted({s * m for s in (-1, 1) for e in range(-6, 9) for m in [(1 + i / 8) * 2.0 ** e for i in range(8)] if m <= 448} |
                             {s * i * 2.0 ** -9 for s in (-1, 1) for i in range(8)}))
    x = np.random.default_rng(0).standard_normal(4000) * np.exp2(np.random.default_rng(1).uniform(-12, 8, 4000))
    x = np.clip(x, -448, 448)
    r = ho.round_e4m3(x)
    assert np.all(np.isin(r, values))
    assert np.array_equal(np.abs(r - x), np.abs(values[None] - x[:, None]).min(axis=1))
    assert ho.round_e4m3(17.0) == 16.0 and ho.round_e4m3(19.0) == 20.0         # halfway: to the even neighbour
    assert np.isnan(ho.round_e4m3(np.nan))


def test_scale_is_the_smallest_power_of_two():
    for amax in (0.0, 1e-45, 448.0, 448.0000001, 1.75, 1.7500001, 3e38):
        e = ho.scale_exponent(amax)
        assert amax <= 448 * 2.0 ** e and (e == -100 or amax > 448 * 2.0 ** (e - 1))


def test_attention_weights_and_empty_rows():
    g = np.random.default_rng(3)
    q, k8, v8 = g.standard_normal((2, 5, 4, 8)), ho.round_e4m3(g.standard_normal((2, 2, 64, 8))), np.ones((2, 2, 64, 8))
    one = np.ones((2, 2, 1))
    o, _ = ho.attention(q, k8, v8, one, 3 * one, [3, 0], 0.3, causal=True)
    assert np.all(o[0, :2] == 0) and np.allclose(o[0, 2:], 3.0) and np.all(o[1] == 0)
