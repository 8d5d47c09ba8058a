"""The oracle of the serving loop against hand cases and against the single-layout rotation."""
import numpy as np
import pytest

from oracle import mquant_oracle as orc


def test_plan_of_a_hand_case():
    """Pages of 16: sequence 0 has 15 tokens and gets 3 (one new page), 1 has ended and owned two pages behind a shared
    one, 2 asks for more than there is room for, 3 comes behind it and gets nothing."""
    table = np.array([[4, -1, -1], [0, 2, 3], [-1, -1, -1], [1, -1, -1]], dtype=np.int32)
    ring = np.array([7, -1, -1, -1, -1, 5, 6, 8], dtype=np.int32)              # 5, 6, 8, 7 from place 5 on
    out = orc.step_plan([15, 40, 0, 3], [3, -1, 48, 1], table, 16, ring, [5, 4], 50, shared=[0, 1, 0, 0], order=[1, 2, 0] + [0] * 47)
    start, pos, slots, length, state = out
    assert start.tolist() == [0, 3, 3, 3, 3] and length.tolist() == [18, 0, 0, 3]
    assert pos[:4].tolist() == [16, 17, 15, -1] and slots[:4].tolist() == [80, 81, 79, -1]
    assert table[0].tolist() == [4, 5, -1] and ring.tolist() == [7, 2, 3, -1, -1, 5, 6, 8] and state.tolist() == [6, 5]


def test_rotary_of_interleaved_pairs_is_the_plain_rotation():
    rng = np.random.default_rng(0)
    x, pos = rng.standard_normal((7, 3 * 16)), rng.integers(0, 9000, 7)
    f = orc.rotary_frequencies(16, 10000.0)
    assert np.allclose(orc.rotary_f64(x, None, pos, 3, f, halves=False), orc.rope_apply_f64(x, pos, 3), atol=1e-12)
    # halves: the same pairs at other places
    place = np.concatenate([np.arange(0, 16, 2), np.arange(1, 16, 2)])
    y = orc.rotary_f64(x.reshape(7, 3, 16)[:, :, place].reshape(7, 48), None, pos, 3, f, halves=True)
    assert np.allclose(y.reshape(7, 3, 16), orc.rope_apply_f64(x, pos, 3).reshape(7, 3, 16)[:, :, place], atol=1e-12)


def test_rotary_of_axes_and_parts():
    x = np.tile([1.0, 0.0, 1.0, 0.0, 5.0, 6.0], (1, 1))
    y = orc.rotary_f64(x, None, [[2], [3]], 1, [0.5, 1.0], halves=False, sections=(1, 1), scale=2.0)
    assert np.allclose(y, [[2 * np.cos(1), 2 * np.sin(1), 2 * np.cos(3), 2 * np.sin(3), 5, 6]], atol=1e-15)


def test_stretched_frequencies():
    f = orc.rotary_frequencies(64, 1e4)
    assert np.allclose(orc.rotary_frequencies(64, 1e4, "linear", 4.0), f / 4)
    b = orc.rotary_frequencies(64, 1e4, "base", 4.0)
    assert b[0] == 1 and np.isclose(b[-1], f[-1] / 4)                           # the slowest pair is stretched by the factor
    t = orc.rotary_frequencies(64, 1e4, "turns", 4.0, trained=4096, low=1, high=32)
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(t[turns >= 32], f[turns >= 32]) and np.allclose(t[turns <= 1], f[turns <= 1] / 4)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (t[between] < f[between]).all() and (t[between] > f[between] / 4).all()


@pytest.mark.parametrize("args,u,want", [
    ((1.0, 0, 1.0, 0.0), 0.0, 0), ((1.0, 0, 1.0, 0.0), 0.3, 1), ((1.0, 0, 1.0, 0.0), 0.99, 3), ((0.0, 0, 1.0, 0.0), 0.99, 1),
    ((1.0, 1, 1.0, 0.0), 0.99, 1), ((1.0, 0, 0.5, 0.0), 0.99, 1), ((1.0, 0, 0.55, 0.0), 0.99, 2), ((1.0, 0, 0.55, 0.0), 0.5, 1),
    ((1.0, 0, 1.0, 0.3), 0.99, 2), ((1.0, 0, 1.0, 0.6), 0.99, 1)])
def test_tokens_of_a_hand_case(args, u, want):
    """Probabilities 1/8, 1/2, 1/4, 1/8."""
    token, logprob = orc.sample_f64(np.log([0.125, 0.5, 0.25, 0.125]), *args, u)
    assert token == want and logprob <= 0


def test_equal_logits_and_rows_without_tokens():
    assert orc.sample_f64([2.0, 2.0, 2.0], 1.0, 2, 1.0, 0.0, 0.99)[0] == 1          # of equal ones the lowest numbers are kept
    assert orc.sample_f64([-np.inf, np.nan], 1.0, 0, 1.0, 0.0, 0.5) == (-1, -np.inf)
    assert orc.sample_f64([3.0, np.inf, np.inf], 1.0, 0, 1.0, 0.0, 0.6) == (2, pytest.approx(-np.log(2)))
