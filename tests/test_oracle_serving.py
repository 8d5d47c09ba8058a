"""The oracle of the serving step against hand cases, brute force and the single-prompt attention."""
import numpy as np
import pytest

from oracle import mquant_oracle as orc


def test_norm_of_a_hand_case():
    """A head (3, 4, 0, 0) has mean square 25/4: divided by 2.5; position 0 turns nothing."""
    x = np.array([[3.0, 4.0, 0.0, 0.0]])
    y = orc.qk_norm_rope_f64(x, np.array([1.0, 2.0, 1.0, 1.0]), [0], 1, eps=0.0)
    assert np.allclose(y, [[1.2, 3.2, 0.0, 0.0]], rtol=0, atol=1e-15)


def test_norm_then_rotation_keeps_the_root_mean_square():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 3 * 16)) * 7
    y = orc.qk_norm_rope_f64(x, np.ones(16), np.arange(5) * 1000, 3, eps=0.0)
    assert np.allclose((y.reshape(5, 3, 16) ** 2).mean(axis=2), 1.0, atol=1e-12)
    assert np.allclose(orc.qk_norm_rope_f64(x, None, np.arange(5), 3), orc.rope_apply_f64(x, np.arange(5), 3), atol=0)


def test_slots_of_a_hand_case():
    table = np.array([[4, -1, 2], [0, 9, 1]])
    assert orc.cache_slot(table, 16, 0, 0, 5) == (4, 0)
    assert orc.cache_slot(table, 16, 0, 47, 5) == (2, 15)
    assert orc.cache_slot(table, 16, 1, 33, 5) == (1, 1)
    for seq, pos in ((0, 16), (1, 16), (0, 48), (0, -1)):          # no page, page out of range, behind the table, negative
        assert orc.cache_slot(table, 16, seq, pos, 5) is None


@pytest.mark.parametrize("spans", [[], [(3, 20)], [(0, 4), (10, 9)]])
def test_a_prompt_through_the_cache_is_the_prompt_by_itself(spans):
    """Rows in AIFS order, appended to a cache and attended over it, give what attention by the unified mask gives."""
    rng = np.random.default_rng(1)
    T, hq, hkv, D, P = 41, 4, 2, 8, 16
    q, k, v = (rng.standard_normal((T, h * D)) for h in (hq, hkv, hkv))
    perm, _, _ = orc.aifs_build_perm(T, spans)
    kp, vp = np.full((5, hkv, P, D), np.nan), np.full((5, hkv, P, D), np.nan)
    table = np.array([[7, 7, 7], [3, 0, 2]])
    start = np.array([0, 0, T])
    orc.kv_append(kp, vp, table, start, perm, k[perm], v[perm])
    got = orc.paged_attention_f64(q[perm], kp, vp, table, start, perm, hq)
    want = orc.aifs_attention_f64(q[perm], k[perm], v[perm], perm, hq, hkv)
    assert np.allclose(got, want, atol=1e-13)


def test_rows_that_see_nothing_and_rows_of_no_sequence():
    rng = np.random.default_rng(2)
    kp, vp = rng.standard_normal((2, 1, 16, 8)), rng.standard_normal((2, 1, 16, 8))
    o = orc.paged_attention_f64(rng.standard_normal((4, 8)), kp, vp, np.array([[1]]), np.array([1, 3]), np.array([5, -1, 0, 5]), 1)
    assert np.isnan(o[0]).all() and np.isnan(o[3]).all()
    assert (o[1] == 0).all() and np.allclose(o[2], vp[1, 0, 0], atol=1e-15)


def test_adapters_of_a_hand_case():
    x = np.array([[1.0, 2.0], [3.0, 5.0]])
    a = np.array([[[1.0, 1.0]], [[2.0, 0.0]]])
    b = np.array([[[10.0], [1.0], [0.0]], [[0.5], [0.0], [1.0]]])
    base = np.ones((2, 3))
    y = orc.lora_f64(x, [1, 0], [0, 1], a, b, [2.0, 1.0], base)
    assert np.array_equal(y, [[161.0, 17.0, 1.0], [2.0, 1.0, 3.0]])
    assert np.array_equal(orc.lora_f64(x, None, [-1, 2], a, b, [2.0, 1.0], base), base)
