"""Closed forms that pin the 64-bit restatement of the operators between the linears of a decoder layer."""
import numpy as np

from oracle import np_layer


def test_rmsnorm_of_a_constant_row_and_of_zeros():
    v, h = np_layer.rmsnorm(np.full((1, 8), 3.0), np.arange(8.0), 0.0)
    np.testing.assert_allclose(v[0], np.arange(8.0), rtol=1e-15)
    v, h = np_layer.rmsnorm(np.ones((1, 8)), np.ones(8), 1e-5, residual=-np.ones((1, 8)))
    assert not v.any() and not h.any() and np_layer.a8_scale(v)[0] == 1.0
    v, _ = np_layer.rmsnorm(np.array([[3.0, 4.0]]), np.ones(2), 0.0)
    np.testing.assert_allclose(v, np.array([[3.0, 4.0]]) / np.sqrt(12.5))


def test_rope_keeps_lengths_and_relative_angles():
    rng = np.random.default_rng(0)
    a, b = rng.normal(size=(1, 64)), rng.normal(size=(1, 64))
    np.testing.assert_array_equal(np_layer.rope_rotate(a, 0, 1e4), a)
    at = lambda x, p: np_layer.rope_rotate(x, p, 1e4)[0]  # noqa: E731
    np.testing.assert_allclose(np.linalg.norm(at(a, 91)), np.linalg.norm(a))
    np.testing.assert_allclose(at(a, 17) @ at(b, 5), at(a, 1012) @ at(b, 1000))   # only the distance counts
    one = np.zeros((1, 64))
    one[0, 0] = 1.0     # the first pair turns by one radian per position
    np.testing.assert_allclose(at(one, 2)[[0, 32]], [np.cos(2.0), np.sin(2.0)])


def test_attention_of_equal_scores_is_a_mean_and_of_nothing_is_zero():
    rng = np.random.default_rng(1)
    k, v = rng.normal(size=(6, 2, 4)), rng.normal(size=(6, 2, 4))
    out, spread, _ = np_layer.attn(np.zeros((3, 4, 4)), k, v, 3, 1.0)
    for i in range(3):
        for h in range(4):
            np.testing.assert_allclose(out[i, h], v[: 4 + i, h // 2].mean(axis=0))
            np.testing.assert_allclose(spread[i, h], np.abs(v[: 4 + i, h // 2]).mean(axis=0))
    out, _, _ = np_layer.attn(rng.normal(size=(3, 4, 4)), k, v, -2, 1.0)
    assert not out[:2].any()
    np.testing.assert_array_equal(out[2, 3], v[0, 1])
    assert np_layer.positions([0, 2, 2, 5], [2, 7, 1]) == ([0, 0, 2, 2, 2], [0, 1, -2, -1, 0])


def test_lora_batch_picks_the_requests_adapters():
    rng = np.random.default_rng(2)
    x, a, b = rng.normal(size=(5, 8)), rng.normal(size=(2, 3, 8)), rng.normal(size=(2, 4, 3))
    side, absside = np_layer.lora_batch(x, a, b, [0, 2, 3, 5], [1, -1, 0], np.array([2.0, -1.0]))
    np.testing.assert_allclose(side[:2], -(x[:2] @ a[1].T) @ b[1].T)
    assert not side[2].any() and not absside[2].any()
    np.testing.assert_allclose(side[3:], 2 * (x[3:] @ a[0].T) @ b[0].T)
    assert (absside >= np.abs(side) - 1e-12).all()
