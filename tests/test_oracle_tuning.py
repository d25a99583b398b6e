"""The fp64 fine-tuning oracle pinned by closed forms, invariants and central
differences of its own losses (no GPU).

Differences: with step h = 1e-6 and losses of order one, the central
difference is off by about h^2 f''' / 6 + 1e-16 / h = 1e-10; the bound is 1e-8."""
import numpy as np
import pytest

from oracle import tuning as T


def _problem(seed, rows=23, cols=11, masked=0.3):
    rng = np.random.default_rng(seed)
    x = 2.0 * rng.standard_normal((rows, cols))
    y = rng.integers(0, cols, rows)
    y[rng.random(rows) < masked] = -100
    return rng, x, y


def _difference(f, x, d, h=1e-6):
    return (f(x + h * d) - f(x - h * d)) / (2.0 * h)


def test_logprobs_closed_forms():
    lp = T.token_logprobs(np.zeros((3, 8)), [0, 7, -1])
    np.testing.assert_allclose(lp, [-np.log(8.0), -np.log(8.0), 0.0], rtol=1e-15)
    # two columns: the logistic function of the difference over the temperature
    lp = T.token_logprobs(np.array([[1.0, 3.0]]), [0], temperature=0.5)
    np.testing.assert_allclose(lp, [-np.log1p(np.exp(4.0))], rtol=1e-14)
    # a banned column does not count
    lp = T.token_logprobs(np.array([[0.0, -np.inf, 0.0]]), [2])
    np.testing.assert_allclose(lp, [-np.log(2.0)], rtol=1e-15)
    # shifting a row changes nothing
    _, x, y = _problem(0)
    np.testing.assert_allclose(T.token_logprobs(x + 300.0, y), T.token_logprobs(x, y), atol=1e-12)


def test_factor_logprobs_are_those_of_the_product():
    rng, _, y = _problem(1)
    A, B = rng.standard_normal((23, 5)), rng.standard_normal((11, 5))
    np.testing.assert_array_equal(T.factor_logprobs(A, B, y, 0.7), T.token_logprobs(A @ B.T, y, 0.7))


def test_gradient_rows_sum_to_zero_and_left_out_rows_are_zero():
    rng, x, y = _problem(2)
    x[y < 0] = np.nan
    d = T.logits_gradient(x, y, rng.standard_normal(23), 1.3)
    np.testing.assert_allclose(d.sum(axis=1), 0.0, atol=1e-15)
    assert np.all(d[y < 0] == 0.0)


@pytest.mark.parametrize("smoothing,average", [(0.0, False), (0.1, False), (0.0, True), (0.2, True)])
def test_preference_gradient_by_differences(smoothing, average):
    rng, x, y = _problem(3)
    offsets = np.array([0, 4, 4, 11, 15, 20, 21])      # an empty sequence; rows 21, 22 in none
    ref = T.token_logprobs(x, y) + 0.5 * rng.standard_normal(23)
    args = dict(beta=0.7, smoothing=smoothing, average=average, temperature=1.3)
    d = rng.standard_normal(x.shape)
    got = T.preference_loss(x, y, offsets, ref, **args)
    want = _difference(lambda z: T.preference_loss(z, y, offsets, ref, **args)["loss"], x, d)
    assert abs(np.sum(got["grad"] * d) - want) < 1e-8


def test_preference_at_the_reference_is_log_two():
    _, x, y = _problem(4)
    ref = T.token_logprobs(x, y)
    r = T.preference_loss(x, y, np.array([0, 5, 23]), ref)
    np.testing.assert_allclose(r["loss"], np.log(2.0), rtol=1e-14)
    np.testing.assert_allclose(r["margins"], 0.0, atol=1e-14)


@pytest.mark.parametrize("sequences", [False, True])
@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_policy_gradient_by_differences(sequences, kl):
    rng, x, y = _problem(5)
    offsets = np.array([0, 0, 9, 15, 21]) if sequences else None
    lp = T.token_logprobs(x, y, 0.8)
    old = lp - rng.choice([-0.6, -0.1, 0.1, 0.6], 23)   # away from the borders of the clipped range
    ref = lp + 0.4 * rng.standard_normal(23)
    adv = rng.standard_normal(23)
    args = dict(offsets=offsets, clip_low=0.2, clip_high=0.3, kl_coef=kl, temperature=0.8)
    d = rng.standard_normal(x.shape)
    got = T.policy_loss(x, y, old, ref, adv, **args)
    want = _difference(lambda z: T.policy_loss(z, y, old, ref, adv, **args)["loss"], x, d)
    assert abs(np.sum(got["grad"] * d) - want) < 1e-8
    assert 0.0 < got["clipped"] < 1.0 and got["kl"] > 0.0


def test_policy_weights():
    y = np.array([1, -1, 2, -1, -1, 3])
    np.testing.assert_allclose(T.policy_weights(y), [1 / 3, 0, 1 / 3, 0, 0, 1 / 3])
    w = T.policy_weights(y, np.array([0, 3, 5, 6]))
    np.testing.assert_allclose(w, [1 / 6, 0, 1 / 6, 0, 0, 1 / 3])
    assert np.all(T.policy_weights(-np.ones(4, int)) == 0.0)


def test_clip_grad_norm():
    norm, out = T.clip_grad_norm([np.array([3.0]), np.zeros(0), np.array([[0.0, 4.0]])], 1.0)
    assert norm == 5.0
    np.testing.assert_allclose(out[0], [0.6])
    np.testing.assert_allclose(out[2], [[0.0, 0.8]])
    norm, out = T.clip_grad_norm([np.array([3.0, 4.0])], 5.0)
    assert norm == 5.0 and np.array_equal(out[0], [3.0, 4.0])
    # squares past the range of fp64
    norm, out = T.clip_grad_norm([np.array([3e200, 4e200])], 1.0)
    np.testing.assert_allclose(norm, 5e200)
    norm, _ = T.clip_grad_norm([np.array([3e-200, 4e-200])], 1.0)
    np.testing.assert_allclose(norm, 5e-200)


def test_policy_rows_outside_every_sequence():
    rng, x, y = _problem(6)
    y[[0, 1, 21, 22]] = 2
    lp = T.token_logprobs(x, y)
    old, ref, adv = lp - 0.1, lp + 0.3, rng.standard_normal(23)
    out, offsets = np.array([0, 1, 21, 22]), np.array([2, 9, 9, 21])
    inside = y.copy()
    inside[out] = -1
    want = T.policy_loss(x, inside, old, ref, adv, offsets, kl_coef=0.1)
    old[0], ref[1], adv[21], x[22] = np.nan, np.inf, -np.inf, np.nan
    got = T.policy_loss(x, y, old, ref, adv, offsets, kl_coef=0.1)
    for name in ("loss", "kl", "clipped", "coef"):
        np.testing.assert_array_equal(got[name], want[name])
    np.testing.assert_array_equal(got["grad"], want["grad"])
