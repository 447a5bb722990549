"""Closed forms and differences that pin the log-probability oracle."""

import numpy as np

from oracle import logprob_oracle as lo


def test_uniform_and_two_entries():
    logprob, entropy, lse, _, _ = lo.logprob_rows(np.zeros((1, 8)), np.array([3]))
    assert abs(logprob[0] + np.log(8)) < 1e-15 and abs(entropy[0] - np.log(8)) < 1e-15 and abs(lse[0] - np.log(8)) < 1e-15
    z = np.array([[0.0, np.log(3.0)]])
    logprob, entropy, lse, _, _ = lo.logprob_rows(z, np.array([0]))
    assert abs(logprob[0] - np.log(0.25)) < 1e-15
    assert abs(entropy[0] - (0.25 * np.log(4) + 0.75 * np.log(4 / 3))) < 1e-15
    # twice the scale: odds 1 : 9
    logprob, _, _, _, _ = lo.logprob_rows(z, np.array([0]), logit_scale=2.0)
    assert abs(logprob[0] - np.log(0.1)) < 1e-15


def test_masked_rows_and_rows_of_minus_infinity():
    z = np.array([[1.0, 2.0], [-np.inf, -np.inf], [0.0, -np.inf]])
    logprob, entropy, lse, log_q, counts = lo.logprob_rows(z, np.array([-100, 1, 0]))
    assert logprob[0] == entropy[0] == lse[0] == 0 and not counts[0]
    assert logprob[1] == lse[1] == -np.inf and entropy[1] == 0
    assert logprob[2] == entropy[2] == lse[2] == 0
    d = lo.logprob_grad(log_q, entropy, counts, np.array([-100, 1, 0]), np.ones(3), np.ones(3))
    assert not d.any()


def test_gradient_is_that_of_differences():
    rng = np.random.default_rng(1)
    z, y, r, h, a = rng.normal(size=(4, 9)), np.array([0, 5, 8, 2]), rng.normal(size=4), rng.normal(size=4), 0.7

    def value(z):
        logprob, entropy, _, _, _ = lo.logprob_rows(z, y, a)
        return (r * logprob + h * entropy).sum()

    _, entropy, _, log_q, counts = lo.logprob_rows(z, y, a)
    d = lo.logprob_grad(log_q, entropy, counts, y, r, h, a)
    for i in np.ndindex(*z.shape):
        up, down = z.copy(), z.copy()
        up[i] += 1e-5
        down[i] -= 1e-5
        assert abs((value(up) - value(down)) / 2e-5 - d[i]) < 1e-9
    assert np.abs(d.sum(1)).max() < 1e-15  # a shift of all logits changes nothing


def test_best_breaks_ties_by_column():
    z = np.array([[1.0, 3.0, 3.0, np.nan, -np.inf, 2.0]])
    assert lo.best(z, 6).tolist() == [[1, 2, 5, 0, 3, 4]]
