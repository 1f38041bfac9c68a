"""Pins of the 64-bit oracle of the layer norm and of the calls on rows of logits: gradients against differences of
the forward formulas, hand cases, and limits that reduce to known results.  No GPU."""
import numpy as np
import pytest

from oracle import lm

H = 1e-6          # central differences of smooth functions in 64 bits: error about H^2 + 1e-16 / H
TOL = 2e-8


def _numeric(f, x):
    g = np.zeros_like(x)
    for at in np.ndindex(*x.shape):
        keep = x[at]
        x[at] = keep + H
        up = f()
        x[at] = keep - H
        g[at] = (up - f()) / (2 * H)
        x[at] = keep
    return g


def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(1)
    x, w, b, dy = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=7), rng.normal(size=(3, 7))
    f = lambda: float((lm.layer_norm_fwd(x, w, b, 1e-3).y * dy).sum())
    fwd = lm.layer_norm_fwd(x, w, b, 1e-3)
    got = lm.layer_norm_bwd(dy, x, w, fwd.mean, fwd.rstd)
    assert np.allclose(got.dx, _numeric(f, x), atol=TOL)
    assert np.allclose(got.dweight, _numeric(f, w), atol=TOL)
    assert np.allclose(got.dbias, _numeric(f, b), atol=TOL)


def test_layer_norm_by_hand():
    y = lm.layer_norm_fwd(np.array([[1.0, 3.0]]), None, None, 0.0)
    assert np.array_equal(y.y, [[-1.0, 1.0]]) and y.mean[0] == 2.0 and y.rstd[0] == 1.0
    one = lm.layer_norm_fwd(np.array([[5.0]]), np.array([2.0]), np.array([0.5]), 1e-5)
    assert one.y[0, 0] == 0.5


def test_log_probs_by_hand():
    r = lm.log_probs(np.array([[0.0, np.log(3.0)], [-np.inf, 2.0], [-np.inf, -np.inf], [np.nan, 1.0]]), 1.0)
    assert np.allclose(np.exp(r.logp[0]), [0.25, 0.75])
    assert np.isclose(r.entropy[0], -(0.25 * np.log(0.25) + 0.75 * np.log(0.75)))
    assert r.logp[1, 1] == 0.0 and r.logp[1, 0] == -np.inf and r.entropy[1] == 0.0
    assert (r.logp[2] == -np.inf).all() and r.max[2] == -np.inf and r.logsum[2] == 0.0
    assert np.isnan(r.logp[3]).all()
    assert list(lm.top_columns(np.array([1.0, np.nan, 2.0, 1.0, -np.inf, -0.0, 0.0]), 7)) == [2, 0, 3, 5, 6, 4, 1]


@pytest.mark.parametrize("inv_t", [1.0, 0.5])
def test_log_prob_gradient_against_differences(inv_t):
    rng = np.random.default_rng(2)
    x = rng.normal(size=(3, 6))
    x[1, 2] = -np.inf
    tokens, a, c = np.array([4, 0, -1]), rng.normal(size=3), rng.normal(size=3)

    def f():
        r = lm.log_probs(x, inv_t)
        return float(sum((a[i] * r.logp[i, tokens[i]] if tokens[i] >= 0 else 0.0) + c[i] * r.entropy[i] for i in range(3)))

    r = lm.log_probs(x, inv_t)
    got = lm.log_probs_bwd(x, inv_t, tokens, r.max, r.logsum, r.entropy, a, c)
    with np.errstate(invalid="ignore"):
        want = _numeric(f, x)
    assert got[1, 2] == 0.0
    got[1, 2] = want[1, 2] = 0.0
    assert np.allclose(got, want, atol=TOL)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("inv_t", [1.0, 2.0])
def test_distillation_gradient_against_differences(tail, inv_t):
    rng = np.random.default_rng(3)
    x = rng.normal(size=(4, 9))
    x[3, 5] = -np.inf
    teacher = rng.normal(size=(4, 9))
    ids = np.array([[0, 3, 8], [1, 2, -1], [4, 4, 6], [7, 0, 99]])       # an empty slot, a column named twice, a bad id
    t = np.take_along_axis(teacher, np.clip(ids, 0, 8), 1) - np.log(np.exp(teacher).sum(1, keepdims=True))
    t[2, 1] -= 1.0
    scale = rng.normal(size=4)
    f = lambda: float((lm.distill(x, inv_t, ids, t, tail, None).loss * scale).sum())
    got = lm.distill(x, inv_t, ids, t, tail, scale).grad
    with np.errstate(invalid="ignore"):
        want = _numeric(f, x)
    got[3, 5] = want[3, 5] = 0.0
    assert np.allclose(got, want, atol=TOL)


def test_distillation_limits():
    rng = np.random.default_rng(4)
    x = rng.normal(size=(2, 5))
    lp = lm.log_probs(x, 1.0).logp
    every = np.tile(np.arange(5), (2, 1))
    for tail in (False, True):        # the teacher is the student: nothing to learn
        r = lm.distill(x, 1.0, every, lp, tail, None)
        assert np.allclose(r.loss, 0.0, atol=1e-14) and np.allclose(r.grad, 0.0, atol=1e-14)
    r = lm.distill(x, 1.0, np.array([[1, 3], [0, 2]]), np.take_along_axis(lp, np.array([[1, 3], [0, 2]]), 1), True, None)
    assert np.allclose(r.loss, 0.0, atol=1e-14) and np.allclose(r.grad, 0.0, atol=1e-14)
    one = lm.distill(x, 1.0, np.array([[2], [4]]), np.zeros((2, 1)), False, None)        # a hard label: cross entropy
    assert np.allclose(one.loss, [-lp[0, 2], -lp[1, 4]])
    none = lm.distill(x, 1.0, np.array([[-1], [5]]), np.zeros((2, 1)), False, None)
    assert not none.loss.any() and not none.grad.any()
    none = lm.distill(x, 1.0, np.array([[-1], [5]]), np.zeros((2, 1)), True, None)       # all mass in the remainder
    assert np.allclose(none.loss, 0.0, atol=1e-14) and np.allclose(none.grad, 0.0, atol=1e-14)
    x[0, 2] = -np.inf
    assert lm.distill(x, 1.0, np.array([[2], [4]]), np.zeros((2, 1)), False, None).loss[0] == np.inf
    x[0] = -np.inf
    r = lm.distill(x, 1.0, np.array([[2], [4]]), np.zeros((2, 1)), False, None)
    assert r.loss[0] == 0.0 and not r.grad[0].any()
