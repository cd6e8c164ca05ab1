"""The oracle of the residual step and the vocabulary loss against differences and closed forms, on the CPU."""
import numpy as np
import pytest

from oracle import lm


def _difference(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        g[i] = (up - f()) / (2 * h)
        x[i] = keep
    return g


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("per", [1, 2, 5])
def test_residual_gradients_are_the_differences(post, pre, center, per):
    rng = np.random.default_rng(7 * per + post)
    rows, n = 5, 6
    X, H, dXo, dZ = (rng.standard_normal((rows, n)) for _ in range(4))
    gate = rng.standard_normal((-(-rows // per), n))
    w_post, b_post, w_pre, b_pre = (rng.standard_normal(n) for _ in range(4))
    kw = dict(gate=gate, per=per, w_post=w_post, b_post=b_post, w_pre=w_pre, post=post, pre=pre, center=center, skip=0.7, scale=1.3, eps=1e-3)

    def value():
        Xo, Z = lm.residual_forward(X, H, b_pre=b_pre, **kw)
        return (dXo * Xo).sum() + ((dZ * Z).sum() if pre else 0.0)

    g = lm.residual_backward(lm.residual_forward(X, H, b_pre=b_pre, **kw)[0], H, dXo, dZ, **kw)
    pairs = {"dX": X, "dH": H, "dgate": gate}
    pairs.update({"dw_post": w_post, "db_post": b_post} if post else {})
    pairs.update({"dw_pre": w_pre, "db_pre": b_pre} if pre else {})
    for name, x in pairs.items():
        np.testing.assert_allclose(g[name], _difference(value, x), rtol=1e-6, atol=1e-7, err_msg=name)


@pytest.mark.parametrize("tau", [1.0, 2.5])
@pytest.mark.parametrize("terms", ["label", "top", "both"])
def test_vocabulary_gradients_are_the_differences(tau, terms):
    rng = np.random.default_rng(3)
    rows, d, vocab = 4, 3, 7
    X, W = rng.standard_normal((rows, d)), rng.standard_normal((vocab, d))
    label = np.array([2, -100, 6, 7]) if terms != "top" else None
    ids = np.array([[2, 5, -1], [0, 0, 3], [-1, -1, -1], [6, 1, 9]]) if terms != "label" else None
    y = rng.standard_normal((rows, 3))
    dl, dt = rng.standard_normal(rows), rng.standard_normal(rows)

    def value():
        o = lm.vocab_loss(X, W, label, ids, y, tau)
        return (dl * o["label_loss"]).sum() + (dt * o["top_loss"]).sum()

    o = lm.vocab_loss(X, W, label, ids, y, tau, dl, dt)
    np.testing.assert_allclose(o["dX"], _difference(value, X), rtol=1e-6, atol=1e-8)
    np.testing.assert_allclose(o["dW"], _difference(value, W), rtol=1e-6, atol=1e-8)


def test_vocabulary_losses_in_closed_form():
    # equal logits: every label costs log vocab; a teacher that is uniform over k of them costs log(vocab / k)
    X, W = np.ones((2, 4)), np.ones((8, 4))
    o = lm.vocab_loss(X, W, np.array([3, 8]), np.array([[1, 2], [-1, -1]]), np.zeros((2, 2)), 3.0)
    np.testing.assert_allclose(o["label_loss"], [np.log(8), 0.0])
    np.testing.assert_allclose(o["top_loss"], [np.log(4), 0.0])
    # the same entry twice is one entry with both shares
    a = lm.vocab_loss(X, W, None, np.array([[1, 1, 2], [1, 2, -1]]), np.array([[0.0, 0.0, 0.0], [np.log(2), 0.0, 5.0]]), 1.0)["top_loss"]
    np.testing.assert_allclose(a[0], a[1])
    # the lowest value of fp32 and minus infinity both leave the other entry everything
    y = np.array([[1.0, np.finfo(np.float32).min], [1.0, -np.inf]])
    np.testing.assert_allclose(lm.vocab_loss(X, W, None, np.array([[1, 2], [1, 2]]), y, 0.5)["top_loss"], [np.log(8)] * 2)
