"""The gradient in the logits, entry by entry, where a group of 64 logits holds some that lie far below the others, on the host build of
tests/test_cpu_lm.py (the same cases on the GPU: tests/test_gpu_vocab_far_logits.py).

X is the identity, so that the logits of row t are the column t of W, exactly, and column t of dW is the gradient in them, rounded to bf16.

Tolerance of an entry, in terms of what it is made of, its share p of the softmax times the row's weight (and the teacher's q): two roundings to bf16 (b = 2^-8, half
a unit of the last place in relative terms, each), the steps between the product and the gradient, and E.  Steps: with one temperature 65534 of them cover
at most the 104 log2 e = 150 powers of two below which no share is left in fp32, so a logit is off by at most 75 / 65534 powers of two, a share by
ln 2 times that, 8e-4; with two temperatures half as many cover them, 1.6e-3.  E, with u = 2^-24: the sum of the exponentials, (vocab / 8 + 64) u; the roundings of z,
of the logarithm and of their multiples, 16 u of each, over the temperature.  Shares below 2^-120 need not be there.
"""
import numpy as np
import pytest

from oracle import lm
from test_cpu_lm import _narrow, _wide, driver, pytestmark  # noqa: F401

B, U = 2.0 ** -8, 2.0 ** -24
# labels?, the teacher's temperature (None: no teacher)
TERMS = [(True, None), (True, 0.25), (True, 0.5), (True, 1.0), (True, 2.0), (True, 4.0), (True, 16.0), (False, 0.25), (False, 1.0), (False, 16.0)]


def case(rows, vocab, label, tau, far, seed):
    """Inputs as stored and as values: normal logits of a deviation of 3, one to three of every 64 about `far` below them."""
    rng = np.random.default_rng(seed)
    z = 3 * rng.standard_normal((vocab, rows))
    for at in range(0, vocab, 64):
        for t in range(rows):
            z[at + rng.permutation(min(64, vocab - at))[: rng.integers(1, 4)], t] -= far * (0.3 + 0.7 * rng.random())
    stored = {"X": _narrow(np.eye(rows), "bf16"), "W": _narrow(z, "bf16")}
    if label:
        stored["label"] = rng.integers(0, vocab, rows).astype(np.int64)
        stored["dlabel"] = (0.5 + rng.random(rows)).astype(np.float32)
    if tau:
        stored["top_id"] = rng.integers(0, vocab, (rows, 2)).astype(np.int64)
        stored["top_logit"] = rng.standard_normal((rows, 2)).astype(np.float32)
        stored["dtop"] = (0.5 + rng.random(rows)).astype(np.float32)
    return stored


def check(stored, dW, tau, rounding=B):
    """dW: as float64.  rounding: of the gradient in the logits before it is multiplied."""
    W = _wide(stored["W"], "bf16")
    vocab, rows = W.shape
    label, ids = stored.get("label"), stored.get("top_id")
    o = lm.vocab_loss(np.eye(rows), W, label, ids, stored.get("top_logit"), tau or 1.0, stored.get("dlabel"), stored.get("dtop"))
    z, size, E = W.T, np.zeros((rows, vocab)), np.zeros((rows, vocab))

    def term(weight, temperature, entries):
        lp = lm._log_softmax(z / temperature)
        part = weight[:, None] * np.exp(lp)
        of_all = np.abs(z / temperature - lp)                       # the logarithm of the sum
        E[:] += part * ((vocab / 8 + 64) * U + 16 * U * (np.abs(z / temperature) + of_all))
        size[:] += part + weight[:, None] * entries

    if label is not None:
        term(stored["dlabel"].astype(np.float64) * (label >= 0), 1.0, np.eye(vocab)[label % vocab])
    if tau:
        term(stored["dtop"].astype(np.float64) / tau, tau, lm.teacher(ids, stored["top_logit"], vocab, tau)[0])
    steps = 1.6e-3 if label is not None and tau and tau != 1.0 else 8e-4
    off = np.abs(dW.T - o["dz"]) - ((rounding + steps) * size + E + B * np.abs(o["dz"]) + 2.0 ** -120)
    t, v = np.unravel_index(off.argmax(), off.shape)
    assert off.max() <= 0, f"row {t} column {v}: {dW[v, t]:.6e}, exactly {o['dz'][t, v]:.6e}, made of {size[t, v]:.6e}; {(off > 0).sum()} entries"


@pytest.mark.parametrize("label,tau", TERMS)
@pytest.mark.parametrize("rows,vocab", [(5, 200), (40, 130)])
@pytest.mark.parametrize("far", [0.0, 40.0, 300.0, 3000.0, 1e30])
def test_every_entry(driver, rows, vocab, label, tau, far):  # noqa: F811
    stored = case(rows, vocab, label, tau, far, rows)
    numbers = dict(rows=rows, d=rows, vocab=vocab, ntop=2 if tau else 0, tau=tau or 1.0, dtype=1)
    got = driver("vocab_backward", numbers, stored, {"dX": ((rows, rows), "bf16"), "dW": ((vocab, rows), "bf16")})
    check(stored, got["dW"], tau)


def unlabelled(stored, share):
    """Some of the rows without a label: the others are closed up, and their second numbers lie behind those that are there."""
    rows = stored["label"].shape[0]
    stored["label"][[t for t in range(rows) if (t * 7) % 10 < 10 * share]] = -100
    return stored


@pytest.mark.parametrize("rows,vocab,label,tau,share", [(1, 70, True, None, 0.0), (32, 100, True, 2.0, 0.0), (33, 130, True, None, 0.0), (64, 70, False, 0.5, 0.0),
                                                        (65, 200, True, 4.0, 0.0), (100, 64, True, None, 0.6), (128, 96, True, None, 0.0), (128, 80, True, None, 0.8),
                                                        (200, 70, True, None, 0.6)])
def test_two_numbers(driver, rows, vocab, label, tau, share):  # noqa: F811
    """Up to 128 rows with a term hold the gradient in the logits as two bf16 numbers: every entry with the second number's rounding, 2^-8 of what the
    first's (2^-8) left, in the place of the first's."""
    stored = case(rows, vocab, label, tau, 0.0, rows)
    if share:
        unlabelled(stored, share)
    numbers = dict(rows=rows, d=rows, vocab=vocab, ntop=2 if tau else 0, tau=tau or 1.0, dtype=1)
    got = driver("vocab_backward", numbers, stored, {"dX": ((rows, rows), "bf16"), "dW": ((vocab, rows), "bf16")})
    check(stored, got["dW"], tau, rounding=B * B)
