"""Up to 128 rows with a term hold the gradient in the logits of bf16 storage as two bf16 numbers, on the host build of tests/test_cpu_lm.py: every entry, as in
tests/test_cpu_lm_far_logits.py, with the second number's rounding, 2^-8 of what the first's (2^-8) left, in the place of the first's."""
import pytest

from test_cpu_lm import driver, pytestmark  # noqa: F401
from test_cpu_lm_far_logits import B, case, check


def unlabelled(stored, share):
    """Some of the rows without a label: the others are closed up, and their second numbers lie behind those that are there."""
    rows = stored["label"].shape[0]
    stored["label"][[t for t in range(rows) if (t * 7) % 10 < 10 * share]] = -100
    return stored


@pytest.mark.parametrize("rows,vocab,label,tau,share", [(1, 70, True, None, 0.0), (32, 100, True, 2.0, 0.0), (33, 130, True, None, 0.0), (64, 70, False, 0.5, 0.0),
                                                        (65, 200, True, 4.0, 0.0), (100, 64, True, None, 0.6), (128, 96, True, None, 0.0), (128, 80, True, None, 0.8), (200, 70, True, None, 0.6)])
def test_every_entry(driver, rows, vocab, label, tau, share):  # noqa: F811
    stored = case(rows, vocab, label, tau, 0.0, rows)
    if share:
        unlabelled(stored, share)
    numbers = dict(rows=rows, d=rows, vocab=vocab, ntop=2 if tau else 0, tau=tau or 1.0, dtype=1)
    got = driver("vocab_backward", numbers, stored, {"dX": ((rows, rows), "bf16"), "dW": ((vocab, rows), "bf16")})
    check(stored, got["dW"], tau, rounding=B * B)
