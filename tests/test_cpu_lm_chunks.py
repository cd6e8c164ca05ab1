"""The vocabulary loss in several chunks of rows, without a GPU: the host build of tests/test_cpu_lm.py with chunks of the fewest rows that the
library takes (256 rows in bf16, 64 in fp32), so that small calls have two to five of them, the last one shorter or without a listed row."""
import pytest

import test_cpu_lm
from test_cpu_lm import driver, pytestmark, vocab_case  # noqa: F401

LIMITS = ("kChunkCodes = 1L << 31", "kChunkLogits = 1L << 28")


@pytest.fixture(scope="module", autouse=True)
def smallest_chunks():
    """The limits of a chunk's logits lowered in the sources that `driver` builds (set up behind this fixture) for this module."""
    found, plain = set(), test_cpu_lm._host_source

    def lowered(text):
        for limit in LIMITS:
            if limit in text:
                found.add(limit)
                text = text.replace(limit, limit.split("=")[0] + "= 1")
        return plain(text)

    with pytest.MonkeyPatch.context() as mp:
        mp.setattr(test_cpu_lm, "_host_source", lowered)
        yield found


# up to 1024 labelled rows, or 256 with a teacher, are listed by the launch that gathers them, more by one of their own
@pytest.mark.parametrize("rows,d,vocab,dtype,ignored", [(66, 4, 130, "f32", 0.0), (200, 20, 70, "f32", 0.2), (150, 8, 33, "f32", 0.7), (1030, 4, 40, "f32", 0.3),
                                                        (300, 40, 100, "bf16", 0.0), (600, 32, 70, "bf16", 0.2), (700, 33, 64, "bf16", 0.7),
                                                        (1100, 16, 50, "bf16", 0.3)])
def test_labels(driver, smallest_chunks, rows, d, vocab, dtype, ignored):  # noqa: F811
    assert smallest_chunks == set(LIMITS)
    vocab_case(driver, rows, d, vocab, dtype, ignored=ignored, seed=rows)


@pytest.mark.parametrize("rows,d,vocab,dtype,label", [(100, 24, 90, "f32", False), (129, 12, 300, "f32", True), (260, 8, 50, "f32", True), (256, 16, 64, "bf16", True),
                                                      (513, 24, 90, "bf16", True), (300, 48, 130, "bf16", False)])
def test_teacher(driver, rows, d, vocab, dtype, label):  # noqa: F811
    vocab_case(driver, rows, d, vocab, dtype, top=3, tau=2.0, label=label, ignored=0.4, seed=rows)
