"""Calls of the embedding, the norms and rotation of queries and keys, and attention with decay that ask for a part of the outputs, come in many steps or lie at the
ends of what is allowed, without a GPU (as tests/test_cpu_seq.py)."""
import itertools

import numpy as np
import pytest

from oracle import seq
from seq_cases import decay_case, decay_check, embed_case, head_case, narrow, walk_bound, walk_case, wide
from test_cpu_seq import driver, pytestmark, run_decay  # noqa: F401

HEAD_GRADS = ("dQ", "dK", "dw_q", "dw_k")


@pytest.mark.parametrize("t,d,rot,adjacent", [("bf16", 64, 64, 0), ("f32", 50, 20, 1)])
def test_any_set_of_head_gradients(driver, t, d, rot, adjacent):  # noqa: F811
    """Every set of outputs has the bits of the call that asks for all of them: 70 heads, so that all wavefronts of a workgroup have some, weights of queries unlike
    those of keys."""
    rows, heads = 3, 70
    c = head_case(rows, heads, heads, d, t, seed=1)
    numbers = dict(rows=rows, heads=heads, kv_heads=heads, d=d, rot=rot, ld_q=heads * d, ld_k=heads * d, ld_qout=heads * d, ld_kout=heads * d, base=10000.0,
                   dtype=int(t == "bf16"), flags=0x800 | 0x2000 * adjacent)
    shapes = {"dQ": ((rows, heads, d), t), "dK": ((rows, heads, d), t), "dw_q": ((d,), "f32"), "dw_k": ((d,), "f32")}
    full = driver("head_backward", numbers, c, shapes)
    for n in range(1, 4):
        for some in itertools.combinations(HEAD_GRADS, n):
            got = driver("head_backward", numbers, c, {k: shapes[k] for k in some})
            assert all(np.array_equal(got[k], full[k]) for k in some), some


@pytest.mark.parametrize("step,length", [(1, 3000), (6, 6000)])
def test_decay_token_by_token_for_long(driver, step, length):  # noqa: F811
    """States after thousands of tokens, a few a call: lambda's own rounding, which has the same sign at each token, is not in them."""
    s, want = walk_case(length, 8, 8)
    numbers = dict(rows=length, sequences=1, length=length, heads=3, kv_heads=3, dk=8, dv=8, seq_step=step, token_step=1, ld_q=24, ld_k=24, ld_v=24, ld_o=24, scale=1.0,
                   dtype=0, in_place=1, step=step)
    got = driver("decay_forward", numbers, s, {"O": ((length, 3, 8), "f32"), "state_out": ((1, 3, 8, 8), "f32")})["state_out"][0]
    off = np.linalg.norm(got - want, axis=(1, 2)) / np.linalg.norm(want, axis=(1, 2))
    assert (off <= walk_bound(length, 2)).all(), off


def test_decay_in_short_calls_for_long(driver):  # noqa: F811
    """The same where a call has one chunk: 2500 calls of 8 tokens, sums of 32 products (24 of them zeros) and a product by lambda^8 a call."""
    step, calls = 8, 2500
    s, want = walk_case(step * calls, 8, 8)
    numbers = dict(rows=step * calls, sequences=1, length=step * calls, heads=3, kv_heads=3, dk=8, dv=8, seq_step=step, token_step=1, ld_q=24, ld_k=24, ld_v=24, ld_o=24, scale=1.0,
                   dtype=0, in_place=1, step=step)
    got = driver("decay_forward", numbers, s, {"O": ((step * calls, 3, 8), "f32"), "state_out": ((1, 3, 8, 8), "f32")})["state_out"][0]
    off = np.linalg.norm(got - want, axis=(1, 2)) / np.linalg.norm(want, axis=(1, 2))
    assert (off <= walk_bound(calls, 9)).all(), (off, walk_bound(calls, 9))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("length", [5, 20, 40, 70])
def test_decay_of_a_state_alone(driver, length, t):  # noqa: F811
    """Keys and queries of zeros: states and their gradients fade by lambda^length, however little of them is left (half a step for each chunk's product, each rounding of
    lambda^n, and what these begin with)."""
    s = decay_case(length, 1, 9, 9, 20, 36, t, seed=2)
    s["K"][:], s["Q"][:] = 0, 0
    s["log_decay"][-1] = -1.0
    left = np.exp(length * s["log_decay"].astype(np.float64))[:, None, None]
    for grads, n, was in ((False, "state", "state"), (True, "dstate", "dstate_out")):
        got = run_decay(driver, s, t, grads, length, 1, length, 9, 9, 20, 36, length, 1)[n]
        assert (np.abs(got - left * s[was]) <= (length // 32 * 3 + 6) * 2.0 ** -24 * left * np.abs(s[was])).all()


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("scale,up,after", [(2.0 ** -100, 2.0 ** 60, 2.0 ** 60), (2.0 ** 100, 2.0 ** -60, 2.0 ** -60), (1e-30, 1.0, 1e9), (1e30, 1e-30, 1e-12)])
def test_decay_gradients_of_scales_far_from_one(driver, scale, up, after, t):  # noqa: F811
    """The state's gradient is held as the formula has it: neither it nor what is handed in is divided by the scale."""
    s = decay_case(70, 1, 2, 1, 20, 36, t, seed=3)
    s["dO"], s["dstate_out"] = narrow(wide(s["dO"], t) * up, t), (s["dstate_out"].astype(np.float64) * after).astype(np.float32)
    at = [list(range(70))]
    got = run_decay(driver, s, t, True, 70, 1, 70, 2, 1, 20, 36, 70, 1, scale=scale)
    decay_check(got, s, at, t, float(np.float32(scale)), 70, ("dQ", "dK", "dV", "dstate"))


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_decay_gradients_of_states_without_tokens_pass_through(driver, t):  # noqa: F811
    """Sequences without tokens: the same bits, whatever the scale; states alike."""
    s = decay_case(40, 3, 2, 1, 20, 36, t, seed=4)
    offset = np.array([0, 0, 40, 40], np.int64)
    got = run_decay(driver, s, t, True, 40, 3, 40, 2, 1, 20, 36, 0, 0, offset, scale=0.7)
    assert all(np.array_equal(got["dstate"][b], s["dstate_out"][b]) for b in (0, 2))
    got = run_decay(driver, s, t, False, 40, 3, 40, 2, 1, 20, 36, 0, 0, offset, scale=0.7)
    assert all(np.array_equal(got["state"][b], s["state"][b]) for b in (0, 2))


@pytest.mark.parametrize("dk,dv", [(1, 256), (256, 1), (129, 129), (128, 128), (33, 97)])
@pytest.mark.parametrize("length", [1, 7])
def test_decay_launches_of_the_most_heads(driver, monkeypatch, tmp_path, length, dk, dv):  # noqa: F811
    """As many heads of all sequences as are allowed: no launch has more threads than 32 bits count in a dimension, and together they have every workgroup."""
    most, t = 4194304, "bf16"
    s = {k: np.zeros((length, w), np.uint16) for k, w in (("Q", dk), ("K", dk), ("V", dv), ("dO", dv))}
    s.update(log_decay=None, state=None, dstate_out=None)
    offset = np.full(most + 1, length, np.int64)
    offset[0] = 0
    numbers = dict(rows=length, sequences=most, length=length, heads=1, kv_heads=1, dk=dk, dv=dv, seq_step=0, token_step=0, ld_q=dk, ld_k=dk, ld_v=dv, ld_o=dv, scale=1.0, dtype=1)
    inputs = {"offset": offset, **{k: s[k] for k in ("Q", "K", "V", "dO")}}
    for call, outs in (("decay_forward", {"O": dv}), ("decay_backward", {"dQ": dk, "dK": dk, "dV": dv})):
        to = tmp_path / call
        monkeypatch.setenv("STL_LAUNCHES", str(to))
        driver(call, numbers, inputs, {k: ((length, w), t) for k, w in outs.items()})
        launches = [ln.split(maxsplit=4) for ln in to.read_text().splitlines()]
        assert all(int(x) * int(threads) < 1 << 32 and int(y) < 1 << 16 and int(z) < 1 << 16 for x, y, z, threads, _ in launches), launches
        groups = sum(int(x) * int(y) for x, y, z, threads, _ in launches)
        if call == "decay_backward":
            blocks = sum(-(-w // 128) for w in (dk, dk, dv))
        else:
            blocks = -(-dv // (32 if length == 1 and dv <= 96 else 128))
        assert groups == most * blocks, launches


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [np.inf, np.nan])
def test_embed_rows_without_a_token_are_zeros_whatever_the_scale(driver, scale, t):  # noqa: F811
    rows, d, vocab = 40, 21, 30
    c = embed_case(rows, d, vocab, t, seed=1, tokens="even")
    there = (c["token"] >= 0) & (c["token"] < vocab)
    numbers = dict(rows=rows, d=d, vocab=vocab, scale=scale, dtype=int(t == "bf16"), accumulate=0)
    got = driver("embed_forward", numbers, {k: c[k] for k in ("token", "W")}, {"X": ((rows, d), t)})["X"]
    assert not there.all() and not got[~there].any() and not np.isfinite(got[there]).any()
    got = driver("embed_backward", numbers, {k: c[k] for k in ("token", "dX")}, {"dW": ((vocab, d), t)})["dW"]
    absent = np.setdiff1d(np.arange(vocab), c["token"])
    assert len(absent) and not got[absent].any() and not np.isfinite(np.delete(got, absent, 0)).any()


@pytest.mark.parametrize("sequences,length,seq_step,token_step,rows", [(1, 5, 10, 2, 9), (1, 20, 1 << 40, 3, 58), (3, 1, 2, 100, 5), (2, 1, 1, 1 << 50, 2), (1, 1, -7, -7, 1)])
def test_decay_distances_that_no_token_has_are_not_checked(driver, sequences, length, seq_step, token_step, rows):  # noqa: F811
    """From sequence to sequence where there is one, from token to token where a sequence has one."""
    s = decay_case(rows, sequences, 2, 1, 8, 12, "f32", seed=length)
    at = seq.decay_rows(sequences, length, seq_step, token_step)
    for grads, names in ((False, ("O", "state")), (True, ("dQ", "dK", "dV", "dstate"))):
        got = run_decay(driver, s, "f32", grads, rows, sequences, length, 2, 1, 8, 12, seq_step, token_step)
        decay_check(got, s, at, "f32", 0.7, length, names)
