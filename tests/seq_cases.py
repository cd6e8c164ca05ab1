"""Inputs, oracle results and error bounds that the CPU and GPU tests of csrc_seq share.

Bounds.  An output is rounded to its type once, at most 2^-8 |O| for bf16 (2^-24 |O| for fp32).  Before it, sums are fp32: a chain of n additions, and the few
products in front of and behind it, is off by at most (n + 32) 2^-24 times the same expression on absolute values.  A two-part bf16 operand is off by
2^-16 of itself (a rounding of 2^-8, of what a rounding of 2^-8 leaves), a three-part one by 2^-24.  Chains: a norm adds d elements; the gradient of a weight
rows x heads; an angle position base^(-2 p / rot) has four roundings of 2^-53 in 64 bits, which turn a pair by 2^-50 |position| at most;
the embedding's gradient up to all rows; attention adds dk (or dv) products for an entry of P, and every token's part once to an output, with
one product by a decay for each chunk of 32 tokens or more.
"""
import numpy as np

from oracle import seq

EPS = 2.0 ** -24
UNIT = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def narrow(a, t):
    """values in the storage type (round to nearest even), as stored"""
    a = np.ascontiguousarray(a, np.float32)
    if t == "f32":
        return a
    u = a.view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def wide(a, t):
    return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64) if t == "bf16" else a.astype(np.float64)


def close(got, want, size, t, chain, name, operand=0.0, more=0.0):
    """chain: additions in fp32; operand: what operands are off by, relative to the same size; more: beside it."""
    off = np.abs(got - want) - (UNIT[t] * np.abs(want) + ((chain * EPS + operand) * size + more) * (1 + UNIT[t]))
    assert np.isfinite(got).all(), name
    assert off.max(initial=-1.0) <= 0, f"{name}: {off.max()} over the bound at {np.unravel_index(off.argmax(), off.shape)}"


def embed_case(rows, d, vocab, t, seed=0, scale=1.0, tokens="zipf"):
    rng = np.random.default_rng(seed)
    if tokens == "zipf":
        token = np.minimum((np.exp(rng.random(rows) * np.log(vocab + 1)) - 1).astype(np.int64), vocab - 1)
    elif tokens == "one":
        token = np.full(rows, vocab // 2, np.int64)
    else:
        token = rng.integers(0, vocab, rows).astype(np.int64)
    bad = rng.random(rows) < 0.1
    token = np.where(bad & (tokens != "one"), rng.choice([-100, -1, vocab, 2 ** 40, -2 ** 63], rows), token)
    return {"token": token, "W": narrow(rng.standard_normal((vocab, d)), t), "dX": narrow(rng.standard_normal((rows, d)), t)}


def head_case(rows, heads, kv_heads, d, t, seed=0, far=True):
    rng = np.random.default_rng(seed)
    x = {n: narrow(1.5 * rng.standard_normal((rows, k, d)) + 0.25, t) for n, k in (("Q", heads), ("K", kv_heads), ("dQout", heads), ("dKout", kv_heads))}
    x["w_q"], x["w_k"] = (narrow(1.0 + 0.3 * rng.standard_normal(d), t) for _ in range(2))
    x["position"] = rng.integers(-1000, 2_000_000 if far else 1000, rows).astype(np.int64)
    return x


def turn_error(position, y):
    """What the angles' roundings in 64 bits can make of heads y (rows, heads, d) in front of their rotation."""
    return 0.0 if position is None else 2.0 ** -50 * np.abs(position.astype(np.float64))[:, None, None] * 2 * np.abs(y).max(-1, keepdims=True)


def decay_case(rows, sequences, heads, kv_heads, dk, dv, t, seed=0, states=True, decays="spread"):
    rng = np.random.default_rng(seed)
    s = {"Q": narrow(rng.standard_normal((rows, heads, dk)) / np.sqrt(dk), t), "K": narrow(rng.standard_normal((rows, kv_heads, dk)), t),
         "V": narrow(rng.standard_normal((rows, kv_heads, dv)), t), "dO": narrow(rng.standard_normal((rows, heads, dv)), t), "log_decay": None, "state": None,
         "dstate_out": None}
    if decays == "spread":
        s["log_decay"] = np.log1p(-(2.0 ** -np.linspace(1, 9, heads))).astype(np.float32)
    elif decays == "none left":
        s["log_decay"] = np.full(heads, -np.inf, np.float32)
    elif decays is not None:
        s["log_decay"] = np.full(heads, decays, np.float32)
    if states:
        s["state"], s["dstate_out"] = (rng.standard_normal((sequences, heads, dk, dv)).astype(np.float32) for _ in range(2))
    return s


def decay_chain(length, dk, dv):
    """Additions behind an output: an entry of P, then all tokens, and the state's (or the gradients') second contraction."""
    return length + 2 * max(dk, dv) + 2 * (length // 32)


def decay_bounds(name, t):
    """(storage type of the output, what its operands are off by): P and the state are given in two parts, what goes into a state in three."""
    if t == "f32":
        return "f32", 0.0
    return ("f32", 2 * 2.0 ** -24) if name in ("state", "dstate") else ("bf16", 2 * 2.0 ** -16)


def decay_check(got, s, rows_of, t, scale, length, names):
    v = {k: wide(s[k], t) for k in ("Q", "K", "V", "dO")}
    grads = any(n.startswith("d") for n in names)
    want = seq.decay(v["Q"], v["K"], v["V"], rows_of, s["log_decay"], scale, s["state"], v["dO"] if grads else None, s["dstate_out"] if grads else None)
    dk, dv = v["Q"].shape[2], v["V"].shape[2]
    covered = np.zeros(v["Q"].shape[0], bool)
    for r in rows_of:
        covered[r] = True
    share = v["Q"].shape[1] // v["K"].shape[1]
    for n in names:
        kind, operand = decay_bounds(n, t)
        g, w, z = got[n], want[n], want["size"][n]
        if n not in ("state", "dstate"):
            g, w, z = g[covered], w[covered], z[covered]
        close(g, w, z, kind, decay_chain(length, dk, dv) + 32 + share, n, operand)
    return want, covered


def walk_case(length, dk, dv):
    """One sequence of fp32 tokens, three heads whose decays last longer than it does and whose lambda is off in fp32 by about as much as it can be, and the state behind
    the last token in 64 bits."""
    rng = np.random.default_rng(5)
    s = {"Q": rng.standard_normal((length, 3, dk)), "K": rng.standard_normal((length, 3, dk)), "V": rng.standard_normal((length, 3, dv)),
         "state": rng.standard_normal((1, 3, dk, dv)) * np.sqrt(length)}
    s = {k: v.astype(np.float32) for k, v in s.items()}
    near = -np.linspace(1e-5, 1e-4, 30000).astype(np.float32)
    off = np.exp(near.astype(np.float64))
    off = np.abs(off.astype(np.float32).astype(np.float64) - off)
    s["log_decay"] = np.array([near[at][off[at].argmax()] for at in np.array_split(np.arange(near.size), 3)])
    lam, state = np.exp(s["log_decay"].astype(np.float64))[:, None, None], s["state"][0].astype(np.float64)
    for k, v in zip(s["K"].astype(np.float64), s["V"].astype(np.float64)):
        state = lam * state + k[:, :, None] * v[:, None, :]
    return s, state


def walk_bound(calls, roundings):
    """Error of a state that is rounded to fp32 so many times in each of so many calls, relative to its norm.  A rounding is off by half a step at most, which is 2^-24 of the
    value at most and by 2^-24 0.42 in the root mean square (evenly spread significands and remainders); roundings of different calls are independent, so that
    n of them are off by 2^-24 0.42 sqrt(n), where what is rounded fades no faster than its error does, as here.  2^-24 sqrt(n) is more than twice that, of a norm over 64
    entries or more."""
    return 2.0 ** -24 * np.sqrt(calls * roundings)
