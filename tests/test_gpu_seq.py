"""GPU parity of the embedding, the norms and rotation of queries and keys, and attention with decay against the 64-bit oracle; bounds as in tests/seq_cases.py."""
import numpy as np
import pytest
import torch

import paper_2503_12211_amd as stl
from gpu_util import STL_DT, TORCH_DT, Guard
from oracle import seq
from seq_cases import close, decay_case, decay_check, embed_case, head_case, turn_error, wide

pytestmark = pytest.mark.gpu
PRE, ADJ = stl.STL_FLAG_PRE_NORM, stl.STL_FLAG_ADJACENT


def up(a):
    """an array as stored (bf16 as its bits) on the GPU"""
    if a is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t.view(torch.bfloat16) if a.dtype == np.uint16 else t


def down(t):
    return t.double().cpu().numpy()


# ---- embedding --------------------------------------------------------------------------------------------------------------------

def embed(c, rows, d, vocab, t, scale=1.0, accumulate=None):
    """(X, dW) through the library; accumulate: what dW holds before"""
    prob, gd = stl.EmbedProblem(rows, d, vocab, scale, STL_DT[t]), Guard()
    token, W, dX = (up(c[k]) for k in ("token", "W", "dX"))
    X, dW = gd.alloc((rows, d), TORCH_DT[t]), gd.alloc((vocab, d), TORCH_DT[t])
    if accumulate is not None:
        dW.copy_(accumulate)
    n = stl.stl_embed_workspace_bytes(prob)
    ws = gd.alloc((n,), torch.uint8, fill=0xFF)
    stl.stl_embed_forward(prob, token, W, X)
    stl.stl_embed_backward(prob, token, dX, dW, int(accumulate is not None), ws, n)
    gd.check()
    return X, dW


def check_embed(rows, d, vocab, t, tokens="zipf", scale=1.0, seed=0):
    c = embed_case(rows, d, vocab, t, seed=seed, scale=scale, tokens=tokens)
    X, dW = embed(c, rows, d, vocab, t, scale)
    want = seq.embed_forward(c["token"], wide(c["W"], t), scale)
    close(down(X), want, np.abs(want), t, 0, "X")
    want = seq.embed_backward(c["token"], wide(c["dX"], t), vocab, scale)
    close(down(dW), want["dW"], want["size"]["dW"], t, rows + 32, "dW")
    was = torch.randn(vocab, d, device="cuda").to(TORCH_DT[t])
    _, more = embed(c, rows, d, vocab, t, scale, was)
    want = seq.embed_backward(c["token"], wide(c["dX"], t), vocab, scale, down(was))
    close(down(more), want["dW"], want["size"]["dW"], t, rows + 32, "dW added to")
    absent = torch.from_numpy(np.setdiff1d(np.arange(vocab), c["token"])).cuda()
    assert torch.equal(more[absent], was[absent]) and not dW[absent].any()
    for _ in range(2):
        assert torch.equal(embed(c, rows, d, vocab, t, scale)[1], dW)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 7, 8, 63, 64, 100, 513, 1021, 2048, 2056, 4100])
def test_embed_widths(d, t):
    check_embed(77, d, 130, t, seed=d, scale=1.5)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,tokens", [(1, 1, "even"), (1, 50001, "even"), (16, 3, "one"), (17, 257, "even"), (63, 1000, "zipf"), (64, 2, "even"), (1000, 1, "one"),
                                               (1025, 255, "zipf"), (3001, 50001, "zipf"), (4096, 32000, "one"), (20000, 256, "zipf"), (70000, 500, "zipf")])
def test_embed_rows_and_vocabularies(rows, vocab, tokens, t):
    check_embed(rows, 24, vocab, t, tokens, seed=rows)


def test_embed_runs_of_many_segments():
    """One id's rows over more segments than a wavefront looks ahead, wide rows and narrow ones."""
    check_embed(30000, 40, 7, "bf16", "one")
    check_embed(5000, 700, 3, "f32", "even")
    check_embed(33000, 2050, 11, "bf16", "zipf")


def test_embed_more_elements_than_32_bits_count():
    vocab, d, rows = 1100000, 2048, 40
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough free memory")
    token = torch.arange(vocab - rows, vocab, device="cuda")
    prob = stl.EmbedProblem(rows, d, vocab)
    W = torch.zeros((vocab, d), dtype=torch.bfloat16, device="cuda")
    W[-rows:] = torch.randn(rows, d, device="cuda")
    X = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda")
    stl.stl_embed_forward(prob, token, W, X)
    assert torch.equal(X, W[-rows:])
    n = stl.stl_embed_workspace_bytes(prob)
    dW = torch.full_like(W, float("nan"))
    stl.stl_embed_backward(prob, token, X, dW, 0, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    assert torch.equal(dW[-rows:], X) and not dW[:-rows].any()


def test_embed_without_rows():
    prob = stl.EmbedProblem(0, 16, 20)
    stl.stl_embed_forward(prob, None, None, None)
    dW = torch.ones((20, 16), dtype=torch.bfloat16, device="cuda")
    stl.stl_embed_backward(prob, None, None, dW, 1)
    assert bool((dW == 1).all())
    stl.stl_embed_backward(prob, None, None, dW, 0)
    assert not dW.any()


# ---- heads ------------------------------------------------------------------------------------------------------------------------

def check_heads(rows, heads, kv, d, rot, t, adjacent=False, norm=True, weights=True, position=True, fused=False, in_place=False, seed=0):
    """fused: queries and keys are parts of the rows of one matrix, which has other things between them"""
    c = head_case(rows, heads, kv, d, t, seed=seed)
    flags = (PRE if norm else 0) | (ADJ if adjacent else 0)
    w = {n: c["w_" + n.lower()] if weights else None for n in "QK"}
    g = {k: up(v) for k, v in c.items()}
    wide_q, wide_k = heads * d, kv * d
    ld = wide_q + wide_k + 3 if fused else None
    prob = stl.HeadNormProblem(rows, heads, kv, d, rot, *([ld] * 4 if fused else [None] * 4), dtype=STL_DT[t])

    def pair(q, k):
        """two matrices, or parts of one, and the latter"""
        if not fused:
            return q, k, None
        both = torch.full((rows, ld), 7.0, dtype=q.dtype, device="cuda")
        both[:, 1:1 + wide_q], both[:, 2 + wide_q:2 + wide_q + wide_k] = q.reshape(rows, -1), k.reshape(rows, -1)
        return both[:, 1:], both[:, 2 + wide_q:], both

    def take(q, k, both):
        return (q[:, :wide_q].reshape(rows, heads, d), k[:, :wide_k].reshape(rows, kv, d)) if fused else (q, k)

    gd = Guard()
    new = lambda: pair(*(gd.alloc((rows, n, d), TORCH_DT[t], fill=0.0) for n in (heads, kv)))  # noqa: E731
    x, wq, wk, at = pair(g["Q"], g["K"]), up(w["Q"]), up(w["K"]), g["position"] if position else None
    given = [v.clone() for v in take(*x)]
    out = x if in_place else new()
    stl.stl_head_norm_forward(prob, x[0], x[1] if kv else None, wq, wk, at, out[0], out[1] if kv else None, flags)
    gd.check()
    kw = dict(position=c["position"] if position else None, rot=rot, adjacent=adjacent, norm=norm)
    for n, v in zip("QK"[:2 if kv else 1], take(*out)):
        want, size = seq.head_forward(wide(c[n], t), wide(w[n], t) if weights and norm else None, **kw)
        close(down(v), want, size, t, d + 32, n, more=turn_error(kw["position"], want))
    if fused:
        assert bool((out[2][:, 0] == 7).all()) and bool((out[2][:, 1 + wide_q] == 7).all()) and bool((out[2][:, -1] == 7).all())
    x, ups = pair(*given), pair(g["dQout"], g["dKout"])
    dx = ups if in_place else new()
    dw = [gd.alloc((d,), torch.float32) if norm else None for _ in range(2)]
    n_ws = stl.stl_head_norm_workspace_bytes(prob, flags)
    ws = gd.alloc((n_ws,), torch.uint8, fill=0xFF)
    run = lambda dx, dw, accumulate=0: stl.stl_head_norm_backward(  # noqa: E731
        prob, x[0], x[1] if kv else None, wq, wk, at, ups[0], ups[1] if kv else None, dx[0], dx[1] if kv else None, dw[0], dw[1] if kv else None, accumulate, ws, n_ws, flags)
    run(dx, dw)
    gd.check()
    for i, n in enumerate("QK"[:2 if kv else 1]):
        want = seq.head_backward(wide(c[n], t), wide(c[f"d{n}out"], t), wide(w[n], t) if weights and norm else None, **kw)
        close(down(take(*dx)[i]), want["dx"], want["size"]["dx"], t, 2 * d + 64, "d" + n, more=turn_error(kw["position"], want["size"]["dx"]))
        if norm:
            close(down(dw[i]), want["dw"], want["size"]["dw"], "f32", rows * (heads, kv)[i] + d + 64, "dw_" + n)
    if in_place or not norm:
        return
    again, added = new(), [torch.full_like(v, 2.0) for v in dw]
    run(again, added, 1)
    assert all(torch.equal(a, b) for a, b in zip(take(*again), take(*dx)))
    for i in range(2 if kv else 1):
        assert torch.equal(added[i], dw[i] + 2.0)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot", [(1, 0), (2, 2), (3, 2), (8, 8), (16, 16), (31, 30), (48, 32), (50, 50), (64, 64), (64, 32), (80, 80), (96, 48), (128, 128), (160, 96), (255, 128),
                                   (256, 256), (512, 512), (1000, 10), (1024, 1024)])
def test_head_sizes(d, rot, t):
    check_heads(13, 3, 2, d, rot, t, seed=d)
    check_heads(5, 2, 1, d, rot, t, adjacent=True, fused=True, seed=d + 1)


@pytest.mark.parametrize("rows", [1, 2, 64, 1023, 2049, 4100, 8200])
@pytest.mark.parametrize("heads,kv", [(1, 0), (8, 2)])
def test_head_rows(rows, heads, kv):
    check_heads(rows, heads, kv, 64, 64, "bf16", seed=rows)
    check_heads(rows, heads, kv, 32, 16, "f32", adjacent=True, seed=rows)


@pytest.mark.parametrize("rows,heads,kv,d,rot", [(16500, 12, 12, 64, 32), (16500, 3, 1, 32, 32), (8300, 5, 1, 96, 96), (40000, 1, 1, 16, 16)])
def test_head_turns_of_many_rows(rows, heads, kv, d, rot):
    """More rows than workgroups take at once, heads that leave lanes idle."""
    check_heads(rows, heads, kv, d, rot, "bf16", adjacent=rot < d, seed=rows)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_head_parts_left_out(t, adjacent):
    for norm in (True, False):
        for position in (True, False):
            check_heads(9, 3, 2, 96, 64, t, adjacent, norm, weights=not position, position=position, seed=3)
    check_heads(33, 3, 2, 64, 64, t, adjacent, fused=True, in_place=True, seed=4)
    check_heads(33, 3, 2, 50, 20, t, adjacent, in_place=True, seed=5)


def test_head_without_rows():
    prob = stl.HeadNormProblem(0, 2, 1, 16)
    stl.stl_head_norm_forward(prob, None, None, None, None, None, None, None, PRE)
    dw = torch.ones(16, device="cuda")
    stl.stl_head_norm_backward(prob, None, None, None, None, None, None, None, None, None, dw, None, 1, None, 0, PRE)
    assert bool((dw == 1).all())
    stl.stl_head_norm_backward(prob, None, None, None, None, None, None, None, None, None, dw, None, 0, None, 0, PRE)
    assert not dw.any()


def test_head_gradients_that_are_not_there():
    """A missing upstream gradient stands for zeros; outputs that are not asked for change nothing."""
    c = {k: up(v) for k, v in head_case(20, 3, 2, 64, "bf16").items()}
    prob = stl.HeadNormProblem(20, 3, 2, 64)
    n = stl.stl_head_norm_workspace_bytes(prob, PRE)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def run(dq_up, dk_up, want):
        out = {k: torch.empty_like(c[k[1:]]) if k in ("dQ", "dK") else torch.empty(64, device="cuda") for k in want}
        stl.stl_head_norm_backward(prob, c["Q"], c["K"], c["w_q"], c["w_k"], c["position"], dq_up, dk_up, *(out.get(k) for k in ("dQ", "dK", "dw_q", "dw_k")), 0, ws, n, PRE)
        return out

    every = ("dQ", "dK", "dw_q", "dw_k")
    full = run(c["dQout"], c["dKout"], every)
    half = run(c["dQout"], None, every)
    assert torch.equal(half["dQ"], full["dQ"]) and torch.equal(half["dw_q"], full["dw_q"]) and not half["dK"].any() and not half["dw_k"].any()
    for k in every:
        assert torch.equal(run(c["dQout"], c["dKout"], (k,))[k], full[k]), k


def test_a_rotation_of_a_head_that_is_no_number_stays_there():
    c = head_case(6, 2, 1, 48, "f32")
    prob, outs = stl.HeadNormProblem(6, 2, 1, 48, 20, dtype=stl.STL_F32), []
    for value in (0.5, float("inf"), float("nan")):
        g = {k: up(v) for k, v in c.items()}
        g["Q"][2, 1, 47] = value                                       # behind what is turned, in a pair with element 46
        Qout, Kout = torch.empty_like(g["Q"]), torch.empty_like(g["K"])
        stl.stl_head_norm_forward(prob, g["Q"], g["K"], None, None, g["position"], Qout, Kout, 0)
        outs.append(Qout)
    keep = torch.ones_like(outs[0], dtype=torch.bool)
    keep[2, 1, 47] = False
    assert torch.equal(outs[0][keep], outs[1][keep]) and torch.equal(outs[0][keep], outs[2][keep])


# ---- attention --------------------------------------------------------------------------------------------------------------------

def strided(x, extra):
    """The same rows, `extra` elements further apart and one element off"""
    rows, wide_ = x.shape[0], x[0].numel()
    m = torch.full((rows, wide_ + extra), float("nan"), dtype=x.dtype, device="cuda")
    m[:, 1:1 + wide_] = x.reshape(rows, -1)
    return m[:, 1:], m


def decay_problem(s, t, at, scale, extra=0):
    q, k, v = s["Q"].shape, s["K"].shape, s["V"].shape
    ld = [w[1] * w[2] + extra if extra else None for w in (q, k, v, (0, q[1], v[2]))]
    return stl.DecayAttentionProblem(q[0], at["sequences"], at["length"], q[1], k[1], q[2], v[2], at.get("seq_step"), at.get("token_step", 1), *ld, scale=scale, dtype=STL_DT[t])


def decay_run(s, t, at, scale=0.7, extra=0, grads=True, in_place=False, ws_fill=0xFF):
    """dict of the library's outputs on the GPU; rows of no sequence keep the NaN that they held"""
    prob, gd = decay_problem(s, t, at, scale, extra), Guard()
    offset = up(at.get("offset"))
    g = {k: up(s[k]) for k in ("Q", "K", "V", "dO", "log_decay", "state", "dstate_out")}
    a = {k: strided(g[k], extra)[0] if extra else g[k] for k in ("Q", "K", "V", "dO")}
    shape = {"O": g["dO"].shape, "dQ": g["Q"].shape, "dK": g["K"].shape, "dV": g["V"].shape}
    raw = {}

    def out(n):
        rows, w = shape[n][0], int(np.prod(shape[n][1:]))
        raw[n] = gd.alloc((rows, w + extra), TORCH_DT[t])
        return raw[n].view(-1)[1:] if extra else raw[n]

    def got(n):
        w = int(np.prod(shape[n][1:]))
        if extra:
            flat = raw[n].view(-1)
            assert bool(torch.isnan(flat[0])), n
            body = flat[1:1 + (shape[n][0] - 1) * (w + extra) + w]
            return body.as_strided((shape[n][0], w), (w + extra, 1)).reshape(shape[n])
        return raw[n].view(shape[n])

    state_shape = (at["sequences"], s["Q"].shape[1], s["Q"].shape[2], s["V"].shape[2])
    after = gd.alloc(state_shape, torch.float32)
    before = g["state"]
    if in_place and before is not None:
        after.copy_(before)
        before = after
    n = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_FORWARD)
    ws = gd.alloc((max(n, 16),), torch.uint8, fill=ws_fill)
    stl.stl_decay_attention_forward(prob, a["Q"], a["K"], a["V"], g["log_decay"], offset, before, out("O"), after, ws, n)
    gd.check()
    r = {"O": got("O"), "state": after}
    if grads:
        dstate = gd.alloc(state_shape, torch.float32)
        n = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
        ws = gd.alloc((max(n, 16),), torch.uint8, fill=ws_fill)
        stl.stl_decay_attention_backward(prob, a["Q"], a["K"], a["V"], g["log_decay"], offset, g["state"], a["dO"], g["dstate_out"], out("dQ"), out("dK"), out("dV"), dstate, ws, n)
        gd.check()
        r.update({k: got(k) for k in ("dQ", "dK", "dV")}, dstate=dstate)
    return r


ALL = ("O", "state", "dQ", "dK", "dV", "dstate")


def check_decay(sequences, length, heads, kv, dk, dv, t, at=None, rows=None, extra=0, seed=0, scale=0.7, in_place=False, **kw):
    at = dict(dict(sequences=sequences, length=length), **(at or {}))
    rows = rows or sequences * length
    s = decay_case(rows, sequences, heads, kv, dk, dv, t, seed=seed, **kw)
    got = decay_run(s, t, at, scale, extra, in_place=in_place)
    where = seq.decay_rows(sequences, length, at.get("seq_step", length), at.get("token_step", 1), at.get("offset"), rows)
    want, covered = decay_check({k: down(v) for k, v in got.items()}, s, where, t, scale, length, ALL)
    assert all(bool(torch.isnan(got[n][torch.from_numpy(~covered).cuda()]).all()) for n in ("O", "dQ", "dK", "dV"))
    return s, at, got, want


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 700])
def test_decay_lengths(length, t):
    check_decay(2, length, 2, 2, 64, 64, t, seed=length)
    check_decay(1, length, 3, 1, 40, 72, t, seed=length + 1, states=False)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("dk", [1, 16, 31, 32, 33, 64, 65, 96, 128, 129, 256])
@pytest.mark.parametrize("dv", [1, 32, 50, 128, 130, 256])
def test_decay_widths(dk, dv, t):
    check_decay(1, 70, 2, 1, dk, dv, t, seed=dk + dv)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("length", [1, 5, 90])
def test_decay_rows_far_apart(length, t):
    check_decay(3, length, 4, 2, 48, 80, t, extra=7, seed=1)
    check_decay(4, length, 2, 2, 64, 32, t, dict(seq_step=1, token_step=5), rows=5 * length, extra=2, seed=2)
    check_decay(2, length, 2, 2, 64, 32, t, dict(seq_step=3 * length, token_step=2), rows=6 * length, seed=3)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_decay_packed(t):
    offset = np.array([2, 2, 130, 131, 400, 400, 433], np.int64)
    check_decay(6, 269, 4, 2, 64, 128, t, dict(offset=offset), rows=450, seed=1)
    check_decay(6, 269, 2, 2, 100, 60, t, dict(offset=offset), rows=433, extra=3, seed=2, in_place=True)
    check_decay(6, 100, 2, 2, 32, 32, t, dict(offset=offset), rows=433, seed=3)          # the longest is cut off
    single = np.array([0, 1, 1, 2, 3, 3, 4], np.int64)                                    # a serving step in which two of six have no token
    check_decay(6, 1, 4, 4, 64, 64, t, dict(offset=single), rows=4, seed=4, in_place=True)
    check_decay(3, 40, 2, 2, 32, 32, t, dict(offset=np.array([-9, 30, 30, 500], np.int64)), rows=60, seed=5)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("decays", [None, "none left", -1e-6, -0.7, -20.0, -3e38])
def test_decays(decays, t):
    check_decay(1, 150, 2, 2, 64, 96, t, decays=decays, seed=1)
    check_decay(3, 1, 2, 2, 64, 96, t, decays=decays, seed=2)


def test_decay_of_long_sequences():
    check_decay(1, 5000, 2, 1, 32, 40, "bf16", seed=1)
    check_decay(2, 2100, 2, 2, 64, 64, "f32", seed=2, decays=-0.0005)
    check_decay(3, 1000, 2, 2, 128, 128, "bf16", seed=3, decays=-0.002)


def test_decay_errors_are_one_roundings():
    """bf16: outputs are off by no more than what their own rounding costs (1.66e-3 of the norm in the mean over values with evenly spread logarithms), fp32 states by sums'."""
    for length in (64, 513):
        s, _, got, want = check_decay(2, length, 4, 4, 128, 128, "bf16", seed=length)
        for n in ALL:
            off = float(np.linalg.norm(down(got[n]) - want[n]) / np.linalg.norm(want[n]))
            assert off <= (1e-6 if n in ("state", "dstate") else 1.9e-3), (n, off)


def test_decay_goes_on_from_call_to_call():
    """A prompt in one call, in three parts, and token by token: the same outputs within two roundings, states within the sums'."""
    t, heads, dk, dv, length = "bf16", 3, 64, 80, 150
    s = decay_case(length, 1, heads, heads, dk, dv, t, seed=4)
    whole = decay_run(s, t, dict(sequences=1, length=length), grads=False)
    for cuts in ([0, 64, 65, length], list(range(length + 1))):
        state, parts = s["state"], []
        for lo, hi in zip(cuts[:-1], cuts[1:]):
            part = dict(s, state=state, **{n: s[n][lo:hi] for n in ("Q", "K", "V", "dO")})
            r = decay_run(part, t, dict(sequences=1, length=hi - lo), grads=False, in_place=True)
            state = r["state"].cpu().numpy()
            parts.append(r["O"])
        O = torch.cat(parts)
        assert float((O.double() - whole["O"].double()).norm() / whole["O"].double().norm()) <= 2.0 ** -7
        assert float((torch.from_numpy(state).cuda().double() - whole["state"].double()).norm() / whole["state"].double().norm()) <= 1e-6


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["Q", "K", "V"])
@pytest.mark.parametrize("value", ["nan", "inf"])
def test_decay_values_that_are_no_numbers(name, value, t):
    """They reach their own and later tokens of their sequence alone (Q: its own)."""
    s = decay_case(400, 2, 2, 2, 64, 64, t, seed=9)
    at = dict(sequences=2, length=200)
    clean = decay_run(s, t, at, grads=False)["O"]
    for where in (0, 3, 64, 100, 199):
        bad = dict(s, **{name: s[name].copy()})
        bad[name][where, 1, 5] = {"bf16": {"nan": 0x7fc0, "inf": 0x7f80}, "f32": {"nan": np.nan, "inf": np.inf}}[t][value]
        got = decay_run(bad, t, at, grads=False)["O"]
        assert torch.equal(got[200:], clean[200:]) and torch.equal(got[:200, 0], clean[:200, 0])
        # (a chunk with such a value of V is summed in another order)
        assert torch.allclose(got[:where], clean[:where], rtol=2.0 ** -7, atol=1e-5)
        if name == "Q":
            assert torch.equal(got[where + 1:], clean[where + 1:]) and not torch.isfinite(got[where, 1]).all()
        elif name == "V":
            assert not torch.isfinite(got[where:200, 1, 5]).any()
        else:
            assert not torch.isfinite(got[where:200, 1]).any()


def test_decay_same_bits_and_outputs_left_out():
    s = decay_case(3 * 333, 3, 4, 2, 64, 96, "bf16", seed=11)
    at = dict(sequences=3, length=333)
    first = decay_run(s, "bf16", at)
    for fill in (0, 0x7F):
        again = decay_run(s, "bf16", at, ws_fill=fill)
        assert all(torch.equal(first[n], again[n]) for n in ALL)
    prob = decay_problem(s, "bf16", at, 0.7)
    g = {k: up(s[k]) for k in ("Q", "K", "V", "dO", "log_decay", "state", "dstate_out")}
    n = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for one in ("dQ", "dK", "dV", "dstate"):
        out = {k: torch.empty_like(first[k]) if k == one else None for k in ("dQ", "dK", "dV", "dstate")}
        stl.stl_decay_attention_backward(prob, g["Q"], g["K"], g["V"], g["log_decay"], None, g["state"], g["dO"], g["dstate_out"], *out.values(), ws, n)
        assert torch.equal(out[one], first[one]), one


def test_decay_without_tokens():
    prob = stl.DecayAttentionProblem(0, 2, 0, 3, 3, 16)
    state, after = torch.randn(2, 3, 16, 16, device="cuda"), torch.empty(2, 3, 16, 16, device="cuda")
    for op in (stl.STL_OP_FORWARD, stl.STL_OP_BACKWARD):
        n = stl.stl_decay_attention_workspace_bytes(prob, op)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        if op == stl.STL_OP_FORWARD:
            stl.stl_decay_attention_forward(prob, None, None, None, None, None, state, None, after, ws, n)
        else:
            stl.stl_decay_attention_backward(prob, None, None, None, None, None, None, None, state, None, None, None, after, ws, n)
        assert torch.equal(after, state)
    stl.stl_decay_attention_forward(prob, None, None, None, None, None, None, None, after, None, 0)
    assert not after.any()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_decay_without_tokens_and_with_shared_heads(t):
    """Empty sequences: gradients of keys and values have no rows to write, states pass through."""
    prob = stl.DecayAttentionProblem(6, 2, 6, 4, 2, 16, scale=0.5, dtype=STL_DT[t])
    n = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    Q, dO = (torch.randn(6, 4, 16, device="cuda").to(TORCH_DT[t]) for _ in range(2))
    K, V = (torch.randn(6, 2, 16, device="cuda").to(TORCH_DT[t]) for _ in range(2))
    state, after = torch.randn(2, 4, 16, 16, device="cuda"), torch.empty(2, 4, 16, 16, device="cuda")
    outs = [torch.full_like(x, 3.0) for x in (Q, K, V)]
    offset = torch.tensor([2, 2, 2], device="cuda")
    stl.stl_decay_attention_backward(prob, Q, K, V, None, offset, None, dO, state, *outs, after, ws, n)
    assert torch.equal(after, state) and all(bool((o == 3).all()) for o in outs)
    none = stl.DecayAttentionProblem(0, 2, 0, 4, 2, 16, scale=0.5, dtype=STL_DT[t])
    after.zero_()
    stl.stl_decay_attention_backward(none, Q, K, V, None, None, None, dO, state, *outs, after, ws, n)
    assert torch.equal(after, state) and all(bool((o == 3).all()) for o in outs)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("length", [3, 6, 7, 9])
def test_decay_few_tokens(t, length):
    """Around the number of tokens up to which they go one by one; heads enough for wide workgroups, and fewer; widths that end inside one."""
    for sequences, heads, kv, dk, dv in ((3, 4, 2, 64, 64), (70, 16, 8, 40, 128), (129, 8, 8, 24, 97), (2, 2, 1, 256, 130), (40, 30, 30, 16, 96)):
        check_decay(sequences, length, heads, kv, dk, dv, t, seed=length + dv, in_place=True)


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("share", [1, 2])
def test_decay_in_segments(t, share):
    """Few heads and long sequences, which come in segments: rows one after the other, far apart, packed, and not of whole pieces."""
    for length, dk, dv in ((1024, 64, 48), (777, 33, 70), (2049, 128, 128)):
        check_decay(2, length, 2 * share, 2, dk, dv, t, seed=length)
    check_decay(3, 600, 2 * share, 2, 48, 64, t, at=dict(sequences=3, length=600, seq_step=1, token_step=3), seed=1, in_place=True)
    offset = np.array([5, 5, 1200, 1201, 1900, 2500], np.int64)
    check_decay(5, 1195, 2 * share, 2, 64, 64, t, at=dict(sequences=5, length=1195, offset=offset), rows=2600, seed=2)


def test_decay_gradients_are_differences():
    """Against central differences of the library's own forward call, fp32."""
    s = decay_case(40, 2, 2, 1, 8, 8, "f32", seed=13)
    at = dict(sequences=2, length=20)
    got = decay_run(s, "f32", at)

    def loss(**kw):
        r = decay_run(dict(s, **kw), "f32", at, grads=False)
        return float((r["O"].double() * up(s["dO"]).double()).sum() + (r["state"].double() * up(s["dstate_out"]).double()).sum())

    rng = np.random.default_rng(0)
    for n, g in (("Q", "dQ"), ("K", "dK"), ("V", "dV"), ("state", "dstate")):
        way = rng.standard_normal(s[n].shape).astype(np.float32)
        h = 2.0 ** -6
        want = (loss(**{n: s[n] + h * way}) - loss(**{n: s[n] - h * way})) / (2 * h)
        have = float((got[g].double().cpu().numpy().reshape(way.shape) * way).sum())
        # the loss is of the first order in each of them: what is left are fp32 sums' errors, a few 2^-24 of a few hundred terms of size 1, over h
        assert abs(have - want) <= 2e-3 * max(1.0, np.abs(got[g].double().cpu().numpy().reshape(way.shape) * way).sum() / 30), (n, have, want)


# ---- together, streams and graphs ---------------------------------------------------------------------------------------------------

class Block:
    """Embedding, norms and rotation, and attention as a model calls them in a row, forward and backward, on buffers of its own: queries, keys and values are parts of
    the embedding's rows."""

    def __init__(self, seed=0, batch=2, length=130, heads=2, d=64, vocab=200):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        self.rows, self.batch, self.length, self.heads, self.d, self.wide = batch * length, batch, length, heads, d, 3 * heads * d
        self.token = torch.randint(-2, vocab, (self.rows,), generator=g, device="cuda")
        self.position = torch.arange(self.rows, device="cuda") % length
        self.W, self.w_q, self.w_k, self.dO = r(vocab, self.wide), r(d), r(d), r(self.rows, heads * d)
        self.log_decay = torch.log1p(-(2.0 ** -torch.linspace(2, 6, heads, device="cuda")))
        self.state = torch.randn((batch, heads, d, d), generator=g, device="cuda")
        self.embed = stl.EmbedProblem(self.rows, self.wide, vocab, 0.5)
        self.norm = stl.HeadNormProblem(self.rows, heads, heads, d, ld_q=self.wide, ld_k=self.wide, ld_qout=self.wide, ld_kout=self.wide)
        self.attend = stl.DecayAttentionProblem(self.rows, batch, length, heads, dk=d, ld_q=self.wide, ld_k=self.wide, ld_v=self.wide, scale=0.125)
        self.X, self.Y, self.dX, self.dY = (torch.empty((self.rows, self.wide), dtype=torch.bfloat16, device="cuda") for _ in range(4))
        self.O = torch.empty((self.rows, heads * d), dtype=torch.bfloat16, device="cuda")
        self.after, self.dstate = torch.empty_like(self.state), torch.empty_like(self.state)
        self.dW, self.dw_q, self.dw_k = torch.empty_like(self.W), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        self.n = max(stl.stl_embed_workspace_bytes(self.embed), stl.stl_head_norm_workspace_bytes(self.norm),
                     *(stl.stl_decay_attention_workspace_bytes(self.attend, op) for op in (stl.STL_OP_FORWARD, stl.STL_OP_BACKWARD)))
        self.ws = torch.empty(self.n, dtype=torch.uint8, device="cuda")

    def outputs(self):
        return self.O, self.after, self.dstate, self.dW, self.dw_q, self.dw_k

    def parts(self, m):
        w = self.heads * self.d
        return m[:, :w], m[:, w:2 * w], m[:, 2 * w:]

    def __call__(self):
        X, Y, dX, dY = (self.parts(m) for m in (self.X, self.Y, self.dX, self.dY))
        stl.stl_embed_forward(self.embed, self.token, self.W, self.X)
        Y[2].copy_(X[2])
        stl.stl_head_norm_forward(self.norm, X[0], X[1], self.w_q, self.w_k, self.position, Y[0], Y[1])
        stl.stl_decay_attention_forward(self.attend, *Y, self.log_decay, None, self.state, self.O, self.after, self.ws, self.n)
        stl.stl_decay_attention_backward(self.attend, *Y, self.log_decay, None, self.state, self.dO, None, *dY, self.dstate, self.ws, self.n)
        stl.stl_head_norm_backward(self.norm, X[0], X[1], self.w_q, self.w_k, self.position, dY[0], dY[1], dX[0], dX[1], self.dw_q, self.dw_k, 0, self.ws, self.n)
        dX[2].copy_(dY[2])
        stl.stl_embed_backward(self.embed, self.token, self.dX, self.dW, 0, self.ws, self.n)


def test_together_against_the_oracle():
    """Every step on what the step before it left in bf16."""
    b = Block()
    b()
    torch.cuda.synchronize()
    heads = lambda m: tuple(down(p).reshape(b.rows, b.heads, b.d) for p in b.parts(m))  # noqa: E731
    X, Y, dX, dY = (heads(m) for m in (b.X, b.Y, b.dX, b.dY))
    want = seq.embed_forward(b.token.cpu().numpy(), down(b.W), 0.5)
    close(down(b.X), want, np.abs(want), "bf16", 0, "X")
    at = dict(position=b.position.cpu().numpy(), rot=b.d)
    for i, (w, dw) in enumerate(((b.w_q, b.dw_q), (b.w_k, b.dw_k))):
        want, size = seq.head_forward(X[i], down(w), **at)
        close(Y[i], want, size, "bf16", b.d + 32, "head")
        want = seq.head_backward(X[i], dY[i], down(w), **at)
        close(dX[i], want["dx"], want["size"]["dx"], "bf16", 2 * b.d + 64, "dX")
        close(down(dw), want["dw"], want["size"]["dw"], "f32", b.rows * b.heads + b.d + 64, "dw")
    rows_of = seq.decay_rows(b.batch, b.length, b.length, 1)
    want = seq.decay(*Y, rows_of, b.log_decay.cpu().numpy(), 0.125, down(b.state), down(b.dO).reshape(b.rows, b.heads, b.d))
    two, three, chain = 2 * 2.0 ** -16, 2 * 2.0 ** -24, b.length + 4 * b.d
    for n, g in (("O", down(b.O).reshape(want["O"].shape)), ("dQ", dY[0]), ("dK", dY[1]), ("dV", dY[2])):
        close(g, want[n], want["size"][n], "bf16", chain, n, two)
    for n, g in (("state", b.after), ("dstate", b.dstate)):
        close(down(g), want[n], want["size"][n], "f32", chain, n, three)
    want = seq.embed_backward(b.token.cpu().numpy(), down(b.dX), b.W.shape[0], 0.5)
    close(down(b.dW), want["dW"], want["size"]["dW"], "bf16", b.rows + 32, "dW")


def test_on_another_stream():
    a, b = Block(3), Block(3)
    a()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b()
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.outputs(), b.outputs()))


def test_in_captured_graphs_that_share_a_workspace():
    a, b = Block(5), Block(6, batch=1, length=70)
    b.ws, b.n = a.ws, a.n
    graphs = []
    for block in (a, b):
        block()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block()
        graphs.append(graph)
    for k in range(4):
        for block in (a, b):
            block.token.copy_(torch.randint_like(block.token, 0, 200))
            block.dO.copy_(torch.randn_like(block.dO))
        wants = []
        for block in (a, b):
            block()
            torch.cuda.synchronize()
            wants.append([o.clone() for o in block.outputs()])
            for o in block.outputs():
                o.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for block, want in zip((a, b), wants):
            assert all(torch.equal(x, y) for x, y in zip(want, block.outputs())), k
