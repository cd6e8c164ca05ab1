"""Calls of the embedding, the norms and rotation of queries and keys, and attention with decay that ask for a part of the outputs, come in many steps or lie at the
ends of what is allowed, on the GPU."""
import itertools

import numpy as np
import pytest
import torch

import paper_2503_12211_amd as stl
from gpu_util import STL_DT, TORCH_DT
from oracle import seq
from seq_cases import close, decay_bounds, decay_case, decay_chain, decay_check, head_case, narrow, walk_bound, walk_case, wide
from test_gpu_seq import ADJ, PRE, decay_problem, decay_run, down, up

pytestmark = pytest.mark.gpu
GRADS = ("dQ", "dK", "dV", "dstate")


@pytest.mark.parametrize("t,d,rot,adjacent", [("bf16", 64, 64, False), ("bf16", 128, 64, True), ("f32", 64, 64, False), ("f32", 50, 20, True), ("bf16", 256, 256, False)])
@pytest.mark.parametrize("rows", [3, 300])
def test_any_set_of_head_gradients(rows, t, d, rot, adjacent):
    """Every set of outputs has the bits of the call that asks for all of them: 70 heads, so that all wavefronts of a workgroup have some, weights of queries unlike
    those of keys."""
    heads, flags = 70, PRE | (ADJ if adjacent else 0)
    c = {k: up(v) for k, v in head_case(rows, heads, heads, d, t, seed=1).items()}
    prob = stl.HeadNormProblem(rows, heads, heads, d, rot, dtype=STL_DT[t])
    n = stl.stl_head_norm_workspace_bytes(prob, flags)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    every = ("dQ", "dK", "dw_q", "dw_k")

    def run(some):
        out = {k: torch.full_like(c[k[1:]], 3.0) if k in ("dQ", "dK") else torch.full((d,), 3.0, device="cuda") for k in some}
        stl.stl_head_norm_backward(prob, *(c[k] for k in ("Q", "K", "w_q", "w_k", "position", "dQout", "dKout")), *(out.get(k) for k in every), 0, ws, n, flags)
        return out

    full = run(every)
    for size in range(1, 4):
        for some in itertools.combinations(every, size):
            for k, v in run(some).items():
                assert torch.equal(v, full[k]), (some, k)


@pytest.mark.parametrize("step", [1, 5])
def test_decay_token_by_token_for_long(step):
    """States after thousands of tokens, a few a call and in place: lambda's own rounding, which has the same sign at each token, is not in them."""
    length = 6000
    s, want = walk_case(length, 32, 32)
    g = {k: up(v) for k, v in s.items()}
    prob, O, state = stl.DecayAttentionProblem(step, 1, step, 3, dk=32, dtype=stl.STL_F32), torch.empty((step, 3, 32), device="cuda"), g["state"]
    assert stl.stl_decay_attention_workspace_bytes(prob) == 0
    for at in range(0, length, step):
        stl.stl_decay_attention_forward(prob, *(g[n][at:at + step] for n in "QKV"), g["log_decay"], None, state, O, state)
    off = np.linalg.norm(down(state)[0] - want, axis=(1, 2)) / np.linalg.norm(want, axis=(1, 2))
    assert (off <= walk_bound(length, 2)).all(), off


@pytest.mark.parametrize("length,step,roundings", [(40000, 8, 9), (40000, 32, 33), (200000, 512, 16 * 33)])
def test_decay_in_short_calls_for_long(length, step, roundings):
    """The same where a call has one chunk of up to 32 products and a product by a power of lambda, or several chunks in segments."""
    s, want = walk_case(length, 32, 32)
    g = {k: up(v) for k, v in s.items()}
    probs = {n: stl.DecayAttentionProblem(n, 1, n, 3, dk=32, dtype=stl.STL_F32) for n in (step, length % step) if n}
    n, O, state = stl.stl_decay_attention_workspace_bytes(probs[step]), torch.empty((step, 3, 32), device="cuda"), g["state"]
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    calls = -(-length // step)
    for at in range(0, length, step):                            # (the last call takes what is left)
        prob = probs[min(step, length - at)]
        stl.stl_decay_attention_forward(prob, *(g[k][at:at + step] for k in "QKV"), g["log_decay"], None, state, O, state, ws, n)
    off = np.linalg.norm(down(state)[0] - want, axis=(1, 2)) / np.linalg.norm(want, axis=(1, 2))
    assert (off <= walk_bound(calls, roundings)).all(), (off, walk_bound(calls, roundings))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("length", [5, 20, 40, 70])
def test_decay_of_a_state_alone(length, t):
    """Keys and queries of zeros: states and their gradients fade by lambda^length, however little of them is left (half a step for each chunk's product, each rounding of
    lambda^n, and what these begin with)."""
    s = decay_case(length, 1, 9, 9, 20, 36, t, seed=2)
    s["K"][:], s["Q"][:] = 0, 0
    s["log_decay"][-1] = -1.0
    left = np.exp(length * s["log_decay"].astype(np.float64))[:, None, None]
    got = decay_run(s, t, dict(sequences=1, length=length))
    for n, was in (("state", "state"), ("dstate", "dstate_out")):
        assert (np.abs(down(got[n]) - left * s[was]) <= (length // 32 * 3 + 6) * 2.0 ** -24 * left * np.abs(s[was])).all(), n


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("length", [70, 700])
@pytest.mark.parametrize("scale,more,after", [(2.0 ** -100, 2.0 ** 60, 2.0 ** 60), (2.0 ** 100, 2.0 ** -60, 2.0 ** -60), (1e-30, 1.0, 1e9), (1e30, 1e-30, 1e-12)])
def test_decay_gradients_of_scales_far_from_one(length, scale, more, after, t):
    """The state's gradient is held as the formula has it: neither it nor what is handed in is divided by the scale.  In one piece and in segments."""
    s = decay_case(length, 1, 2, 1, 20, 36, t, seed=3)
    s["dO"], s["dstate_out"] = narrow(wide(s["dO"], t) * more, t), (s["dstate_out"].astype(np.float64) * after).astype(np.float32)
    got = decay_run(s, t, dict(sequences=1, length=length), scale)
    decay_check({k: down(got[k]) for k in GRADS}, s, [list(range(length))], t, float(np.float32(scale)), length, GRADS)


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_decay_gradients_of_states_without_tokens_pass_through(t):
    """Sequences without tokens: the same bits, whatever the scale; states alike."""
    for length in (40, 700):
        s = decay_case(length, 3, 2, 1, 20, 36, t, seed=4)
        got = decay_run(s, t, dict(sequences=3, length=length, offset=np.array([0, 0, length, length], np.int64)), 0.7)
        for b in (0, 2):
            assert torch.equal(got["dstate"][b], up(s["dstate_out"][b])) and torch.equal(got["state"][b], up(s["state"][b]))


@pytest.mark.parametrize("t,dk,dv", [("bf16", 16, 136), ("f32", 130, 8)])
def test_decay_of_the_most_heads(t, dk, dv):
    """As many heads of all sequences as are allowed, in more workgroups than one launch has room for: all but the first and the last few sequences are empty."""
    most, length, rows = 4194304, 9, 40
    s = decay_case(rows, 1, 1, 1, dk, dv, t, seed=1, states=False)
    offset = np.full(most + 1, 16, np.int64)
    offset[:3], offset[-3:] = [0, 9, 16], [16, 25, 32]
    at = dict(sequences=most, length=length, offset=offset)
    prob, g = decay_problem(s, t, at, 0.7), {k: up(v) for k, v in s.items()}
    out = {n: torch.full(s[like].shape, float("nan"), dtype=TORCH_DT[t], device="cuda") for n, like in (("O", "dO"), ("dQ", "Q"), ("dK", "K"), ("dV", "V"))}
    where, n = up(offset), stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    stl.stl_decay_attention_forward(prob, g["Q"], g["K"], g["V"], g["log_decay"], where, None, out["O"], None, ws, n)
    stl.stl_decay_attention_backward(prob, g["Q"], g["K"], g["V"], g["log_decay"], where, None, g["dO"], None, out["dQ"], out["dK"], out["dV"], None, ws, n)
    rows_of = [list(range(9)), list(range(9, 16)), list(range(16, 25)), list(range(25, 32))]
    _, covered = decay_check({k: down(v) for k, v in out.items()}, s, rows_of, t, 0.7, length, ("O", "dQ", "dK", "dV"))
    assert all(bool(torch.isnan(v[32:]).all()) for v in out.values()) and covered[:32].all()


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [float("inf"), float("nan")])
def test_embed_rows_without_a_token_are_zeros_whatever_the_scale(scale, t):
    token, W = torch.tensor([3, -100, 0, 30, 2 ** 40, 29], device="cuda"), torch.randn(30, 21, device="cuda").to(TORCH_DT[t])
    X = torch.empty((6, 21), dtype=W.dtype, device="cuda")
    stl.stl_embed_forward(stl.EmbedProblem(6, 21, 30, scale, STL_DT[t]), token, W, X)
    assert not X[[1, 3, 4]].any() and not torch.isfinite(X[[0, 2, 5]]).any()


def far(x, ld, fill=None):
    """The same rows, ld elements from row to row, in memory that holds nothing else"""
    rows, wide_ = x.shape[0], x[0].numel()
    v = torch.empty((rows - 1) * ld + wide_, dtype=x.dtype, device="cuda").as_strided((rows, wide_), (ld, 1))
    return v.fill_(fill) if fill is not None else v.copy_(x.reshape(rows, -1))


def test_heads_more_elements_apart_than_32_bits_count():
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("not enough free memory")
    rows, heads, d, ld = 4, 3, 64, (1 << 30) + 17
    c = {k: up(v) for k, v in head_case(rows, heads, heads, d, "bf16", seed=1).items()}
    want, prob = {}, stl.HeadNormProblem(rows, heads, heads, d)
    apart = stl.HeadNormProblem(rows, heads, heads, d, None, ld, ld, ld, ld)
    n = stl.stl_head_norm_workspace_bytes(prob)
    ws, dw = torch.empty(n, dtype=torch.uint8, device="cuda"), [torch.empty(d, device="cuda") for _ in range(4)]
    want = {k: torch.empty_like(c["Q"]) for k in ("Qout", "Kout", "dQ", "dK")}
    stl.stl_head_norm_forward(prob, c["Q"], c["K"], c["w_q"], c["w_k"], c["position"], want["Qout"], want["Kout"])
    stl.stl_head_norm_backward(prob, c["Q"], c["K"], c["w_q"], c["w_k"], c["position"], c["dQout"], c["dKout"], want["dQ"], want["dK"], dw[0], dw[1], 0, ws, n)
    x = {k: far(c[k], ld) for k in ("Q", "K", "dQout", "dKout")}
    stl.stl_head_norm_backward(apart, x["Q"], x["K"], c["w_q"], c["w_k"], c["position"], x["dQout"], x["dKout"], x["dQout"], x["dKout"], dw[2], dw[3], 0, ws, n)
    stl.stl_head_norm_forward(apart, x["Q"], x["K"], c["w_q"], c["w_k"], c["position"], x["Q"], x["K"])
    for k, v in (("Qout", "Q"), ("Kout", "K"), ("dQ", "dQout"), ("dK", "dKout")):
        assert torch.equal(x[v].reshape(rows, heads, d), want[k]), k
    assert torch.equal(dw[0], dw[2]) and torch.equal(dw[1], dw[3])
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t,rows,ld,kv", [("bf16", 300, 1 << 23, 2), ("bf16", 70, 1 << 25, 1), ("bf16", 5, 1 << 29, 2), ("f32", 300, 1 << 23, 1)])
def test_decay_more_elements_apart_than_32_bits_count(t, rows, ld, kv):
    """Rows as far apart as the ring of loads takes them, and further."""
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("not enough free memory")
    assert rows * ld > 1 << 31
    s = decay_case(rows, 1, 2, kv, 32, 48, t, seed=2)
    g = {k: up(v) for k, v in s.items()}
    x = {k: far(g[k], ld) for k in ("Q", "K", "V", "dO")}
    out = {k: far(x[like], ld, float("nan")) for k, like in (("O", "dO"), ("dQ", "Q"), ("dK", "K"), ("dV", "V"))}
    prob = stl.DecayAttentionProblem(rows, 1, rows, 2, kv, 32, 48, None, 1, ld, ld, ld, ld, scale=0.7, dtype=STL_DT[t])
    state, dstate = torch.empty_like(g["state"]), torch.empty_like(g["state"])
    n = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    stl.stl_decay_attention_forward(prob, x["Q"], x["K"], x["V"], g["log_decay"], None, g["state"], out["O"], state, ws, n)
    stl.stl_decay_attention_backward(prob, x["Q"], x["K"], x["V"], g["log_decay"], None, g["state"], x["dO"], g["dstate_out"], out["dQ"], out["dK"], out["dV"], dstate, ws, n)
    got = {k: down(v).reshape(rows, -1, 48 if k in ("O", "dV") else 32) for k, v in out.items()}
    decay_check(dict(got, state=down(state), dstate=down(dstate)), s, [list(range(rows))], t, 0.7, rows, ("O", "state", *GRADS))
    del x, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_heads_of_zeros_with_the_smallest_eps(t):
    x, out = torch.zeros((3, 2, 64), dtype=TORCH_DT[t], device="cuda"), [torch.full((3, 2, 64), 3.0, dtype=TORCH_DT[t], device="cuda") for _ in range(2)]
    for eps in (1e-30, 1.2e-38, 1e-40):
        prob = stl.HeadNormProblem(3, 2, 0, 64, eps=eps, dtype=STL_DT[t])
        n = stl.stl_head_norm_workspace_bytes(prob)
        ws, dw = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(64, device="cuda")
        stl.stl_head_norm_forward(prob, x, None, None, None, None, out[0], None)
        stl.stl_head_norm_backward(prob, x, None, None, None, None, x, None, out[1], None, dw, None, 0, ws, n)
        assert not out[0].any() and not out[1].any() and not dw.any(), eps


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
def test_decay_gradients_of_more_sequences_than_a_grid_is_high(packed, t):
    """Shared key heads of 70000 sequences: the bits of two calls with half of them each."""
    n, length, heads, d = 70000, 3, 2, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda k: torch.randn((n * length, k, d), generator=g, device="cuda").to(TORCH_DT[t])  # noqa: E731
    Q, K, V, dO = r(heads), r(1), r(1), r(heads)
    # packed: 0 to 3 tokens each, and rows of no sequence at the end
    ends = torch.randint(0, length + 1, (n,), generator=g, device="cuda").cumsum(0) if packed else None
    offset = torch.cat([ends.new_zeros(1), ends]) if packed else None
    decay = torch.tensor([-0.1, -0.5], device="cuda")

    def grads(first, last):
        count, at = last - first, slice(first * length, last * length)
        some = [x if packed else x[at] for x in (Q, K, V, dO)]
        prob = stl.DecayAttentionProblem(some[0].shape[0], count, length, heads, 1, d, scale=0.5, dtype=STL_DT[t])
        size = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        outs = [torch.full_like(x, 3.0) for x in some[:3]]
        stl.stl_decay_attention_backward(prob, *some[:3], decay, offset[first:last + 1].clone() if packed else None, None, some[3], None, *outs, None, ws, size)
        return outs

    whole, low, high = grads(0, n), grads(0, n // 2), grads(n // 2, n)
    for w, a, b in zip(whole, low, high):
        if packed:
            cut, end = int(offset[n // 2]), int(offset[-1])
            assert torch.equal(w[:cut], a[:cut]) and torch.equal(w[cut:], b[cut:]) and bool((a[cut:] == 3).all()) and bool((w[end:] == 3).all())
        else:
            assert torch.equal(w, torch.cat([a, b]))


def test_embed_of_the_most_rows():
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("not enough free memory")
    rows, vocab = stl.STL_MAX_DIM, 1000
    token = torch.randint(-1, vocab, (rows,), device="cuda")
    at = torch.cat([torch.arange(5000, device="cuda"), torch.arange(rows - 5000, rows, device="cuda"), torch.randint(0, rows, (5000,), device="cuda")])
    W = torch.randn(vocab, 2048, device="cuda").to(torch.bfloat16)
    X = torch.empty((rows, 2048), dtype=W.dtype, device="cuda")
    stl.stl_embed_forward(stl.EmbedProblem(rows, 2048, vocab), token, W, X)
    assert torch.equal(X[at], torch.where((token[at] >= 0)[:, None], W[token[at].clamp_min(0)], 0.0).to(W.dtype))
    del X
    torch.cuda.empty_cache()
    # gradients that are small whole numbers: their sums are too
    dX, dW = torch.randint(-2, 3, (rows, 8), device="cuda").float(), torch.empty((vocab, 8), device="cuda")
    prob = stl.EmbedProblem(rows, 8, vocab, dtype=stl.STL_F32)
    n = stl.stl_embed_workspace_bytes(prob)
    stl.stl_embed_backward(prob, token, dX, dW, 0, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    want = torch.zeros((vocab + 1, 8), dtype=torch.float64, device="cuda").index_add_(0, torch.where(token < 0, vocab, token), dX.double())
    assert torch.equal(dW.double(), want[:vocab])


def test_heads_of_the_most_rows():
    rows, d = stl.STL_MAX_DIM, 16
    Q, up_ = (torch.randn((rows, 1, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    position, w = torch.arange(rows, device="cuda"), torch.randn(d, device="cuda").to(torch.bfloat16)
    out, dQ, dw = torch.empty_like(Q), torch.empty_like(Q), torch.empty(d, device="cuda")
    prob = stl.HeadNormProblem(rows, 1, 0, d)
    n = stl.stl_head_norm_workspace_bytes(prob)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    stl.stl_head_norm_forward(prob, Q, None, w, None, position, out, None)
    stl.stl_head_norm_backward(prob, Q, None, w, None, position, up_, None, dQ, None, dw, None, 0, ws, n)
    for lo in (0, rows // 2 - 50, rows - 100):
        some = slice(lo, lo + 100)
        part, b, c = stl.HeadNormProblem(100, 1, 0, d), torch.empty_like(Q[some]), torch.empty_like(Q[some])
        stl.stl_head_norm_forward(part, Q[some].clone(), None, w, None, position[some].clone(), b, None)
        stl.stl_head_norm_backward(part, Q[some].clone(), None, w, None, position[some].clone(), up_[some].clone(), None, c, None, None, None, 0, ws, n)
        assert torch.equal(out[some], b) and torch.equal(dQ[some], c)
    angle = position.double()[:, None] * 10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    x, u = Q[:, 0].double(), up_[:, 0].double()
    a, b = u[:, :d // 2], u[:, d // 2:]
    back = torch.cat([a * angle.cos() + b * angle.sin(), b * angle.cos() - a * angle.sin()], 1)
    hat = x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt()
    # a workgroup's sums are chains of rows / 1024, its lanes' and the workgroups' come behind them
    assert bool(((dw.double() - (back * hat).sum(0)).abs() <= (rows // 1024 + 64) * 2.0 ** -24 * (back * hat).abs().sum(0)).all())


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_decay_of_the_longest_sequence(t):
    """16.8 million tokens in segments; a token sees some thousand before it."""
    rows, d = stl.STL_MAX_DIM, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    Q, K, V, dO = (torch.randn((rows, 1, d), generator=g, device="cuda").to(TORCH_DT[t]) for _ in range(4))
    decay = torch.tensor([-0.02], device="cuda")
    prob = stl.DecayAttentionProblem(rows, 1, rows, 1, dk=d, scale=0.5, dtype=STL_DT[t])
    n = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    O, dQ, dK, dV = (torch.empty_like(Q) for _ in range(4))
    state = torch.empty((1, 1, d, d), device="cuda")
    stl.stl_decay_attention_forward(prob, Q, K, V, decay, None, None, O, state, ws, n)
    stl.stl_decay_attention_backward(prob, Q, K, V, decay, None, None, dO, None, dQ, dK, dV, None, ws, n)
    window, inner = 2400, 1000                                   # what is behind 1000 tokens has faded to 2e-9
    for lo in (0, rows // 256 * 100 - window // 2, rows - window):
        some = slice(lo, lo + window)
        cut = slice(0 if lo == 0 else inner, window if lo == rows - window else window - inner)
        s = {"Q": Q, "K": K, "V": V, "dO": dO}
        s = {k: v[some].cpu() for k, v in s.items()}
        want = seq.decay(*(s[k].double().numpy() for k in "QKV"), [list(range(window))], decay.cpu().numpy(), 0.5, None, s["dO"].double().numpy())
        for name, got in (("O", O), ("dQ", dQ), ("dK", dK), ("dV", dV)):
            kind, operand = decay_bounds(name, t)
            close(down(got[some])[cut], want[name][cut], want["size"][name][cut], kind, decay_chain(window, d, d) + 33, name, operand + 2e-8)
    kind, operand = decay_bounds("state", t)
    close(down(state), want["state"], want["size"]["state"], kind, decay_chain(window, d, d) + 33, "state", operand + 2e-8)
