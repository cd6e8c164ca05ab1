"""What lies between a language model's tokens and its layers, as cases to time: the embedding's rows and their gradient, the norms of queries
and keys for each head with the rotation by position, and attention whose past decays, over prompts and a token at a time, with its gradients.

A case is one `kind` of call and its sizes:

  embed            stl_embed_forward
  embed_grads      stl_embed_backward
  head_norm        stl_head_norm_forward
  head_norm_grads  stl_head_norm_backward
  decay            stl_decay_attention_forward (prompts, and single tokens that read and write a state)
  decay_grads      stl_decay_attention_backward

Values: activations ~ N(0, 1); tokens by Zipf's law, as in text (the commonest is one token in ten); positions from anywhere in a long context; queries and keys
of length about 1 before the attention, decays from a few tokens to a few thousand, spread over the heads.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _embed(name, kind, dtype, rows, d, vocab, scale=1.0, padded=0.0):
    """padded: share of the rows whose token is none (-100)."""
    c = {"kind": kind, "dtype": dtype, "rows": rows, "d": d, "vocab": vocab, "scale": scale, "padded": padded}
    return {"name": name, **c} if name else c


def _head(name, kind, dtype, rows, heads, kv_heads, d, rot, adjacent=False):
    """rot: rotated elements of a head, the first ones; adjacent: pairs (0, 1), (2, 3), ... in the place of (0, rot / 2), (1, rot / 2 + 1), ..."""
    c = {"kind": kind, "dtype": dtype, "rows": rows, "heads": heads, "kv_heads": kv_heads, "d": d, "rot": rot, "adjacent": adjacent}
    return {"name": name, **c} if name else c


def _decay(name, kind, dtype, sequences, length, heads, kv_heads, dk, dv, rows="by sequence", states=False):
    """rows: "by sequence" (one after the other, of `length` tokens each), "packed" (of different lengths up to `length`, one of them empty) or "by position" (all
    sequences' first tokens, then all second ones); states: a state in front of the first token, and the one behind the last asked for."""
    c = {"kind": kind, "dtype": dtype, "sequences": sequences, "length": length, "heads": heads, "kv_heads": kv_heads, "dk": dk, "dv": dv, "rows": rows,
         "states": states}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a prompt of the benchmark's row count and width, rows scaled by sqrt(d) as models with tied vocabularies do
        _embed("embed_prompt", "embed", "bf16", 8192, 4096, 65536, scale=64.0),
        # the training step of a model of that many tokens a step
        _embed("embed_train", "embed_grads", "bf16", 16384, 2048, 32000),
        # an odd vocabulary and width in fp32, a padded batch
        _embed("embed_train_odd_f32", "embed_grads", "f32", 3001, 1021, 50001, scale=0.5, padded=0.2),
        # one new token of 16 sequences on its way through a serving loop: the launch counts
        _head("head_tokens", "head_norm", "bf16", 16, 32, 8, 128, 128),
        # a prompt's queries and keys, four query heads to a key head
        _head("head_prompt", "head_norm", "bf16", 8192, 32, 8, 128, 128),
        # images of 197 tokens, twelve heads, a part of each rotated, pairs side by side
        _head("head_train_images", "head_norm_grads", "bf16", 64 * 197, 12, 12, 64, 32, adjacent=True),
        # one token of one sequence, small heads
        _decay("decay_token", "decay", "bf16", 1, 1, 8, 8, 64, 64, states=True),
        # one token each of 64 sequences: reading and writing the states is the work
        _decay("decay_tokens", "decay", "bf16", 64, 1, 32, 32, 128, 128, states=True),
        # one long prompt
        _decay("decay_prompt", "decay", "bf16", 1, 8192, 32, 32, 128, 128),
        # packed prompts of different lengths that go on from earlier ones, shared key heads, an odd width
        _decay("decay_packed", "decay", "bf16", 13, 777, 16, 4, 96, 128, rows="packed", states=True),
        # a training step
        _decay("decay_train", "decay_grads", "bf16", 4, 2048, 16, 16, 128, 128),
        # a small fp32 training step, rows as STL layers want them (four sequences at one position to a tile), odd sizes, gradients of the states
        _decay("decay_train_odd_f32", "decay_grads", "f32", 8, 333, 4, 2, 48, 80, rows="by position", states=True),
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], uniform in its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / step)) * step, -(-lo // step) * step), hi // step * step)


_MOST = 2.6e8                                          # bytes of a drawn case, somewhat below those of the largest listed ones


def draw(rng):
    kind = rng.choice(["embed", "embed_grads", "head_norm", "head_norm_grads", "decay", "decay", "decay_grads", "decay_grads"])
    dtype, odd = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.random() < 0.4
    if kind.startswith("embed"):
        c = _embed(None, kind, dtype, _log_int(rng, 1, 32768), _log_int(rng, 64, 4096, 1 if odd else 64), _log_int(rng, 1000, 131072, 1 if odd else 128),
                   rng.choice([1.0, 1.0, 32.0, 0.3]), rng.choice([0.0, 0.0, 0.3]))
        while work(c)["bytes"] > _MOST:
            c["rows"], c["vocab"] = -(-c["rows"] // 2), max(1000, c["vocab"] // 2)
        return c
    if kind.startswith("head"):
        kv = rng.choice([1, 2, 4, 8, 12])
        d = rng.choice([64, 128, 128, 256, 80, 96, 50] if odd else [64, 128, 128, 256])
        c = _head(None, kind, dtype, _log_int(rng, 1, 16384), kv * rng.choice([1, 1, 2, 4]), kv, d, rng.choice([d, d, d // 2 // 2 * 2]), rng.random() < 0.3)
        while work(c)["bytes"] > _MOST:
            c["rows"] = -(-c["rows"] // 2)
        return c
    dims = [32, 64, 64, 128, 128, 128, 256] + ([48, 80, 96, 100, 37] if odd else [])
    kv = rng.choice([1, 2, 4, 8, 16])
    single = kind == "decay" and rng.random() < 0.3
    c = _decay(None, kind, dtype, _log_int(rng, 1, 64), 1 if single else _log_int(rng, 2, 4096), kv * rng.choice([1, 1, 2]), kv, rng.choice(dims), rng.choice(dims),
               rng.choice(["by sequence", "by sequence", "packed", "by position"]), single or rng.random() < 0.5)
    while work(c)["bytes"] > _MOST / 2 or work(c)["flops"] > 1e10 or c["sequences"] * c["heads"] * c["length"] ** 2 > 1 << 30:
        c["sequences"], c["length"] = -(-c["sequences"] // 2), c["length"] if c["sequences"] > 1 or single else c["length"] // 2
    return c


def _lengths(case):
    """Tokens of each sequence: packed ones from `length` down, the last but one of them empty where there are more than two."""
    n, length = case["sequences"], case["length"]
    if case["rows"] != "packed":
        return [length] * n
    at = [max(1, length - (i * length * 7) // (n * 8)) for i in range(n)]
    if n > 2:
        at[n - 2] = 0
    return at


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind.startswith("embed"):
        there = case["rows"] - int(case["rows"] * case["padded"])
        # rows of the vocabulary that occur, each once; a third of the tokens are others' repetition in the mean of these ranges
        if kind == "embed":
            return {"bytes": size * case["d"] * (case["rows"] + min(there * 2 // 3 + 1, case["vocab"])) + 8 * case["rows"], "flops": case["rows"] * case["d"]}
        return {"bytes": size * case["d"] * (there + case["vocab"]) + 8 * case["rows"], "flops": 2 * there * case["d"]}
    if kind.startswith("head"):
        n = case["rows"] * (case["heads"] + case["kv_heads"]) * case["d"]
        return {"bytes": (2 if kind == "head_norm" else 3) * size * n + 8 * case["rows"] + 12 * case["d"], "flops": (10 if kind == "head_norm" else 20) * n}
    rows, dk, dv = sum(_lengths(case)), case["dk"], case["dv"]
    queries, keys, values, outs = (rows * h * w for h, w in ((case["heads"], dk), (case["kv_heads"], dk), (case["kv_heads"], dv), (case["heads"], dv)))
    state = 4 * case["sequences"] * case["heads"] * dk * dv if case["states"] else 0
    if kind == "decay":
        return {"bytes": size * (queries + keys + values + outs) + 2 * state, "flops": 4 * rows * case["heads"] * dk * dv}
    # (the state in front is read, its gradient and that of the state behind the last token are written and read)
    return {"bytes": size * (2 * (queries + keys + values) + outs) + 3 * state, "flops": 12 * rows * case["heads"] * dk * dv}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)

    if case["kind"].startswith("embed"):
        s = _prepare_embed(case, g, randn, rand, dt)
    elif case["kind"].startswith("head"):
        s = _prepare_head(case, g, randn, dt)
    else:
        s = _prepare_decay(case, randn, dt)
    s["case"] = dict(case)
    if own:
        import paper_2503_12211_amd as stl
        s["ws_bytes"] = 0
        if case["kind"].startswith("embed"):
            s["prob"] = stl.EmbedProblem(case["rows"], case["d"], case["vocab"], case["scale"], stl.STL_BF16 if dt == torch.bfloat16 else stl.STL_F32)
            s["ws_bytes"] = stl.stl_embed_workspace_bytes(s["prob"])
        elif case["kind"].startswith("head"):
            s["prob"] = stl.HeadNormProblem(case["rows"], case["heads"], case["kv_heads"], case["d"], case["rot"], base=_BASE, eps=_EPS,
                                            dtype=stl.STL_BF16 if dt == torch.bfloat16 else stl.STL_F32)
            s["flags"] = stl.STL_FLAG_PRE_NORM | (stl.STL_FLAG_ADJACENT if case["adjacent"] else 0)
            s["ws_bytes"] = stl.stl_head_norm_workspace_bytes(s["prob"], s["flags"])
        else:
            by_position = case["rows"] == "by position"
            s["prob"] = stl.DecayAttentionProblem(sum(_lengths(case)), case["sequences"], case["length"], case["heads"], case["kv_heads"], case["dk"], case["dv"],
                                                  seq_step=1 if by_position else case["length"], token_step=case["sequences"] if by_position else 1,
                                                  scale=s["scale"], dtype=stl.STL_BF16 if dt == torch.bfloat16 else stl.STL_F32)
            s["ws_bytes"] = stl.stl_decay_attention_workspace_bytes(s["prob"], stl.STL_OP_FORWARD if case["kind"] == "decay" else stl.STL_OP_BACKWARD)
        s["ws"] = torch.empty(max(s["ws_bytes"], 16), dtype=torch.uint8, device="cuda")
    return s


def _prepare_embed(case, g, randn, rand, dt):
    rows, d, vocab = case["rows"], case["d"], case["vocab"]
    rank = torch.exp(rand(rows) * math.log(vocab + 1.0)).long().clamp(1, vocab) - 1          # P(rank) ~ 1 / rank
    token = torch.randperm(vocab, generator=g, device="cuda")[rank]
    none = torch.randperm(rows, generator=g, device="cuda")[:int(rows * case["padded"])]
    s = {"token": token.index_fill(0, none, -100)}
    s["W" if case["kind"] == "embed" else "dX"] = randn(vocab if case["kind"] == "embed" else rows, d).to(dt)
    return s


_BASE, _EPS = 10000.0, 1e-6


def _prepare_head(case, g, randn, dt):
    rows, d = case["rows"], case["d"]
    s = {"Q": (randn(rows, case["heads"], d) * 1.5 + 0.25).to(dt), "K": (randn(rows, case["kv_heads"], d) * 0.7).to(dt),
         "w_q": (1.0 + 0.1 * randn(d)).to(dt), "w_k": (1.0 + 0.1 * randn(d)).to(dt)}
    first = torch.randint(0, 131072, (1,), generator=g, device="cuda")
    if rows <= 64:                                                              # single tokens of sequences of all lengths
        first = torch.randint(0, 131072, (rows,), generator=g, device="cuda")
        s["position"] = first
    else:
        s["position"] = first + torch.arange(rows, device="cuda")
    if case["kind"] == "head_norm_grads":
        s["dQout"], s["dKout"] = randn(rows, case["heads"], d).to(dt), randn(rows, case["kv_heads"], d).to(dt)
    return s


def _prepare_decay(case, randn, dt):
    heads, kv, dk, dv = (case[k] for k in ("heads", "kv_heads", "dk", "dv"))
    lengths = _lengths(case)
    rows, n = sum(lengths), case["sequences"]
    s = {"Q": (randn(rows, heads, dk) / math.sqrt(dk)).to(dt), "K": (randn(rows, kv, dk) / math.sqrt(dk)).to(dt), "V": randn(rows, kv, dv).to(dt), "scale": 1.0,
         "offset": None, "state": None, "dstate": None}
    if case["rows"] == "packed":
        s["offset"] = torch.tensor([0] + lengths, device="cuda").cumsum(0)
    # decays 1 - 2^-2 ... 1 - 2^-11 over the heads
    span = torch.linspace(2.0, 11.0, heads, device="cuda", dtype=torch.float64)
    s["log_decay"] = torch.log1p(-(2.0 ** -span)).float()
    if case["states"]:
        s["state"] = randn(n, heads, dk, dv) * 0.5
        s["next"] = torch.empty_like(s["state"])                                 # a serving loop alternates between two buffers
    if case["kind"] == "decay_grads":
        s["dO"] = randn(rows, heads, dv).to(dt)
        if case["states"]:
            s["dstate"] = randn(n, heads, dk, dv) * 0.1
    return s


def run(s):
    kind = s["case"]["kind"]
    if kind == "embed":
        return _own_embed(s) if own else _plain_embed(s)
    if kind == "embed_grads":
        return _own_embed_grads(s) if own else _plain_embed_grads(s)
    if kind == "head_norm":
        return _own_head(s) if own else _plain_head(s)
    if kind == "head_norm_grads":
        return _own_head_grads(s) if own else _plain_head_grads(s)
    if kind == "decay":
        return _own_decay(s) if own else _plain_decay(s)
    return _own_decay_grads(s) if own else _plain_decay_grads(s)


# ---- the framework's operators ----------------------------------------------------------------------------------------------------

def _own_embed(s):
    import paper_2503_12211_amd as stl
    X = torch.empty((s["case"]["rows"], s["case"]["d"]), dtype=s["W"].dtype, device="cuda")
    stl.stl_embed_forward(s["prob"], s["token"], s["W"], X)
    return {"X": X}


def _own_embed_grads(s):
    import paper_2503_12211_amd as stl
    dW = torch.empty((s["case"]["vocab"], s["case"]["d"]), dtype=s["dX"].dtype, device="cuda")
    stl.stl_embed_backward(s["prob"], s["token"], s["dX"], dW, 0, s["ws"], s["ws_bytes"])
    return {"dW": dW}


def _own_head(s):
    import paper_2503_12211_amd as stl
    Qout, Kout = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
    stl.stl_head_norm_forward(s["prob"], s["Q"], s["K"], s["w_q"], s["w_k"], s["position"], Qout, Kout, s["flags"])
    return {"Qout": Qout, "Kout": Kout}


def _own_head_grads(s):
    import paper_2503_12211_amd as stl
    dQ, dK = torch.empty_like(s["Q"]), torch.empty_like(s["K"])
    dw_q, dw_k = (torch.empty(s["case"]["d"], dtype=torch.float32, device="cuda") for _ in range(2))
    stl.stl_head_norm_backward(s["prob"], s["Q"], s["K"], s["w_q"], s["w_k"], s["position"], s["dQout"], s["dKout"], dQ, dK, dw_q, dw_k, 0, s["ws"], s["ws_bytes"],
                               s["flags"])
    return {"dQ": dQ, "dK": dK, "dw_q": dw_q, "dw_k": dw_k}


def _own_decay(s):
    import paper_2503_12211_amd as stl
    O = torch.empty((s["Q"].shape[0], s["Q"].shape[1], s["V"].shape[2]), dtype=s["Q"].dtype, device="cuda")
    after = s["next"] if s["state"] is not None else None
    stl.stl_decay_attention_forward(s["prob"], s["Q"], s["K"], s["V"], s["log_decay"], s["offset"], s["state"], O, after, s["ws"], s["ws_bytes"])
    return {"O": O, "state": after}


def _own_decay_grads(s):
    import paper_2503_12211_amd as stl
    dQ, dK, dV = torch.empty_like(s["Q"]), torch.empty_like(s["K"]), torch.empty_like(s["V"])
    before = s["next"] if s["state"] is not None else None
    stl.stl_decay_attention_backward(s["prob"], s["Q"], s["K"], s["V"], s["log_decay"], s["offset"], s["state"], s["dO"], s["dstate"], dQ, dK, dV, before, s["ws"],
                                     s["ws_bytes"])
    return {"dQ": dQ, "dK": dK, "dV": dV, "dstate": before}


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ---------------------------------------------------------

def _plain_embed(s):
    c = s["case"]
    there = (s["token"] >= 0) & (s["token"] < c["vocab"])
    rows = s["W"][torch.where(there, s["token"], 0)].float() * c["scale"]
    return {"X": torch.where(there[:, None], rows, 0.0).to(s["W"].dtype)}


def _plain_embed_grads(s):
    c = s["case"]
    there = ((s["token"] >= 0) & (s["token"] < c["vocab"])).float()[:, None]
    sums = torch.zeros((c["vocab"], c["d"]), device="cuda").index_add_(0, s["token"].clamp(0, c["vocab"] - 1), s["dX"].float() * there)
    return {"dW": (sums * c["scale"]).to(s["dX"].dtype)}


def _turned(c, position, x, back=False):
    """The pairs of x (rows, heads, d) turned by their angles, or back."""
    half = c["rot"] // 2
    f = _BASE ** (-torch.arange(half, device="cuda", dtype=torch.float64) * 2.0 / max(c["rot"], 1))
    angle = position.double()[:, None] * f                                       # in 64 bits: a far position's angle is large
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    if back:
        sin = -sin
    head, tail = x[..., :c["rot"]], x[..., c["rot"]:]
    a, b = (head[..., 0::2], head[..., 1::2]) if c["adjacent"] else (head[..., :half], head[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["adjacent"] else torch.cat([a, b], -1)
    return torch.cat([turned, tail], -1)


def _plain_head(s):
    c, out = s["case"], {}
    x, w = {"Q": s["Q"].float(), "K": s["K"].float()}, {"Q": s["w_q"].float(), "K": s["w_k"].float()}
    norm = {n: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + _EPS) * w[n] for n, v in x.items()}
    out = {n + "out": _turned(c, s["position"], v).to(s["Q"].dtype) for n, v in norm.items()}
    return out


def _plain_head_grads_of(s, x, w, up):
    x, w = x.float(), w.float()
    dy = _turned(s["case"], s["position"], up.float(), back=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
    hat, t = x * r, dy * w
    return (r * (t - hat * (t * hat).mean(-1, keepdim=True))).to(s["Q"].dtype), (dy * hat).sum((0, 1))


def _plain_head_grads(s):
    dQ, dw_q = _plain_head_grads_of(s, s["Q"], s["w_q"], s["dQout"])
    dK, dw_k = _plain_head_grads_of(s, s["K"], s["w_k"], s["dKout"])
    return {"dQ": dQ, "dK": dK, "dw_q": dw_q, "dw_k": dw_k}


def _places(s):
    """Row of token t of sequence b (sequences, length), and whether there is one."""
    c = s["case"]
    b, t = torch.arange(c["sequences"], device="cuda")[:, None], torch.arange(c["length"], device="cuda")[None]
    if c["rows"] == "packed":
        return (s["offset"][:-1, None] + t).clamp_max(s["Q"].shape[0] - 1), t < (s["offset"][1:] - s["offset"][:-1])[:, None]
    return (t * c["sequences"] + b if c["rows"] == "by position" else b * c["length"] + t), (t < c["length"]).expand(c["sequences"], c["length"])


def _by_head(x, heads, place, there):
    """(rows, some heads, d) -> (sequences, heads, length, d) in 32 bits, zeros where there is no token."""
    x = torch.where(there[..., None, None], x[place].float(), 0.0).transpose(1, 2)
    return x.repeat_interleave(heads // x.shape[1], 1).contiguous()


def _by_row(x, like, place, there):
    """Back to the rows of `like`; heads that share one of its heads are added up."""
    n, heads, length, d = x.shape
    x = x.view(n, like.shape[1], heads // like.shape[1], length, d).sum(2).transpose(1, 2)
    out = torch.zeros(like.shape[:2] + (d,), device="cuda")
    out[place[there]] = x[there]
    return out.to(like.dtype)


def _fades(s, there):
    """exp(a (t - s)) for s <= t (heads, length, length), exp(a (t + 1)) (heads, length), exp(a (last - t)) (sequences, heads, length), exp(a tokens)."""
    a = s["log_decay"].float()
    t = torch.arange(there.shape[1], device="cuda", dtype=torch.float32)
    n = there.sum(1).float()
    ago = t[:, None] - t[None]
    between = torch.where(ago >= 0, torch.exp(a[:, None, None] * ago.clamp_min(0)), 0.0)
    left = torch.where(there[:, None], torch.exp(a[:, None] * (n[:, None, None] - 1 - t).clamp_min(0)), 0.0)
    return between, torch.exp(a[:, None] * (t + 1)), left, torch.exp(a * n[:, None])


def _plain_decay(s):
    heads = s["case"]["heads"]
    place, there = _places(s)
    Q, K, V = (_by_head(s[n], heads, place, there) for n in "QKV")
    between, since, left, whole = _fades(s, there)
    O = (Q @ K.transpose(2, 3).contiguous() * between) @ V
    after = None
    if s["state"] is not None:
        O = O + (Q @ s["state"]) * since[..., None]
        after = s["state"] * whole[..., None, None] + (K * left[..., None]).transpose(2, 3).contiguous() @ V
    like = s["Q"].new_empty(s["Q"].shape[:2] + (V.shape[3],))
    return {"O": _by_row(O * s["scale"], like, place, there), "state": after}


def _plain_decay_grads(s):
    heads = s["case"]["heads"]
    place, there = _places(s)
    Q, K, V, dO = (_by_head(s[n], heads, place, there) for n in ("Q", "K", "V", "dO"))
    between, since, left, whole = _fades(s, there)
    dO = dO * s["scale"]
    P = (dO @ V.transpose(2, 3).contiguous()).mul_(between)
    dQ, dK = P @ K, P.transpose(2, 3).contiguous() @ Q
    P = (Q @ K.transpose(2, 3).contiguous()).mul_(between)
    dV, before = P.transpose(2, 3).contiguous() @ dO, None
    if s["state"] is not None:
        dQ = dQ + (dO @ s["state"].transpose(2, 3).contiguous()) * since[..., None]
        dK = dK + (V @ s["dstate"].transpose(2, 3).contiguous()) * left[..., None]
        dV = dV + (K @ s["dstate"]) * left[..., None]
        before = s["dstate"] * whole[..., None, None] + (Q * since[..., None]).transpose(2, 3).contiguous() @ dO
    return {"dQ": _by_row(dQ, s["Q"], place, there), "dK": _by_row(dK, s["K"], place, there), "dV": _by_row(dV, s["V"], place, there), "dstate": before}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------------

def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        if case["kind"].startswith("embed"):
            return _exact_embed(s)
        return _exact_head(s) if case["kind"].startswith("head") else _exact_decay(s)


def _exact_embed(s):
    """As a product with the matrix that has a one where a row's token is, some of the vocabulary at a time."""
    c, parts = s["case"], []
    X = torch.zeros((c["rows"], c["d"]), dtype=torch.float64, device="cuda")
    for at in range(0, c["vocab"], 8192):
        ids = torch.arange(at, min(c["vocab"], at + 8192), device="cuda")
        one = (s["token"][:, None] == ids[None]).double()
        if c["kind"] == "embed":
            X += c["scale"] * torch.matmul(one, s["W"][ids].double())
        else:
            parts.append(c["scale"] * torch.matmul(one.t().contiguous(), s["dX"].double()))
    return {"X": X} if c["kind"] == "embed" else {"dW": torch.cat(parts)}


def _exact_head(s):
    c = s["case"]
    d, rot = c["d"], c["rot"]
    # a head's rotation as a matrix of complex numbers: the pair (a, b) is a + ib, turned by exp(i angle)
    pair = torch.arange(rot // 2, device="cuda")
    first, second = (2 * pair, 2 * pair + 1) if c["adjacent"] else (pair, pair + rot // 2)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["position"].double()[:, None] * torch.exp(-pair.double() * (2.0 * math.log(_BASE) / max(rot, 1))))[:, None]

    def turned(x, by):
        z = torch.complex(x[..., first], x[..., second]) * by
        x = x.clone()
        x[..., first], x[..., second] = z.real, z.imag
        return x

    out = {}
    for n, w in (("Q", s["w_q"].double()), ("K", s["w_k"].double())):
        x = s[n].double()
        dev = (x.pow(2).sum(-1, keepdim=True) / d + _EPS).sqrt()
        if c["kind"] == "head_norm":
            out[n + "out"] = turned(x / dev * w, turn)
        else:
            dy = turned(s["d%sout" % n].double(), turn.conj())
            out["d" + n] = dy * w / dev - x * (dy * w * x).sum(-1, keepdim=True) / (d * dev.pow(3))
            out["dw_" + n.lower()] = (dy * x / dev).flatten(0, 1).sum(0)
    return out


def _exact_decay(s):
    """The recurrence itself, token by token, all sequences and heads at once."""
    c = s["case"]
    heads, group = c["heads"], c["heads"] // c["kv_heads"]
    lengths = torch.tensor(_lengths(c))
    start = torch.cumsum(lengths, 0) - lengths
    row = lambda t: ((t * c["sequences"] + torch.arange(c["sequences"])) if c["rows"] == "by position" else start + t).cuda()  # noqa: E731
    live = [torch.nonzero(lengths > t)[:, 0].cuda() for t in range(c["length"])]
    lam = torch.exp(s["log_decay"].double())[:, None, None]
    Q, K, V = (s[n].double() for n in "QKV")
    shared = torch.arange(heads, device="cuda") // group
    S = s["state"].double().clone() if s["state"] is not None else torch.zeros((c["sequences"], heads, c["dk"], c["dv"]), dtype=torch.float64, device="cuda")
    grads = c["kind"] == "decay_grads"
    O = torch.zeros(s["Q"].shape[:2] + (c["dv"],), dtype=torch.float64, device="cuda")
    dQ, dK, dV = torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)
    dO = s["dO"].double() * s["scale"] if grads else None
    for t in range(c["length"]):
        b, r = live[t], row(t)[live[t]]
        S[b] = lam * S[b] + K[r][:, shared, :, None] * V[r][:, shared, None, :]
        if grads:
            dQ[r] = (S[b] * dO[r][:, :, None, :]).sum(3)
        else:
            O[r] = s["scale"] * (S[b] * Q[r][:, :, :, None]).sum(2)
    if not grads:
        return {"O": O, "state": S if s["state"] is not None else None}
    G = s["dstate"].double().clone() if s["dstate"] is not None else torch.zeros_like(S)
    for t in reversed(range(c["length"])):
        b, r = live[t], row(t)[live[t]]
        G[b] += Q[r][:, :, :, None] * dO[r][:, :, None, :]
        k, v = (G[b] * V[r][:, shared, None, :]).sum(3), (G[b] * K[r][:, shared, :, None]).sum(2)
        dK[r], dV[r] = k.view(len(b), -1, group, c["dk"]).sum(2), v.view(len(b), -1, group, c["dv"]).sum(2)
        G[b] = lam * G[b]
    return {"dQ": dQ, "dK": dK, "dV": dV, "dstate": G if s["dstate"] is not None else None}
