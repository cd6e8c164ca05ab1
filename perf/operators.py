"""The ends of a language model around STL layers, as cases to time: the step between two blocks (norm of the block's output,
gate, residual sum, norm before the next block) and the loss over a vocabulary, from labels and from a teacher's top logits, with
their gradients.

A case is one `kind` of call and its sizes:

  residual        stl_residual_norm_forward (a token at a time, or a prompt)
  residual_grads  stl_residual_norm_backward
  loss            stl_vocab_loss_forward (scoring: no gradients)
  grads           stl_vocab_loss_backward (a training step: losses and gradients in one call)

`top` > 0 gives the loss a teacher's `top` logits a row; `label` says whether it has labels.  Values: activations ~ N(0, 1) as they
leave a norm, vocabulary rows ~ N(0, 4/d) (logits of a deviation of 2), the label's row added into its token's activation so that
labels have the probabilities, from a chance hit to nearly 1, that a trained model gives them.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _residual(name, kind, dtype, rows, n, norm="rms", per_gate=0, post=True, bias=False, skip=1.0, scale=1.0):
    """per_gate: rows that share a row of the gate, 0: all of them."""
    c = {"kind": kind, "dtype": dtype, "rows": rows, "n": n, "norm": norm, "per_gate": per_gate, "post": post, "bias": bias, "skip": skip,
         "scale": scale}
    return {"name": name, **c} if name else c


def _loss(name, kind, dtype, rows, d, vocab, label=True, top=0, tau=1.0, ignored=0.0):
    """ignored: share of the rows without a label."""
    c = {"kind": kind, "dtype": dtype, "rows": rows, "d": d, "vocab": vocab, "label": label, "top": top, "tau": tau, "ignored": ignored}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token on its way through a serving loop: a few kilobytes, so the launch counts
        _residual("residual_token", "residual", "bf16", 1, 4096),
        # a prompt of the benchmark's row count and width, gate per channel
        _residual("residual_prompt", "residual", "bf16", 8192, 4096, scale=0.5),
        # images of 197 tokens with a gate for each image, layer norms with offsets, trained
        _residual("residual_images", "residual_grads", "bf16", 64 * 197, 768, norm="layer", per_gate=197, bias=True),
        # the same step of the large model, backward
        _residual("residual_train", "residual_grads", "bf16", 8192, 4096),
        # an odd width in fp32, without the norm behind the block
        _residual("residual_odd_f32", "residual_grads", "f32", 1001, 1021, norm="layer", post=False, bias=True, skip=0.75),
        # scoring the few tokens of a short answer: reading the vocabulary's rows is the work
        _loss("loss_few_rows", "loss", "bf16", 16, 4096, 65536),
        # scoring a prompt
        _loss("loss_prompt", "loss", "bf16", 1024, 2048, 32000),
        # comparing a student with a teacher's stored top logits, an odd vocabulary
        _loss("distill_score", "loss", "bf16", 777, 1024, 50001, label=False, top=16, tau=2.0),
        # the training step of a classifier head, 768 -> 1000 classes, in fp32
        _loss("grads_classes_f32", "grads", "f32", 2048, 768, 1000),
        # fine-tuning on answers: the prompts' tokens have no label, an odd count of tokens
        _loss("grads_answers", "grads", "bf16", 3001, 1024, 50001, ignored=0.6),
        # an STL student trained on labels and its dense teacher's top logits together
        _loss("grads_distill", "grads", "bf16", 2048, 2048, 32000, top=64, tau=2.0),
        # the training step of a large model's head
        _loss("grads_large", "grads", "bf16", 4096, 4096, 131072),
    ]


def _log_int(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], uniform in its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(int(round(v / step)) * step, -(-lo // step) * step), hi // step * step)


def draw(rng):
    kind = rng.choice(["residual", "residual_grads", "loss", "grads", "grads"])
    odd = rng.random() < 0.4
    if kind.startswith("residual"):
        rows, n = _log_int(rng, 1, 16384), _log_int(rng, 64, 8192, 1 if odd else 64)
        rows = max(1, min(rows, 8192 * 4096 // n))
        per = rng.choice([0, 0, 1, 197, 50])
        return _residual(None, kind, rng.choice(["bf16", "bf16", "f32"]) if rows * n <= 1 << 24 else "bf16", rows, n, rng.choice(["rms", "layer"]), min(per, rows),
                         rng.random() < 0.7, rng.random() < 0.4, rng.choice([1.0, 0.75]), rng.choice([1.0, 0.5]))
    rows = _log_int(rng, 1, 8192)
    d = _log_int(rng, 64, 4096, 1 if odd and rng.random() < 0.3 else 64)
    vocab = _log_int(rng, 1000, 131072, 1 if odd else 128)
    dtype = "bf16"
    if rng.random() < 0.15 and rows * d * vocab < 1 << 35:
        dtype = "f32"
    most = 1 << 40                                                    # half the largest listed case
    while rows * d * vocab > most:
        rows = (rows + 1) // 2
    label, top = rng.choice([(True, 0), (True, 0), (True, 32), (False, 64), (True, 100), (False, 5)])
    return _loss(None, kind, dtype, rows, d, vocab, label, min(top, vocab), rng.choice([1.0, 2.0, 4.0]) if top else 1.0,
                 rng.choice([0.0, 0.0, 0.3, 0.8]) if label else 0.0)


def _without_label(case):
    return int(case["rows"] * case["ignored"])


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"].startswith("residual"):
        rows, n = case["rows"], case["n"]
        gates = -(-rows // (case["per_gate"] or rows))
        vectors = (1 + gates + (1 if case["post"] else 0) + (2 if case["bias"] and case["post"] else 1 if case["bias"] else 0)) * n
        if case["kind"] == "residual":
            return {"bytes": size * (4 * rows * n + vectors), "flops": 16 * rows * n}
        return {"bytes": size * (6 * rows * n + vectors) + 4 * vectors, "flops": 40 * rows * n}
    # a row without a label still has its teacher's logits
    rows = case["rows"] - (0 if case["top"] else _without_label(case))
    d, vocab = case["d"], case["vocab"]
    passes, products = (1, 1) if case["kind"] == "loss" else (2, 3)
    return {"bytes": size * passes * (rows + vocab) * d + case["rows"] * (12 * case["top"] + 16), "flops": 2 * products * rows * vocab * d}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    if case["kind"].startswith("residual"):
        return _prepare_residual(case, randn, dt)
    rows, d, vocab, top = case["rows"], case["d"], case["vocab"], case["top"]
    W = (randn(vocab, d) * (2.0 / math.sqrt(d))).to(dt)
    label = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    # logit of the label: up to 16 above the others'
    lift = torch.rand((rows, 1), generator=g, device="cuda") * 4.0
    X = (randn(rows, d) + lift * W[label].float()).to(dt)
    s = {"case": dict(case), "X": X, "W": W, "label": None, "top_id": None, "top_logit": None, "dlabel": None, "dtop": None}
    if top:
        # the label first, then other rows of the vocabulary; lists are of different lengths (-1 behind their end)
        stride = torch.randint(1, max(2, vocab // top), (rows, 1), generator=g, device="cuda")
        at = torch.arange(top, device="cuda")
        ids = (label[:, None] + at * stride) % vocab
        length = top - torch.randint(0, max(1, top // 4), (rows, 1), generator=g, device="cuda")
        s["top_id"] = torch.where(at < length, ids, -1)
        s["top_logit"] = (8.0 - randn(rows, top).abs().cumsum(1) * (8.0 / top)).contiguous()
        s["dtop"] = torch.full((rows,), 1.0 / rows, device="cuda")
    if case["label"]:
        none = torch.randperm(rows, generator=g, device="cuda")[:_without_label(case)]
        s["label"] = label.index_fill(0, none, -100)
        s["dlabel"] = torch.full((rows,), 1.0 / (rows - _without_label(case)), device="cuda")
    if own:
        import paper_2503_12211_amd as stl
        s["prob"] = stl.VocabProblem(rows, d, vocab, top, case["tau"], stl.STL_BF16 if dt == torch.bfloat16 else stl.STL_F32)
        s["ws_bytes"] = stl.stl_vocab_loss_workspace_bytes(s["prob"], stl.STL_OP_FORWARD if case["kind"] == "loss" else stl.STL_OP_BACKWARD)
        s["ws"] = torch.empty(max(s["ws_bytes"], 16), dtype=torch.uint8, device="cuda")
    return s


def _prepare_residual(case, randn, dt):
    rows, n = case["rows"], case["n"]
    per = case["per_gate"] or rows
    s = {"case": dict(case), "per": per, "H": (randn(rows, n) * 1.5 + 0.25).to(dt), "gate": (0.3 + 0.2 * randn(-(-rows // per), n)).to(dt),
         "w_pre": (1.0 + 0.1 * randn(n)).to(dt), "w_post": None, "b_post": None, "b_pre": None}
    if case["post"]:
        s["w_post"] = (1.0 + 0.1 * randn(n)).to(dt)
    if case["bias"]:
        s["b_pre"] = (0.1 * randn(n)).to(dt)
        s["b_post"] = (0.1 * randn(n)).to(dt) if case["post"] else None
    s["X"] = (randn(rows, n) * 2.0).to(dt)
    if case["kind"] == "residual_grads":
        # X is the stream behind the residual sum here: the step's input is not needed any more
        s["dXout"], s["dZ"] = randn(rows, n).to(dt), randn(rows, n).to(dt)
    if own:
        import paper_2503_12211_amd as stl
        s["prob"] = stl.ResidualProblem(rows, n, per, case["skip"], case["scale"], 1e-6, stl.STL_BF16 if dt == torch.bfloat16 else stl.STL_F32)
        s["flags"] = stl.STL_FLAG_PRE_NORM | (stl.STL_FLAG_POST_NORM if case["post"] else 0) | (stl.STL_FLAG_CENTER if case["norm"] == "layer" else 0)
        s["ws_bytes"] = stl.stl_residual_norm_workspace_bytes(s["prob"], s["flags"])
        s["ws"] = torch.empty(max(s["ws_bytes"], 16), dtype=torch.uint8, device="cuda")
    return s


def run(s):
    kind = s["case"]["kind"]
    if kind == "residual":
        return _own_residual(s) if own else _plain_residual(s)
    if kind == "residual_grads":
        return _own_residual_grads(s) if own else _plain_residual_grads(s)
    return _own_loss(s) if own else _plain_loss(s)


# ---- the framework's operators ----------------------------------------------------------------------------------------------------

def _own_residual(s):
    import paper_2503_12211_amd as stl
    Xout, Z = torch.empty_like(s["X"]), torch.empty_like(s["X"])
    stl.stl_residual_norm_forward(s["prob"], s["X"], s["H"], s["gate"], s["w_post"], s["b_post"], s["w_pre"], s["b_pre"], Xout, Z, s["flags"])
    return {"Xout": Xout, "Z": Z}


def _own_residual_grads(s):
    import paper_2503_12211_amd as stl
    dX, dH = torch.empty_like(s["X"]), torch.empty_like(s["X"])
    sums = {"d" + k: torch.empty(s[k].shape, dtype=torch.float32, device="cuda") if s[k] is not None else None for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
    stl.stl_residual_norm_backward(s["prob"], s["X"], s["H"], s["gate"], s["w_post"], s["b_post"], s["w_pre"], s["dXout"], s["dZ"], dX, dH,
                                   sums["dgate"], sums["dw_post"], sums["db_post"], sums["dw_pre"], sums["db_pre"], 0, s["ws"], s["ws_bytes"], s["flags"])
    return {"dX": dX, "dH": dH, **sums}


def _own_loss(s):
    import paper_2503_12211_amd as stl
    rows = s["case"]["rows"]
    label_loss = torch.empty(rows, device="cuda") if s["label"] is not None else None
    top_loss = torch.empty(rows, device="cuda") if s["top_id"] is not None else None
    inputs = (s["prob"], s["X"], s["W"], s["label"], s["top_id"], s["top_logit"])
    if s["case"]["kind"] == "loss":
        stl.stl_vocab_loss_forward(*inputs, label_loss, top_loss, s["ws"], s["ws_bytes"])
        return {"label_loss": label_loss, "top_loss": top_loss}
    dX, dW = torch.empty_like(s["X"]), torch.empty_like(s["W"])
    stl.stl_vocab_loss_backward(*inputs, s["dlabel"], s["dtop"], label_loss, top_loss, dX, dW, s["ws"], s["ws_bytes"])
    return {"label_loss": label_loss, "top_loss": top_loss, "dX": dX, "dW": dW}


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ---------------------------------------------------------

def _plain_norm(v, center):
    if center:
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6)
    return v * r, r


def _plain_norm_back(t, hat, r, center):
    t = t - hat * (t * hat).mean(1, keepdim=True)
    return r * (t - t.mean(1, keepdim=True)) if center else r * t


def _gate_rows(s):
    return s["gate"].float().repeat_interleave(s["per"], 0)[:s["case"]["rows"]]


def _branch(s):
    """The block's output behind its norm, and that norm's parts."""
    H = s["H"].float()
    if s["w_post"] is None:
        return H, None, None
    hat, r = _plain_norm(H, s["case"]["norm"] == "layer")
    u = hat * s["w_post"].float()
    return (u + s["b_post"].float() if s["b_post"] is not None else u), hat, r


def _plain_residual(s):
    c, dt = s["case"], s["X"].dtype
    Xout = c["skip"] * s["X"].float() + c["scale"] * _gate_rows(s) * _branch(s)[0]
    Z = _plain_norm(Xout, c["norm"] == "layer")[0] * s["w_pre"].float()
    if s["b_pre"] is not None:
        Z = Z + s["b_pre"].float()
    return {"Xout": Xout.to(dt), "Z": Z.to(dt)}


def _plain_residual_grads(s):
    c, dt = s["case"], s["X"].dtype
    center = c["norm"] == "layer"
    dZ = s["dZ"].float()
    hat, r = _plain_norm(s["X"].float(), center)
    d = s["dXout"].float() + _plain_norm_back(dZ * s["w_pre"].float(), hat, r, center)
    u, h_hat, h_r = _branch(s)
    d_gate = torch.zeros(s["gate"].shape, device="cuda").index_add_(0, torch.arange(c["rows"], device="cuda") // s["per"], c["scale"] * u * d)
    du = c["scale"] * _gate_rows(s) * d
    post = s["w_post"] is not None
    dH = _plain_norm_back(du * s["w_post"].float(), h_hat, h_r, center) if post else du
    return {"dX": (c["skip"] * d).to(dt), "dH": dH.to(dt), "dgate": d_gate, "dw_post": (du * h_hat).sum(0) if post else None,
            "db_post": du.sum(0) if s["b_post"] is not None else None, "dw_pre": (dZ * hat).sum(0),
            "db_pre": dZ.sum(0) if s["b_pre"] is not None else None}


def _plain_loss(s):
    c, dt, tau = s["case"], s["X"].dtype, s["case"]["tau"]
    X, W = s["X"].float(), s["W"].float()
    rows = X.shape[0]
    z = X @ W.t()
    out, dz = {"label_loss": None, "top_loss": None}, 0.0
    gradients = c["kind"] == "grads"
    if s["label"] is not None:
        has = (s["label"] >= 0) & (s["label"] < W.shape[0])
        label = s["label"].clamp(0, W.shape[0] - 1)[:, None]
        m = z.amax(1, keepdim=True)
        p = (z - m).exp_()
        total = p.sum(1, keepdim=True)
        out["label_loss"] = torch.where(has, (total.log() + m - z.gather(1, label))[:, 0], 0.0)
        if gradients:
            coef = torch.where(has, s["dlabel"], 0.0)[:, None]
            dz = p.mul_(coef / total).scatter_add_(1, label, -coef)
    if s["top_id"] is not None:
        there = (s["top_id"] >= 0) & (s["top_id"] < W.shape[0])
        ids = s["top_id"].clamp(0, W.shape[0] - 1)
        y = torch.where(there, s["top_logit"], -math.inf) / tau
        q = (y - y.amax(1, keepdim=True)).exp()
        log_q = y - y.amax(1, keepdim=True) - q.sum(1, keepdim=True).log()
        q = q / q.sum(1, keepdim=True)
        m = z.amax(1, keepdim=True)
        p = ((z - m) / tau).exp_()
        total = p.sum(1, keepdim=True)
        log_p = (z.gather(1, ids) - m) / tau - total.log()
        out["top_loss"] = torch.where(there, q * (log_q - log_p), 0.0).sum(1)
        if gradients:
            coef = s["dtop"][:, None] / tau
            dz = p.mul_(coef / total).scatter_add_(1, ids, -coef * q) + dz
    if gradients:
        out["dX"], out["dW"] = (dz @ W).to(dt), (dz.t() @ X).to(dt)
    return out


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------------

def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        return _exact_residual(s) if case["kind"].startswith("residual") else _exact_loss(s)


def _f64(v):
    return None if v is None else v.double()


def _exact_residual(s):
    c = s["case"]
    w_post, b_post, w_pre, b_pre, gate = (_f64(s[k]) for k in ("w_post", "b_post", "w_pre", "b_pre", "gate"))
    group = torch.arange(c["rows"], device="cuda") // s["per"]

    def statistics(v):                                             # mean and deviation of every row
        mu = v.sum(1, keepdim=True) / c["n"] if c["norm"] == "layer" else torch.zeros_like(v[:, :1])
        return mu, ((v - mu).pow(2).sum(1, keepdim=True) / c["n"] + 1e-6).sqrt()

    H, X = s["H"].double(), s["X"].double()
    mu, dev = statistics(H)
    u = (H - mu) / dev * w_post + (b_post if b_post is not None else 0.0) if w_post is not None else H
    if c["kind"] == "residual":
        out = c["skip"] * X + c["scale"] * gate[group] * u
        mu, dev = statistics(out)
        return {"Xout": out, "Z": (out - mu) / dev * w_pre + (b_pre if b_pre is not None else 0.0)}

    def through(dy, v, mu, dev):                                   # gradient of sum dy (v - mu) / dev in v, written out
        a = dy / dev
        if c["norm"] == "layer":
            a = a - a.sum(1, keepdim=True) / c["n"]
        return a - (v - mu) * (dy * (v - mu)).sum(1, keepdim=True) / (c["n"] * dev.pow(3))

    dZ = s["dZ"].double()
    mu_x, dev_x = statistics(X)
    d = s["dXout"].double() + through(dZ * w_pre, X, mu_x, dev_x)
    groups = gate.shape[0]
    lead = torch.zeros((groups * s["per"], c["n"]), dtype=torch.float64, device="cuda")
    lead[:c["rows"]] = u * d
    du = c["scale"] * gate[group] * d
    post = w_post is not None
    return {"dX": c["skip"] * d, "dH": through(du * w_post, H, mu, dev) if post else du, "dgate": c["scale"] * lead.view(groups, s["per"], c["n"]).sum(1),
            "dw_post": (du * (H - mu) / dev).sum(0) if post else None, "db_post": du.sum(0) if b_post is not None else None,
            "dw_pre": (dZ * (X - mu_x) / dev_x).sum(0), "db_pre": dZ.sum(0) if b_pre is not None else None}


def _exact_loss(s):
    c, tau = s["case"], s["case"]["tau"]
    W = s["W"].double()
    n_row, vocab = s["X"].shape[0], W.shape[0]
    grads = c["kind"] == "grads"
    dW, parts = torch.zeros_like(W) if grads else None, {"label_loss": [], "top_loss": [], "dX": []}
    for at in range(0, n_row, 1024):                                # rows are independent of each other
        rows = slice(at, min(n_row, at + 1024))
        X = s["X"][rows].double()
        z = torch.matmul(X, W.transpose(0, 1))
        dz = torch.zeros_like(z) if grads else None
        here = torch.arange(X.shape[0], device="cuda")
        if s["label"] is not None:
            label = s["label"][rows]
            have = here[(label >= 0) & (label < vocab)]
            log_p = torch.log_softmax(z[have], 1)
            loss = torch.zeros(X.shape[0], dtype=torch.float64, device="cuda")
            loss[have] = -log_p[torch.arange(len(have), device="cuda"), label[have]]
            parts["label_loss"].append(loss)
            if grads:
                d = log_p.exp()
                d[torch.arange(len(have), device="cuda"), label[have]] -= 1.0
                dz[have] += s["dlabel"][rows][have].double()[:, None] * d
        if s["top_id"] is not None:
            ids = s["top_id"][rows]
            there = (ids >= 0) & (ids < vocab)
            target = torch.zeros_like(z)                             # the teacher's distribution over the whole vocabulary
            y = s["top_logit"][rows].double() / tau
            q = torch.softmax(torch.where(there, y, torch.full_like(y, -math.inf)), 1)
            target.scatter_add_(1, torch.where(there, ids, 0), torch.where(there, q, 0.0))
            log_p = torch.log_softmax(z / tau, 1)
            parts["top_loss"].append(torch.where(target > 0, target * (target.clamp_min(1e-300).log() - log_p), 0.0).sum(1))
            if grads:
                dz += s["dtop"][rows].double()[:, None] / tau * (log_p.exp() - target)
        if grads:
            parts["dX"].append(torch.matmul(dz, W))
            dW += torch.matmul(dz.transpose(0, 1), X)
    out = {k: torch.cat(parts[k]) if parts[k] else None for k in ("label_loss", "top_loss")}
    return {**out, "dX": torch.cat(parts["dX"]), "dW": dW} if grads else out
