"""Oracle of the embedding, the norms and rotation of queries and keys, and attention with decay: their definitions in numpy and 64 bits, and the
gradients by the chain rule.

Every function also gives, under "size", the same expressions evaluated on absolute values: the size of what is added up for an entry, to which rounding
errors of the sums are relative.
"""
import numpy as np


def _f(a):
    return np.asarray(a, np.float64)


def embed_forward(token, W, scale=1.0):
    token, W = np.asarray(token), _f(W)
    there = (token >= 0) & (token < W.shape[0])
    return np.where(there[:, None], scale * W[np.where(there, token, 0)], 0.0)


def embed_backward(token, dX, vocab, scale=1.0, was=None):
    """dict of dW and its size; was: what dW is added to."""
    token, dX = np.asarray(token), _f(dX)
    dW, size = np.zeros((vocab, dX.shape[1])), np.zeros((vocab, dX.shape[1]))
    for i in np.flatnonzero((token >= 0) & (token < vocab)):
        dW[token[i]] += scale * dX[i]
        size[token[i]] += abs(scale) * np.abs(dX[i])
    if was is not None:
        dW, size = dW + _f(was), size + np.abs(_f(was))
    return {"dW": dW, "size": {"dW": size}}


def _pairs(rot, adjacent):
    p = np.arange(rot // 2)
    return (2 * p, 2 * p + 1) if adjacent else (p, p + rot // 2)


def _turn(x, position, rot, base, adjacent, back=False, size=False):
    """x (rows, heads, d) with its pairs turned; size: |x| turned by |cos| and |sin|."""
    x = x.copy()
    if position is None or rot == 0:
        return x
    a, b = _pairs(rot, adjacent)
    angle = (np.asarray(position, np.longdouble)[:, None] * np.longdouble(base) ** (-2 * np.arange(rot // 2, dtype=np.longdouble) / rot)) % (2 * np.longdouble(np.pi))
    c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
    if back:
        s = -s
    if size:
        c, s = np.abs(c), np.abs(s)
        x[..., a], x[..., b] = x[..., a] * c + x[..., b] * s, x[..., b] * c + x[..., a] * s
    else:
        x[..., a], x[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return x


def head_forward(x, w=None, position=None, rot=0, base=10000.0, adjacent=False, norm=True, eps=1e-6):
    """(out, size of it) for x (rows, heads, d)."""
    y = _f(x)
    if norm:
        y = y / np.sqrt(np.mean(y * y, -1, keepdims=True) + eps) * (1.0 if w is None else _f(w))
    return _turn(y, position, rot, base, adjacent), _turn(np.abs(y), position, rot, base, adjacent, size=True)


def head_backward(x, up, w=None, position=None, rot=0, base=10000.0, adjacent=False, norm=True, eps=1e-6):
    """dict of dx, dw and their sizes."""
    x, up = _f(x), _f(up)
    dy = _turn(up, position, rot, base, adjacent, back=True)
    big = _turn(np.abs(up), position, rot, base, adjacent, size=True)
    if not norm:
        return {"dx": dy, "size": {"dx": big}}
    w = np.ones(x.shape[-1]) if w is None else _f(w)
    r = 1.0 / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    hat, t, ts = x * r, dy * w, big * np.abs(w)
    return {"dx": r * (t - hat * np.mean(t * hat, -1, keepdims=True)), "dw": (dy * hat).sum((0, 1)),
            "size": {"dx": r * (ts + np.abs(hat) * np.mean(ts * np.abs(hat), -1, keepdims=True)), "dw": (big * np.abs(hat)).sum((0, 1))}}


def decay(Q, K, V, rows_of, log_decay=None, scale=1.0, state=None, dO=None, dstate=None):
    """Q (rows, heads, dk), K (rows, kv heads, dk), V (rows, kv heads, dv); rows_of: for each sequence its tokens' rows in order; state (sequences, heads, dk, dv) in
    front.  dict of O and state, with dO or dstate also of dQ, dK, dV and dstate in front; rows of no sequence are zeros."""
    Q, K, V = _f(Q), _f(K), _f(V)
    heads, share = Q.shape[1], Q.shape[1] // K.shape[1]
    dk, dv, n = Q.shape[2], V.shape[2], len(rows_of)
    with np.errstate(invalid="ignore"):
        lam = np.ones(heads) if log_decay is None else np.exp(np.asarray(log_decay, np.float64))
    lam = lam[:, None, None]
    zero = np.zeros((n, heads, dk, dv))
    S0 = zero if state is None else _f(state)
    grads = dO is not None or dstate is not None
    out = {"O": np.zeros(Q.shape[:2] + (dv,)), "state": S0.copy()}
    size = {"O": np.zeros_like(out["O"]), "state": np.abs(S0)}
    if grads:
        up = np.zeros_like(out["O"]) if dO is None else _f(dO)
        G0 = zero if dstate is None else _f(dstate)
        for name, like in (("dQ", Q), ("dK", K), ("dV", V)):
            out[name], size[name] = np.zeros(like.shape), np.zeros(like.shape)
        out["dstate"], size["dstate"] = G0.copy(), np.abs(G0)
    for b, rows in enumerate(rows_of):
        for sign in (False, True):                                          # the values, then their sizes
            to = size if sign else out
            f = np.abs if sign else (lambda a: a)
            S, c = f(S0[b]), abs(scale) if sign else scale
            for r in rows:
                k, v = np.repeat(f(K[r]), share, 0), np.repeat(f(V[r]), share, 0)
                S = lam * S + k[:, :, None] * v[:, None, :]
                to["O"][r] = c * (f(Q[r])[:, :, None] * S).sum(1)
                if grads:
                    to["dQ"][r] = c * (S * f(up[r])[:, None, :]).sum(2)
            to["state"][b] = S
            if not grads:
                continue
            G = f(G0[b])
            for r in reversed(rows):
                k, v = np.repeat(f(K[r]), share, 0), np.repeat(f(V[r]), share, 0)
                G = G + c * f(Q[r])[:, :, None] * f(up[r])[:, None, :]
                to["dK"][r] = (G * v[:, None, :]).sum(2).reshape(-1, share, dk).sum(1)
                to["dV"][r] = (G * k[:, :, None]).sum(1).reshape(-1, share, dv).sum(1)
                G = lam * G
            to["dstate"][b] = G
    out["size"] = size
    return out


def decay_rows(sequences, length, seq_step, token_step, offset=None, rows=None):
    """Rows of each sequence's tokens."""
    if offset is None:
        return [[b * seq_step + t * token_step for t in range(length)] for b in range(sequences)]
    found = []
    for b in range(sequences):
        lo = min(max(int(offset[b]), 0), rows)
        hi = min(max(int(offset[b + 1]), lo), rows)
        found.append(list(range(lo, min(hi, lo + length))))
    return found
