"""Oracle of the residual step and the vocabulary loss: their definitions in numpy and 64 bits, and the gradients by the chain rule.

Every function also gives, where a caller asks with `scale=True`, the same expression evaluated on absolute values: the size of what is
added up for an entry, to which rounding errors of the sums are relative.
"""
import numpy as np


def _norm(v, center, eps):
    mu = v.mean(1, keepdims=True) if center else np.zeros((v.shape[0], 1))
    r = 1.0 / np.sqrt(np.mean((v - mu) ** 2, 1, keepdims=True) + eps)
    return (v - mu) * r, r


def _norm_size(v, center, eps):
    """The normalised row on absolute values: what is subtracted counts."""
    return (np.abs(v) + np.abs(v.mean(1, keepdims=True)) * center) * _norm(v, center, eps)[1]


def _norm_backward(t, hat, r, center):
    g = t - hat * np.mean(t * hat, 1, keepdims=True)
    if center:
        g = g - t.mean(1, keepdims=True)
    return r * g


def _vec(w, n, default):
    return np.full(n, default) if w is None else np.asarray(w, np.float64)


def _gate(gate, per, rows, n):
    return np.ones((rows, n)) if gate is None else np.asarray(gate, np.float64)[np.arange(rows) // per]


def residual_forward(X, H, gate=None, per=None, w_post=None, b_post=None, w_pre=None, b_pre=None, post=True, pre=True, center=False, skip=1.0,
                     scale=1.0, eps=1e-6):
    """(Xout, Z); Z is None without `pre`."""
    X, H = np.asarray(X, np.float64), np.asarray(H, np.float64)
    rows, n = X.shape
    u = _norm(H, center, eps)[0] * _vec(w_post, n, 1.0) + _vec(b_post, n, 0.0) if post else H
    Xout = skip * X + scale * _gate(gate, per or rows, rows, n) * u
    return Xout, (_norm(Xout, center, eps)[0] * _vec(w_pre, n, 1.0) + _vec(b_pre, n, 0.0) if pre else None)


def residual_backward(Xout, H, dXout, dZ, gate=None, per=None, w_post=None, b_post=None, w_pre=None, post=True, pre=True, center=False, skip=1.0,
                      scale=1.0, eps=1e-6):
    """dict of dX, dH, dgate, dw_post, db_post, dw_pre, db_pre, and under "size" the absolute terms behind each."""
    Xout, H = np.asarray(Xout, np.float64), np.asarray(H, np.float64)
    rows, n = H.shape
    per = per or rows
    d = np.zeros((rows, n)) if dXout is None else np.asarray(dXout, np.float64)
    size = np.abs(d)
    out, sizes = {}, {}
    if pre:
        dZ = np.zeros((rows, n)) if dZ is None else np.asarray(dZ, np.float64)
        hat, r = _norm(Xout, center, eps)
        t = dZ * _vec(w_pre, n, 1.0)
        d = d + _norm_backward(t, hat, r, center)
        ah = _norm_size(Xout, center, eps)
        size = size + r * (np.abs(t) + ah * np.mean(np.abs(t) * ah, 1, keepdims=True) + center * np.mean(np.abs(t), 1, keepdims=True))
        out["dw_pre"], out["db_pre"] = (dZ * hat).sum(0), dZ.sum(0)
        sizes["dw_pre"], sizes["db_pre"] = (np.abs(dZ) * ah).sum(0), np.abs(dZ).sum(0)
    out["dX"], sizes["dX"] = skip * d, abs(skip) * size
    g = _gate(gate, per, rows, n)
    du, du_size = scale * g * d, np.abs(scale * g) * size
    u, u_size = H, np.abs(H)
    if post:
        hh, rh = _norm(H, center, eps)
        w = _vec(w_post, n, 1.0)
        u = hh * w + _vec(b_post, n, 0.0)
        th, ts = du * w, du_size * np.abs(w)
        u_size = _norm_size(H, center, eps) * np.abs(w) + np.abs(_vec(b_post, n, 0.0))
        out["dH"] = _norm_backward(th, hh, rh, center)
        ah = _norm_size(H, center, eps)
        sizes["dH"] = rh * (ts + ah * np.mean(ts * ah, 1, keepdims=True) + center * np.mean(ts, 1, keepdims=True))
        out["dw_post"], out["db_post"] = (du * hh).sum(0), du.sum(0)
        sizes["dw_post"], sizes["db_post"] = (du_size * ah).sum(0), du_size.sum(0)
    else:
        out["dH"], sizes["dH"] = du, du_size
    if gate is not None:
        out["dgate"], sizes["dgate"] = np.zeros(np.shape(gate)), np.zeros(np.shape(gate))
        np.add.at(out["dgate"], np.arange(rows) // per, scale * u * d)
        np.add.at(sizes["dgate"], np.arange(rows) // per, abs(scale) * u_size * size)
    out["size"] = sizes
    return out


def _log_softmax(z):
    m = z.max(1, keepdims=True)
    return z - m - np.log(np.exp(z - m).sum(1, keepdims=True))


def teacher(ids, logits, vocab, tau):
    """The teacher's distribution over the whole vocabulary, row by row (rows x vocab), and which rows have one: entries outside the
    vocabulary and logits of minus infinity are none."""
    ids, y = np.asarray(ids), np.asarray(logits, np.float64)
    q, has = np.zeros((ids.shape[0], vocab)), np.zeros(ids.shape[0], bool)
    for t in range(ids.shape[0]):
        ok = (ids[t] >= 0) & (ids[t] < vocab) & ~(y[t] == -np.inf)
        if ok.any():
            e = np.exp((y[t][ok] - y[t][ok].max()) / tau)
            np.add.at(q[t], ids[t][ok], e / e.sum())
            has[t] = True
    return q, has


def vocab_loss(X, W, label=None, top_id=None, top_logit=None, tau=1.0, dlabel=None, dtop=None):
    """dict of label_loss and top_loss (rows), and with dlabel / dtop of dX, dW and "dz", the gradient in the logits.  A row without a label
    (outside the vocabulary) or without a teacher has a loss of 0 and no gradient from that term; where it has neither its X is not looked at."""
    X, W = np.asarray(X, np.float64), np.asarray(W, np.float64)
    rows, vocab = X.shape[0], W.shape[0]
    has_l = np.zeros(rows, bool) if label is None else (np.asarray(label) >= 0) & (np.asarray(label) < vocab)
    q, has_t = teacher(top_id, top_logit, vocab, tau) if top_id is not None else (None, np.zeros(rows, bool))
    live = has_l | has_t
    out = {"label_loss": np.zeros(rows), "top_loss": np.zeros(rows)}
    dz = np.zeros((rows, vocab))
    Xl = np.where(live[:, None], X, 0.0)
    z = Xl @ W.T
    if has_l.any():
        at = np.flatnonzero(has_l)
        lp = _log_softmax(z[at])
        col = np.asarray(label)[at]
        out["label_loss"][at] = -lp[np.arange(len(at)), col]
        if dlabel is not None:
            p = np.exp(lp)
            p[np.arange(len(at)), col] -= 1.0
            dz[at] += np.asarray(dlabel, np.float64)[at][:, None] * p
    if has_t.any():
        at = np.flatnonzero(has_t)
        lp = _log_softmax(z[at] / tau)
        qa = q[at]
        with np.errstate(divide="ignore", invalid="ignore"):
            out["top_loss"][at] = np.where(qa > 0, qa * (np.log(np.where(qa > 0, qa, 1.0)) - lp), 0.0).sum(1)
        if dtop is not None:
            dz[at] += np.asarray(dtop, np.float64)[at][:, None] / tau * (np.exp(lp) - qa)
    if dlabel is not None or dtop is not None:
        out["dz"], out["dX"], out["dW"] = dz, dz @ W, dz.T @ Xl
    return out
