"""What the example's functions (examples/stl_lm.py) ask of the library, without a GPU: the entry points are replaced by stand-ins that note their arguments."""
import pytest
import torch

import paper_2503_12211_amd as stl
from paper_2503_12211_amd.examples import stl_lm


class Calls(list):
    def names(self):
        return [name for name, _ in self]


@pytest.fixture
def calls(monkeypatch):
    """Stand-ins: outputs are filled with 1 (losses, streams) and with seeded numbers (gradients of the loss)."""
    noted = Calls()

    def residual_forward(prob, X, H, gate, w_post, b_post, w_pre, b_pre, Xout, Z, flags, stream=None):
        noted.append(("residual_forward", dict(prob=prob, X=X, H=H, gate=gate, w_post=w_post, w_pre=w_pre)))
        Xout.fill_(1.0), Z.fill_(1.0)

    def residual_backward(prob, Xout, H, gate, w_post, b_post, w_pre, dXout, dZ, dX, dH, dgate, dw_post, db_post, dw_pre, db_pre, accumulate, ws, nbytes, flags,
                          stream=None):
        noted.append(("residual_backward", dict(prob=prob, gate=gate, dXout=dXout, dZ=dZ, dgate=dgate)))
        groups = -(-prob.rows // prob.rows_per_gate) if prob.rows else 0
        for t in (dX, dH, dw_post, dw_pre, dgate[:groups]):              # the library writes the rows of the gate that the step has
            t.fill_(1.0 if prob.rows else 0.0)

    def vocab_forward(prob, X, W, label, top_id, top_logit, label_loss, top_loss, ws, nbytes, stream=None):
        noted.append(("vocab_forward", dict(prob=prob, X=X, W=W, label=label, top_id=top_id, top_logit=top_logit)))
        for t in (label_loss, top_loss):
            if t is not None:
                t.fill_(1.0)

    def vocab_backward(prob, X, W, label, top_id, top_logit, dlabel, dtop, label_loss, top_loss, dX, dW, ws, nbytes, stream=None):
        vocab_forward(prob, X, W, label, top_id, top_logit, label_loss, top_loss, ws, nbytes)
        noted[-1] = ("vocab_backward", dict(noted[-1][1], dX=dX, dW=dW))
        g = torch.Generator().manual_seed(0)
        for t in (dX, dW):
            if t is not None:
                t.copy_(torch.randn(t.shape, generator=g))

    monkeypatch.setattr(stl, "stl_residual_norm_forward", residual_forward)
    monkeypatch.setattr(stl, "stl_residual_norm_backward", residual_backward)
    monkeypatch.setattr(stl, "stl_vocab_loss_forward", vocab_forward)
    monkeypatch.setattr(stl, "stl_vocab_loss_backward", vocab_backward)
    return noted


def step(rows=12, n=8, groups=3, dtype=torch.float32):
    shapes = ((rows, n), (rows, n), (groups, n), (n,), (n,))
    return [torch.ones(s, dtype=dtype).requires_grad_() for s in shapes]


@pytest.mark.parametrize("rows,groups", [(12, 1), (12, 3), (12, 12), (5, 3), (394, 2), (1, 1)])
def test_gate_rows_that_divide_the_rows(calls, rows, groups):
    t = step(rows, groups=groups)
    sum(o.sum() for o in stl_lm.residual_norm(*t)).backward()
    prob = calls[0][1]["prob"]
    assert -(-rows // prob.rows_per_gate) == groups
    assert bool((t[2].grad == 1.0).all())


@pytest.mark.parametrize("rows,groups", [(5, 4), (12, 13), (10, 7)])
def test_gate_rows_that_no_rows_would_take(calls, rows, groups):
    """5 rows and 4 gate rows: 2 rows share one, and the fourth's gradient would be whatever memory held."""
    with pytest.raises(ValueError):
        stl_lm.residual_norm(*step(rows, groups=groups))
    assert not calls


def test_step_without_rows(calls):
    t = step(0, groups=2)
    Xout, Z = stl_lm.residual_norm(*t)
    assert Xout.shape == Z.shape == (0, 8)
    (Xout.sum() + Z.sum()).backward()
    assert not t[2].grad.any() and not t[3].grad.any()


def bad_step(**kw):
    t = dict(zip(("X", "H", "gate", "w_post", "w_pre"), step()))
    t.update(kw)
    return t


@pytest.mark.parametrize("kw,error", [
    (dict(w_post=torch.ones(8, dtype=torch.bfloat16)), TypeError), (dict(H=torch.ones(12, 8, dtype=torch.float64)), TypeError),
    (dict(gate=torch.ones(3, 8, dtype=torch.bfloat16)), TypeError), (dict(w_pre=torch.ones(8, dtype=torch.float16)), TypeError),
    (dict(H=torch.ones(11, 8)), ValueError), (dict(H=torch.ones(12, 9)), ValueError), (dict(gate=torch.ones(3, 4)), ValueError), (dict(gate=torch.ones(8)), ValueError),
    (dict(w_post=torch.ones(9)), ValueError), (dict(w_pre=torch.ones(1, 8)), ValueError), (dict(X=torch.ones(2, 6, 8)), ValueError),
    (dict(H=torch.ones(12, 8, device="meta")), ValueError)])
def test_step_arguments_that_are_refused(calls, kw, error):
    with pytest.raises(error):
        stl_lm.residual_norm(**bad_step(**kw))
    assert not calls


def test_step_arguments_are_passed_dense(calls):
    t = bad_step(gate=torch.ones(1, 8).expand(3, 8), w_post=torch.ones(16)[::2], w_pre=torch.ones(1).expand(8), H=torch.ones(8, 12).t())
    t["X"] = t["X"].detach().requires_grad_()
    stl_lm.residual_norm(**t)
    assert all(calls[0][1][k].is_contiguous() for k in ("X", "H", "gate", "w_post", "w_pre"))


def scored(rows=6, d=8, vocab=20, ntop=3, dtype=torch.float32):
    g = torch.Generator().manual_seed(1)
    return dict(X=torch.randn((rows, d), generator=g).to(dtype), W=torch.randn((vocab, d), generator=g).to(dtype), label=torch.randint(0, vocab, (rows,), generator=g),
                top_id=torch.randint(0, vocab, (rows, ntop), generator=g), top_logit=torch.randn((rows, ntop), generator=g))


@pytest.mark.parametrize("kw,error", [
    (dict(label=torch.zeros(6, dtype=torch.int32)), TypeError), (dict(top_id=torch.zeros(6, 3, dtype=torch.int32)), TypeError),
    (dict(top_logit=torch.zeros(6, 3, dtype=torch.bfloat16)), TypeError), (dict(W=torch.zeros(20, 8, dtype=torch.bfloat16)), TypeError),
    (dict(label=torch.zeros(5, dtype=torch.int64)), ValueError), (dict(label=torch.zeros(6, 1, dtype=torch.int64)), ValueError),
    (dict(top_id=torch.zeros(5, 3, dtype=torch.int64)), ValueError), (dict(top_id=torch.zeros(6, dtype=torch.int64)), ValueError), (dict(top_logit=torch.zeros(6, 2)), ValueError), (dict(top_logit=None), ValueError),
    (dict(top_id=None), ValueError), (dict(W=torch.zeros(20, 9)), ValueError), (dict(X=torch.zeros(2, 3, 8)), ValueError),
    (dict(label=torch.zeros(6, dtype=torch.int64, device="meta")), ValueError)])
def test_loss_arguments_that_are_refused(calls, kw, error):
    with pytest.raises(error):
        stl_lm.vocab_loss(**{**scored(), **kw})
    assert not calls


def test_loss_arguments_are_passed_dense(calls):
    s = scored()
    s.update(X=torch.ones(8, 6).t(), W=torch.ones(8, 20).t(), label=torch.zeros(12, dtype=torch.int64)[::2], top_id=torch.zeros(6, 1, dtype=torch.int64).expand(6, 3),
             top_logit=torch.zeros(3, 6).t())
    stl_lm.vocab_loss(**s)
    assert all(calls[0][1][k].is_contiguous() for k in ("X", "W", "label", "top_id", "top_logit"))


def test_loss_gradients_take_the_upstream_factor_in_fp32(calls):
    """A factor that bf16 does not hold (a third is 0.2 % off there) is multiplied in fp32, and the gradient rounded behind it."""
    s = scored(dtype=torch.bfloat16)
    for k in "XW":
        s[k].requires_grad_()
    (stl_lm.vocab_loss(**s) / 3).backward()
    got = calls[0][1]
    factor = torch.tensor(1.0) / 3
    for k in "XW":
        assert s[k].grad.dtype == torch.bfloat16
        assert torch.equal(s[k].grad, (got["d" + k].float() * factor).to(torch.bfloat16)), k


def test_second_derivatives_are_refused(calls):
    """Neither function's gradients come with their own graph: a second derivative would lack their terms."""
    s = scored()
    X, W = s["X"].requires_grad_(), s["W"].requires_grad_()
    scale = torch.ones((), requires_grad=True)
    g = torch.autograd.grad(stl_lm.vocab_loss(**{**s, "X": X, "W": W}) * scale, X, create_graph=True)[0]
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()
    t = step()
    g = torch.autograd.grad(sum(o.square().sum() for o in stl_lm.residual_norm(*t)), t[0], create_graph=True)[0]
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()


@pytest.mark.parametrize("grad_x,grad_w", [(True, True), (True, False), (False, True)])
def test_loss_gradients_are_formed_where_they_are_asked_for(calls, grad_x, grad_w):
    s = scored()
    X, W = s["X"].requires_grad_(grad_x), s["W"].requires_grad_(grad_w)
    stl_lm.vocab_loss(**s).backward()
    assert calls.names() == ["vocab_backward"]
    assert (calls[0][1]["dX"] is not None) == grad_x and (calls[0][1]["dW"] is not None) == grad_w
    assert (X.grad is not None) == grad_x and (W.grad is not None) == grad_w


def test_scoring_is_the_forward_call(calls):
    """A parameter's requires_grad is set under no_grad too."""
    s = scored()
    s["W"] = torch.nn.Parameter(s["W"])
    with torch.no_grad():
        assert not stl_lm.vocab_loss(**s).requires_grad
    stl_lm.vocab_loss(**{**s, "W": s["W"].detach()})
    assert calls.names() == ["vocab_forward"] * 2
