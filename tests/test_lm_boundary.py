"""CPU-side checks of the residual step's and the vocabulary loss's entry points: what is refused, before any launch."""
import pytest

import paper_2503_12211_amd as stl

FAKE = 0x1000  # a non-null "device pointer"; never dereferenced because validation fails first


def refused(status, fn, *args):
    with pytest.raises(stl.StlError) as e:
        fn(*args, stream=0)
    assert e.value.status == status
    assert stl.stl_last_error()


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(n=0), 1), (dict(rows_per_gate=0), 1), (dict(eps=0.0), 1), (dict(eps=float("nan")), 1),
                                       (dict(rows=stl.STL_MAX_DIM + 1), 1), (dict(n=32769), 2), (dict(dtype=5), 2)])
def test_residual_problems_that_are_refused(kw, status):
    prob = stl.ResidualProblem(**{**dict(rows=16, n=64), **kw})
    flags = stl.STL_FLAG_PRE_NORM
    assert stl.stl_residual_norm_workspace_bytes(prob, flags) == 0
    refused(status, stl.stl_residual_norm_forward, prob, FAKE, FAKE, None, None, None, None, None, FAKE, FAKE, flags)
    refused(status, stl.stl_residual_norm_backward, prob, FAKE, FAKE, None, None, None, None, FAKE, FAKE, FAKE, FAKE, None, None, None, None, None, 0, FAKE,
            1 << 40, flags)


def test_residual_arguments_that_are_refused():
    prob = stl.ResidualProblem(16, 64)
    pre, post = stl.STL_FLAG_PRE_NORM, stl.STL_FLAG_POST_NORM
    fwd, bwd = stl.stl_residual_norm_forward, stl.stl_residual_norm_backward
    need = stl.stl_residual_norm_workspace_bytes(prob, pre)
    assert need > 0
    refused(2, fwd, prob, FAKE, FAKE, None, None, None, None, None, FAKE, FAKE, pre | stl.STL_FLAG_GELU)
    for hole in ((None, FAKE, FAKE, FAKE), (FAKE, None, FAKE, FAKE), (FAKE, FAKE, None, FAKE), (FAKE, FAKE, FAKE, None)):
        refused(1, fwd, prob, hole[0], hole[1], None, None, None, None, None, hole[2], hole[3], pre)
    refused(1, fwd, prob, FAKE + 8, FAKE, None, None, None, None, None, FAKE, FAKE, pre)

    def grads(**kw):
        a = dict(Xout=FAKE, H=FAKE, gate=FAKE, w_post=None, b_post=None, w_pre=None, dXout=FAKE, dZ=FAKE, dX=FAKE, dH=FAKE, dgate=None, dw_post=None,
                 db_post=None, dw_pre=None, db_pre=None, accumulate=0, ws=FAKE, ws_bytes=need, flags=pre | post)
        a.update(kw)
        return (prob, *a.values())

    refused(1, bwd, *grads(accumulate=2))
    refused(1, bwd, *grads(gate=None, dgate=FAKE))
    refused(1, bwd, *grads(flags=pre, dw_post=FAKE))
    refused(1, bwd, *grads(flags=post, db_pre=FAKE))
    refused(1, bwd, *grads(Xout=None))
    refused(1, bwd, *grads(H=None))
    refused(1, bwd, *grads(dZ=FAKE + 4))
    refused(3, bwd, *grads(ws=None))
    refused(3, bwd, *grads(ws_bytes=need - 1))
    refused(1, bwd, *grads(ws=FAKE + 8))
    refused(2, bwd, *grads(flags=0x1))


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(d=0), 1), (dict(vocab=0), 1), (dict(ntop=-1), 1), (dict(ntop=1025), 1), (dict(d=1048577), 1),
                                       (dict(vocab=4194305), 1), (dict(rows=stl.STL_MAX_DIM + 1), 1), (dict(dtype=9), 2), (dict(ntop=4, temperature=0.2), 1),
                                       (dict(ntop=4, temperature=17.0), 1), (dict(ntop=4, temperature=float("nan")), 1)])
def test_vocabulary_problems_that_are_refused(kw, status):
    prob = stl.VocabProblem(**{**dict(rows=16, d=64, vocab=100), **kw})
    assert stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD) == 0
    refused(status, stl.stl_vocab_loss_forward, prob, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, 1 << 50)
    refused(status, stl.stl_vocab_loss_backward, prob, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, 1 << 50)


def test_vocabulary_arguments_that_are_refused():
    prob, taught = stl.VocabProblem(16, 64, 100), stl.VocabProblem(16, 64, 100, 4)
    fwd, bwd = stl.stl_vocab_loss_forward, stl.stl_vocab_loss_backward
    need, need_b = (stl.stl_vocab_loss_workspace_bytes(prob, op) for op in (stl.STL_OP_FORWARD, stl.STL_OP_BACKWARD))
    assert 0 < need < need_b
    assert stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_ENCODE_WEIGHT) == 0

    def f(prob=prob, **kw):
        a = dict(X=FAKE, W=FAKE, label=FAKE, top_id=None, top_logit=None, label_loss=FAKE, top_loss=None, ws=FAKE, ws_bytes=need)
        a.update(kw)
        return (prob, *a.values())

    for kw in (dict(X=None), dict(W=None), dict(label=None, label_loss=None), dict(label=None), dict(label_loss=None), dict(top_loss=FAKE), dict(W=FAKE + 2),
               dict(label=FAKE + 8), dict(prob=taught, top_logit=FAKE), dict(prob=taught, top_id=FAKE), dict(ws=FAKE + 4, ws_bytes=1 << 40)):
        refused(1, fwd, *f(**kw))
    refused(3, fwd, *f(ws=None))
    refused(3, fwd, *f(ws_bytes=need - 1))

    def b(prob=prob, **kw):
        a = dict(X=FAKE, W=FAKE, label=FAKE, top_id=None, top_logit=None, dlabel=FAKE, dtop=None, label_loss=None, top_loss=None, dX=FAKE, dW=FAKE, ws=FAKE,
                 ws_bytes=need_b)
        a.update(kw)
        return (prob, *a.values())

    for kw in (dict(dX=None, dW=None), dict(dlabel=None), dict(dlabel=None, dtop=FAKE), dict(dX=FAKE + 8), dict(dlabel=FAKE + 4), dict(X=None)):
        refused(1, bwd, *b(**kw))
    refused(3, bwd, *b(ws_bytes=need_b - 1))


def test_vocabulary_workspace_is_bounded_in_the_rows():
    sizes = [stl.stl_vocab_loss_workspace_bytes(stl.VocabProblem(rows, 4096, 131072), stl.STL_OP_BACKWARD) for rows in (8192, 16384, 1 << 20)]
    assert sizes[0] < 4 << 30 and sizes[2] - sizes[1] < 8 << 20 and sizes[2] < 6 << 30


@pytest.mark.parametrize("prob", [stl.ResidualProblem(5, 64), stl.ResidualProblem(5, 64, 2, 0.5, 2.0, 1e-5, stl.STL_F32), stl.VocabProblem(7, 32, 100, 4, 2.0, stl.STL_F32)])
def test_problems_are_copied_and_sent(prob):
    """As stl.Problem is: with a module that keeps one, or to another process."""
    import copy
    import pickle
    flags = stl.STL_FLAG_PRE_NORM
    for twin in (copy.copy(prob), copy.deepcopy(prob), pickle.loads(pickle.dumps(prob))):
        assert twin == prob
        if isinstance(prob, stl.VocabProblem):
            assert stl.stl_vocab_loss_workspace_bytes(twin, stl.STL_OP_BACKWARD) == stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD) > 0
        else:
            assert stl.stl_residual_norm_workspace_bytes(twin, flags) == stl.stl_residual_norm_workspace_bytes(prob, flags) > 0
