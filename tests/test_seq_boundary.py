"""CPU-side checks of the entry points of the embedding, the norms and rotation of queries and keys, and attention with decay: what is refused, before any launch."""
import copy
import pickle

import pytest

import paper_2503_12211_amd as stl

FAKE = 0x1000  # a non-null "device pointer"; never dereferenced because validation fails first


def refused(status, fn, *args):
    with pytest.raises(stl.StlError) as e:
        fn(*args, stream=0)
    assert e.value.status == status
    assert stl.stl_last_error()


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(d=0), 1), (dict(vocab=0), 1), (dict(rows=stl.STL_MAX_DIM + 1), 1), (dict(d=1048577), 1),
                                       (dict(vocab=4194305), 1), (dict(dtype=2), 2)])
def test_embeddings_that_are_refused(kw, status):
    prob = stl.EmbedProblem(**{**dict(rows=16, d=64, vocab=100), **kw})
    assert stl.stl_embed_workspace_bytes(prob) == 0
    refused(status, stl.stl_embed_forward, prob, FAKE, FAKE, FAKE)
    refused(status, stl.stl_embed_backward, prob, FAKE, FAKE, FAKE, 0, FAKE, 1 << 40)


def test_embedding_arguments_that_are_refused():
    prob = stl.EmbedProblem(16, 64, 100)
    need = stl.stl_embed_workspace_bytes(prob)
    assert need > 0
    for args in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None), (FAKE + 8, FAKE, FAKE), (FAKE, FAKE + 2, FAKE), (FAKE, FAKE, FAKE + 4)):
        refused(1, stl.stl_embed_forward, prob, *args)
        refused(1, stl.stl_embed_backward, prob, *args, 0, FAKE, need)
    refused(1, stl.stl_embed_backward, prob, FAKE, FAKE, FAKE, 2, FAKE, need)
    refused(3, stl.stl_embed_backward, prob, FAKE, FAKE, FAKE, 0, None, need)
    refused(3, stl.stl_embed_backward, prob, FAKE, FAKE, FAKE, 0, FAKE, need - 1)
    refused(1, stl.stl_embed_backward, prob, FAKE, FAKE, FAKE, 0, FAKE + 8, need)


PRE, ADJ = stl.STL_FLAG_PRE_NORM, stl.STL_FLAG_ADJACENT


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(rows=stl.STL_MAX_DIM + 1), 1), (dict(heads=0), 1), (dict(heads=65537), 1), (dict(kv_heads=-1), 1), (dict(d=0), 1),
                                       (dict(d=1026), 2), (dict(rot=-2), 1), (dict(rot=7), 1), (dict(rot=66), 1), (dict(base=0.0), 1), (dict(base=float("nan")), 1),
                                       (dict(base=float("inf")), 1), (dict(eps=0.0), 1), (dict(eps=float("nan")), 1), (dict(ld_q=255), 1), (dict(ld_k=127), 1),
                                       (dict(ld_qout=255), 1), (dict(ld_kout=-1), 1), (dict(dtype=7), 2)])
def test_heads_that_are_refused(kw, status):
    prob = stl.HeadNormProblem(**{**dict(rows=16, heads=4, kv_heads=2, d=64), **kw})
    assert stl.stl_head_norm_workspace_bytes(prob, PRE) == 0
    refused(status, stl.stl_head_norm_forward, prob, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, PRE)
    refused(status, stl.stl_head_norm_backward, prob, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, 0, FAKE, 1 << 40, PRE)


def test_head_arguments_that_are_refused():
    prob, queries = stl.HeadNormProblem(16, 4, 2, 64), stl.HeadNormProblem(16, 4, 0, 64)
    need = stl.stl_head_norm_workspace_bytes(prob, PRE)

    def f(prob=prob, **kw):
        a = dict(Q=FAKE, K=FAKE, w_q=FAKE, w_k=None, position=FAKE, Qout=FAKE, Kout=FAKE, flags=PRE)
        a.update(kw)
        return (prob, *a.values())

    for kw in (dict(Q=None), dict(K=None), dict(Qout=None), dict(Kout=None), dict(Q=FAKE + 1), dict(Kout=FAKE + 1), dict(w_q=FAKE + 2), dict(position=FAKE + 8)):
        refused(1, stl.stl_head_norm_forward, *f(**kw))
    refused(2, stl.stl_head_norm_forward, *f(flags=PRE | stl.STL_FLAG_CENTER))

    def b(prob=prob, **kw):
        a = dict(Q=FAKE, K=FAKE, w_q=FAKE, w_k=None, position=FAKE, dQout=FAKE, dKout=FAKE, dQ=FAKE, dK=FAKE, dw_q=FAKE, dw_k=None, accumulate=0, ws=FAKE, ws_bytes=need,
                 flags=PRE)
        a.update(kw)
        return (prob, *a.values())

    for kw in (dict(Q=None), dict(K=None), dict(accumulate=2), dict(flags=0), dict(dQ=None, dK=None, dw_q=None), dict(dQ=FAKE + 1), dict(dw_q=FAKE + 4), dict(ws=FAKE + 8),
               dict(prob=queries), dict(prob=queries, dK=None, dw_k=FAKE)):
        refused(1, stl.stl_head_norm_backward, *b(**kw))
    refused(3, stl.stl_head_norm_backward, *b(ws=None))
    refused(3, stl.stl_head_norm_backward, *b(ws_bytes=need - 1))
    refused(2, stl.stl_head_norm_backward, *b(flags=1))


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(rows=stl.STL_MAX_DIM + 1), 1), (dict(sequences=0), 1), (dict(length=-1), 1), (dict(heads=0), 1),
                                       (dict(kv_heads=0), 1), (dict(kv_heads=3), 1), (dict(kv_heads=8), 1), (dict(sequences=4194304), 1), (dict(dk=0), 1), (dict(dv=-1), 1),
                                       (dict(dk=257), 2), (dict(dv=300), 2), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
                                       (dict(scale=1e-39), 1), (dict(ld_q=127), 1), (dict(ld_k=63), 1), (dict(ld_v=0), 1), (dict(ld_o=-5), 1), (dict(dtype=3), 2)])
def test_attention_that_is_refused(kw, status):
    prob = stl.DecayAttentionProblem(**{**dict(rows=40, sequences=2, length=20, heads=4, kv_heads=2, dk=32), **kw})
    assert stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD) == 0
    refused(status, stl.stl_decay_attention_forward, prob, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, 1 << 50)
    refused(status, stl.stl_decay_attention_backward, prob, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, FAKE, FAKE, None, FAKE, 1 << 50)


@pytest.mark.parametrize("kw", [dict(rows=39), dict(seq_step=19), dict(seq_step=0), dict(token_step=0), dict(seq_step=1, token_step=1), dict(seq_step=-20), dict(token_step=-1),
                                dict(seq_step=1, token_step=3), dict(seq_step=1 << 40), dict(token_step=1 << 40), dict(seq_step=2, token_step=2)])
def test_rows_of_attention_that_are_refused(kw):
    """Rows outside, and rows that two tokens share."""
    prob = stl.DecayAttentionProblem(**{**dict(rows=40, sequences=2, length=20, heads=4, kv_heads=2, dk=32), **kw})
    refused(1, stl.stl_decay_attention_forward, prob, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, 1 << 50)
    refused(1, stl.stl_decay_attention_backward, prob, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, FAKE, FAKE, None, FAKE, 1 << 50)


def test_attention_arguments_that_are_refused():
    prob = stl.DecayAttentionProblem(40, 2, 20, 4, 2, 32)
    assert stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_ENCODE_WEIGHT) == 0 and stl.stl_last_error()

    def f(**kw):
        a = dict(Q=FAKE, K=FAKE, V=FAKE, log_decay=FAKE, offset=None, state_in=None, O=FAKE, state_out=None, ws=FAKE, ws_bytes=1 << 50)
        a.update(kw)
        return (prob, *a.values())

    for kw in (dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(Q=FAKE + 1), dict(O=FAKE + 1), dict(log_decay=FAKE + 4), dict(offset=FAKE + 8),
               dict(state_in=FAKE + 4), dict(state_out=FAKE + 8)):
        refused(1, stl.stl_decay_attention_forward, *f(**kw))

    def b(**kw):
        a = dict(Q=FAKE, K=FAKE, V=FAKE, log_decay=FAKE, offset=None, state_in=None, dO=FAKE, dstate_out=None, dQ=FAKE, dK=FAKE, dV=FAKE, dstate_in=None, ws=FAKE,
                 ws_bytes=1 << 50)
        a.update(kw)
        return (prob, *a.values())

    for kw in (dict(Q=None), dict(dO=None), dict(dQ=None, dK=None, dV=None), dict(dO=FAKE + 1), dict(dV=FAKE + 1), dict(dstate_out=FAKE + 4), dict(dstate_in=FAKE + 8),
               dict(dstate_in=FAKE, dstate_out=FAKE), dict(dstate_in=FAKE, state_in=FAKE)):
        refused(1, stl.stl_decay_attention_backward, *b(**kw))
    need = stl.stl_decay_attention_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    assert need > 0
    refused(3, stl.stl_decay_attention_backward, *b(ws=None))
    refused(3, stl.stl_decay_attention_backward, *b(ws_bytes=need - 1))
    refused(1, stl.stl_decay_attention_backward, *b(ws=FAKE + 8))


@pytest.mark.parametrize("prob", [stl.EmbedProblem(5, 64, 100), stl.HeadNormProblem(5, 4, 2, 64, 32, ld_q=999, dtype=stl.STL_F32),
                                  stl.DecayAttentionProblem(40, 2, 20, 4, 2, 32, 48, seq_step=1, token_step=2, scale=0.5)])
def test_problems_are_copied_and_sent(prob):
    for twin in (copy.copy(prob), copy.deepcopy(prob), pickle.loads(pickle.dumps(prob))):
        assert twin == prob
        size = {stl.EmbedProblem: stl.stl_embed_workspace_bytes, stl.HeadNormProblem: stl.stl_head_norm_workspace_bytes,
                stl.DecayAttentionProblem: lambda p: stl.stl_decay_attention_workspace_bytes(p, stl.STL_OP_BACKWARD)}[type(prob)]
        assert size(twin) == size(prob) > 0
