"""Up to 128 rows with a term hold the gradient in the logits of bf16 storage as two bf16 numbers: every entry, as in tests/test_cpu_lm_far_logits.py, and the errors of
dX and dW against one rounding of the exact ones."""
import numpy as np
import pytest
import torch

import paper_2503_12211_amd as stl
from test_cpu_lm_far_logits import B, case, check, unlabelled
from oracle import lm
from test_gpu_vocab import check as against_oracle, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab,label,tau,share", [(1, 700, True, None, 0.0), (32, 1000, True, 2.0, 0.0), (33, 1300, True, None, 0.0), (64, 515, False, 0.5, 0.0),
                                                        (65, 2000, True, 4.0, 0.0), (100, 64, True, None, 0.6), (128, 960, True, None, 0.0), (128, 960, True, None, 0.8),
                                                        (600, 333, True, None, 0.8), (1200, 100, True, None, 0.9)])
def test_every_entry(rows, vocab, label, tau, share):
    stored = case(rows, vocab, label, tau, 0.0, rows)
    if share:
        unlabelled(stored, share)
    t = {k: torch.from_numpy(v.view(np.int16) if v.dtype == np.uint16 else v).cuda() for k, v in stored.items()}
    prob = stl.VocabProblem(rows, rows, vocab, 2 if tau else 0, tau or 1.0, stl.STL_BF16)
    n = stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws, dW = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), torch.empty((vocab, rows), dtype=torch.bfloat16, device="cuda")
    stl.stl_vocab_loss_backward(prob, t["X"], t["W"], t.get("label"), t.get("top_id"), t.get("top_logit"), t.get("dlabel"), t.get("dtop"), None, None, None, dW, ws, n)
    check(stored, dW.double().cpu().numpy(), tau, rounding=B * B)


@pytest.mark.parametrize("rows,d,vocab,top,ignored", [(33, 64, 1205, 64, 0.0), (48, 64, 1714, 64, 0.0), (64, 72, 7001, 5, 0.0), (90, 130, 3000, 0, 0.0),
                                                      (128, 320, 2000, 32, 0.0), (700, 96, 1500, 0, 0.9)])
def test_errors_are_those_of_one_rounding(rows, d, vocab, top, ignored):
    """dX and dW rounded once have a relative error of at most 2^-9 of the norm (half a step of 2^-8 for an entry just above a power of two); the steps of the
    logits add less than a tenth of that, root of the sum of squares."""
    p = problem(rows, d, vocab, "bf16", label=top == 0 or top == 32, top=top, ignored=ignored, seed=rows)
    if top:
        p["dtop"] = np.abs(p["dtop"]) + 0.1
    tau = 2.0 if top else 1.0
    _, _, got = against_oracle(rows, d, vocab, "bf16", tau=tau, p=p)
    o = lm.vocab_loss(p["X"], p["W"], p["label"], p["top_id"], p["top_logit"], tau, p["dlabel"], p["dtop"])
    for k in ("dX", "dW"):
        g = got[k].double().cpu().numpy()
        assert np.linalg.norm(g - o[k]) <= 2.0 ** -9 * 1.005 * np.linalg.norm(o[k]), k
