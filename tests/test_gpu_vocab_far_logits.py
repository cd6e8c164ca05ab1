"""The gradient in the logits, entry by entry, where groups of logits hold some that lie far below the others: the cases and tolerances of
tests/test_cpu_lm_far_logits.py on the GPU, and sizes that every form of the logits' product takes (up to 16, 32, 64, 128 rows, more)."""
import numpy as np
import pytest
import torch

import paper_2503_12211_amd as stl
from test_cpu_lm_far_logits import TERMS, case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("label,tau", TERMS)
@pytest.mark.parametrize("rows,vocab", [(5, 200), (32, 1000), (40, 130), (104, 700), (264, 515)])
def test_every_entry(rows, vocab, label, tau):
    for far in (0.0, 40.0, 300.0, 3000.0, 1e30):
        stored = case(rows, vocab, label, tau, far, rows)
        t = {k: torch.from_numpy(v.view(np.int16) if v.dtype == np.uint16 else v).cuda() for k, v in stored.items()}
        prob = stl.VocabProblem(rows, rows, vocab, 2 if tau else 0, tau or 1.0, stl.STL_BF16)
        n = stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD)
        ws, dW = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), torch.empty((vocab, rows), dtype=torch.bfloat16, device="cuda")
        stl.stl_vocab_loss_backward(prob, t["X"], t["W"], t.get("label"), t.get("top_id"), t.get("top_logit"), t.get("dlabel"), t.get("dtop"), None, None, None, dW,
                                    ws, n)
        check(stored, dW.double().cpu().numpy(), tau)
