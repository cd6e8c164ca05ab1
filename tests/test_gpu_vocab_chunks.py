"""The vocabulary loss where its rows come in several chunks (their logits would not fit the workspace's bound at once): every way to list the rows, both
storage types, against 64 bits.

Tolerances, with u = 2^-24.  A logit is off by at most (d + 16) u sum_k |x_k w_k|, with d <= 16 and |x_k w_k| of about 1 below 32 u * 16 = 3e-5; the sum of a
row's exponentials is taken in chains of vocab / 512 terms at most (2^22 / 512 = 8192) and trees, 8192 u = 5e-4 of it at worst.  Losses: their sum, 6e-4.
Gradients: the shares of the softmax have that error too, the sums over the vocabulary and the rows have roundings that are independent of each
other; 1e-3 of the norm in fp32, and 4e-3 in bf16 with the two roundings to bf16 (1.66e-3 each) as in the tests of one chunk.
What is looked for -- a row that is taken for another one, or left out -- is off by the whole of the row.
"""
import pytest
import torch

import paper_2503_12211_amd as stl
from gpu_util import STL_DT, TORCH_DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d,vocab,dtype,label,top", [
    (1000, 8, 300000, "f32", True, 0),            # 894 rows and 106
    (100, 4, 4194304, "f32", False, 2),           # 64 rows and 36, listed by a teacher
    (70, 4, 4194304, "f32", True, 0),
    (1500, 8, 300000, "f32", True, 3),            # more rows than are listed where they are gathered
    (700, 16, 4194304, "bf16", True, 0),          # 512 rows and 188
    (600, 8, 4000001, "bf16", True, 2),
])
def test_rows_of_every_chunk(rows, d, vocab, dtype, label, top):
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough free memory")
    print(f"chunks rows={rows} d={d} vocab={vocab} {dtype} label={label} top={top}", flush=True)
    tau = 2.0 if top else 1.0
    g = torch.Generator(device="cuda").manual_seed(rows)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    X, W = rand(rows, d).to(TORCH_DT[dtype]), (rand(vocab, d) * 0.5).to(TORCH_DT[dtype])
    target = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    lab = dlabel = ids = y = dtop = None
    if label:
        lab, dlabel = target.clone(), torch.rand(rows, generator=g, device="cuda") + 0.5
        lab[1::5] = -100
    if top:
        ids, y, dtop = torch.randint(0, vocab, (rows, top), generator=g, device="cuda"), rand(rows, top), torch.rand(rows, generator=g, device="cuda") + 0.5
        ids[2::7] = -1
    prob = stl.VocabProblem(rows, d, vocab, top, tau, STL_DT[dtype])
    n = stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    losses = [torch.full((rows,), float("nan"), device="cuda") if t is not None else None for t in (lab, ids)]
    dX, dW = torch.full_like(X, float("nan")), torch.full_like(W, float("nan"))
    stl.stl_vocab_loss_backward(prob, X, W, lab, ids, y, dlabel, dtop, *losses, dX, dW, ws, n)
    forward = [torch.empty_like(t) if t is not None else None for t in losses]
    stl.stl_vocab_loss_forward(prob, X, W, lab, ids, y, *forward, ws, n)
    del ws
    W64, want_dw = W.double(), torch.zeros((vocab, d), dtype=torch.float64, device="cuda")
    want_dx = torch.zeros((rows, d), dtype=torch.float64, device="cuda")
    want = [torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(2)]
    for at in range(0, rows, 50):
        s = slice(at, min(rows, at + 50))
        x = X[s].double()
        z = x @ W64.t().contiguous()
        here, dz = torch.arange(x.shape[0], device="cuda"), torch.zeros_like(z)
        if label:
            has = (lab[s] >= 0).double()
            lp = torch.log_softmax(z, 1)
            want[0][s] = -lp[here, lab[s].clamp(0)] * has
            p = lp.exp()
            p[here, lab[s].clamp(0)] -= 1.0
            dz += (dlabel[s].double() * has)[:, None] * p
        if top:
            has = (ids[s, 0] >= 0).double()
            lp, q = torch.log_softmax(z / tau, 1), torch.softmax(y[s].double() / tau, 1)
            want[1][s] = (q * (q.log() - lp.gather(1, ids[s].clamp(0)))).sum(1) * has
            dz += (dtop[s].double() * has / tau)[:, None] * lp.exp().scatter_add_(1, ids[s].clamp(0), -q)
        want_dx[s] = dz @ W64
        want_dw += dz.t().contiguous() @ x
    for got, fwd, w in zip(losses, forward, want):
        if got is not None:
            assert float((got.double() - w).abs().max()) <= 6e-4 and torch.equal(got, fwd)
    bar = 1e-3 if dtype == "f32" else 4e-3
    none = want_dx.abs().sum(1) == 0
    assert not dX[none].any()
    assert float(((dX.double() - want_dx).norm(dim=1) / want_dx.norm(dim=1).clamp_min(1e-30))[~none].max()) <= 4 * bar          # of a single row
    assert float((dX.double() - want_dx).norm() / want_dx.norm()) <= bar
    assert float((dW.double() - want_dw).norm() / want_dw.norm()) <= bar


def test_more_rows_than_a_launch_has_workgroups_for():
    """8.4 million rows of two classes in fp32: 512 threads a row would be 2^32 and more of them."""
    rows, d, vocab = (1 << 23) + 5000, 3, 2
    g = torch.Generator(device="cuda").manual_seed(3)
    X, W = torch.randn((rows, d), generator=g, device="cuda"), torch.randn((vocab, d), generator=g, device="cuda")
    label = torch.randint(-1, vocab, (rows,), generator=g, device="cuda")
    prob = stl.VocabProblem(rows, d, vocab, dtype=stl.STL_F32)
    n = stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws, loss = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    dX, dW, weight = torch.full_like(X, float("nan")), torch.empty_like(W), torch.full((rows,), 1.0, device="cuda")
    stl.stl_vocab_loss_backward(prob, X, W, label, None, None, weight, None, loss, None, dX, dW, ws, n)
    has = (label >= 0).double()
    lp = torch.log_softmax(X.double() @ W.double().t().contiguous(), 1)
    p = lp.exp().scatter_add_(1, label.clamp(0)[:, None], torch.full((rows, 1), -1.0, dtype=torch.float64, device="cuda")) * has[:, None]
    # logits below 20 in size: 16 roundings of 20; sums of 4 million terms of either sign, in chains of 2^22 / 512 and blocks of 32
    assert float((loss.double() + lp.gather(1, label.clamp(0)[:, None])[:, 0] * has).abs().max()) <= 16 * 20 * 2.0 ** -24
    assert float((dX.double() - p @ W.double()).abs().max()) <= 64 * 20 * 2.0 ** -24
    want = p.t().contiguous() @ X.double()
    size = p.abs().t().contiguous() @ X.double().abs()
    assert bool(((dW.double() - want).abs() <= 1e-4 * size).all())
