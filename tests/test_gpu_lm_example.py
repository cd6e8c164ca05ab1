"""The example that runs the residual step and the vocabulary loss together as a model trains with them: its gradients against autograd on elementary
torch operations, and that it learns."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _reference_residual(X, H, gate, w_post, w_pre, scale):
    norm = lambda v: v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6)  # noqa: E731
    rows = X.shape[0]
    Xout = X + scale * gate.repeat_interleave(-(-rows // gate.shape[0]), 0)[:rows] * norm(H) * w_post
    return Xout, norm(Xout) * w_pre


def test_residual_norm_gradients_are_autograds():
    from paper_2503_12211_amd.examples.stl_lm import residual_norm
    torch.manual_seed(0)
    rows, n = 30, 200
    t = [torch.randn(s, device="cuda") for s in ((rows, n), (rows, n), (3, n), (n,), (n,))]
    up = [torch.randn(rows, n, device="cuda") for _ in range(2)]
    mine = [v.clone().requires_grad_() for v in t]
    ref = [v.double().requires_grad_() for v in t]
    got, want = residual_norm(*mine, scale=0.7), _reference_residual(*ref, 0.7)
    sum((o * u).sum() for o, u in zip(got, up)).backward()
    sum((o * u.double()).sum() for o, u in zip(want, up)).backward()
    for a, b in zip([*got, *(v.grad for v in mine)], [*want, *(v.grad for v in ref)]):
        a, b = a.detach().double(), b.detach()
        assert float((a - b).norm() / b.norm()) <= 1e-5                         # fp32 sums of up to 200 terms


def test_vocab_loss_gradients_are_autograds():
    from paper_2503_12211_amd.examples.stl_lm import vocab_loss
    torch.manual_seed(1)
    rows, d, vocab, tau = 40, 48, 300, 2.0
    X, W = torch.randn(rows, d, device="cuda"), torch.randn(vocab, d, device="cuda") * 0.3
    label = torch.randint(0, vocab, (rows,), device="cuda")
    label[::3] = -100
    top_id = torch.stack([torch.randperm(vocab, device="cuda")[:6] for _ in range(rows)])
    top_logit = torch.randn(rows, 6, device="cuda")
    mine, ref = [v.clone().requires_grad_() for v in (X, W)], [v.double().requires_grad_() for v in (X, W)]
    got = vocab_loss(*mine, label, top_id, top_logit, tau, 0.5)
    z = ref[0] @ ref[1].t()
    q = torch.softmax(top_logit.double() / tau, 1)
    want = torch.nn.functional.cross_entropy(z, label) + 0.5 * (q * (q.log() - torch.log_softmax(z / tau, 1).gather(1, top_id))).sum(1).mean()
    (3 * got).backward()
    (3 * want).backward()
    for a, b in zip([got, *(v.grad for v in mine)], [want, *(v.grad for v in ref)]):
        a, b = a.detach().double(), b.detach()
        assert float((a - b).norm() / b.norm()) <= 1e-5
    with torch.no_grad():
        assert float(vocab_loss(X, W, label, top_id, top_logit, tau, 0.5)) == float(got)


def test_the_model_learns_its_language():
    from paper_2503_12211_amd.examples.stl_lm import train
    history, entropy = train(steps=60, batch=8, length=32, vocab=200, width=128, hidden=256)
    # from the uniform guess over the vocabulary (log 200 = 5.3, and what random states add) most of the way to the entropy of what follows a token
    late, least = sum(history[-10:]) / 10, sum(entropy[-10:]) / 10
    assert history[0] > 4.0
    assert least - 0.3 < late < 0.5 * (history[0] + least), (history[0], late, least)
