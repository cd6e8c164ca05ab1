"""GPU parity of the vocabulary loss (labels, a teacher's top logits, both) and its gradients against the 64-bit oracle.

Tolerances, with u = 2^-24 and b = 2^-8 (half a unit of the last place of fp32 and bf16 in relative terms, at most).
  Logits: fp32 sums of d products in chains of at most d terms, off by (d + 16) u sum_k |x_k w_k| =: e_z.  A loss is a difference of a logit (over tau) and a
  logarithm, whose error is at most the largest e_z of the row (it is an average of z's errors) plus the rounding of its sum, (vocab / 8 + 64) u, and
  of |lse| and |z| themselves, 8 u each; the exponentials are taken in base 2 from arguments rounded at |z| log2 e, which the |z| term covers.
  fp32 gradients: dz is off by its shares times (2 max e_z + sums) <= E relative to p (and to q, exactly known up to 64 u); dX and dW then by the
  same factor on absolute values plus (vocab or rows) u for their own sums.
  bf16 gradients: dz rounded once and the 16-bit steps of the logits between, b + 2.5e-4 max(1, tau / 2, 1 / tau) + E, on absolute values; the output once more, b.
The bound is of an entry, |G - O| <= factor * S with S the products on absolute values; and in the mean over all entries bf16 errors are
independent, so the relative Frobenius error stays below 4e-3 (two roundings of 1.66e-3 and the steps).
"""
import numpy as np
import pytest
import torch

import paper_2503_12211_amd as stl
from gpu_util import STL_DT, TORCH_DT, Guard, dev
from oracle import lm

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8


def _round(a, dtype):
    return torch.from_numpy(np.asarray(a, np.float32)).to(TORCH_DT[dtype]).double().numpy()


def problem(rows, d, vocab, dtype, label=True, top=0, ignored=0.0, seed=0, spread=2.0):
    rng = np.random.default_rng(seed)
    W = _round(rng.standard_normal((vocab, d)) * spread / np.sqrt(d), dtype)
    at = rng.integers(0, vocab, rows)
    X = _round(rng.standard_normal((rows, d)) + rng.random((rows, 1)) * 4 * W[at] * (2.0 / spread) ** 2, dtype)
    p = {"X": X, "W": W, "label": None, "top_id": None, "top_logit": None, "dlabel": None, "dtop": None}
    if label:
        p["label"] = np.where(rng.random(rows) < ignored, -100, at).astype(np.int64)
        p["dlabel"] = (rng.random(rows) + 0.5).astype(np.float32)
    if top:
        ids = rng.integers(0, vocab, (rows, top))
        ids[:, 0] = at
        if top > 1:
            ids = np.where(rng.random((rows, top)) < 0.2, -1, ids)          # lists of different lengths; some of their ids twice
        p["top_id"] = ids.astype(np.int64)
        p["top_logit"] = (4 * rng.standard_normal((rows, top))).astype(np.float32)
        p["dtop"] = (rng.random(rows) - 0.2).astype(np.float32)
    return p


def to_dev(p, dtype):
    return {k: None if v is None else dev(v, dtype) if k in "XW" else torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in p.items()}


def workspace(gd, prob, op, poison=True):
    nbytes = stl.stl_vocab_loss_workspace_bytes(prob, op)
    return gd.alloc((max(nbytes, 16),), torch.uint8, fill=0xFF if poison else 0), nbytes


def gpu_forward(prob, t, dtype):
    gd = Guard()
    ll = gd.alloc((prob.rows,), torch.float32) if t["label"] is not None else None
    tl = gd.alloc((prob.rows,), torch.float32) if t["top_id"] is not None else None
    ws, n = workspace(gd, prob, stl.STL_OP_FORWARD)
    stl.stl_vocab_loss_forward(prob, t["X"], t["W"], t["label"], t["top_id"], t["top_logit"], ll, tl, ws, n)
    gd.check()
    return ll, tl


def gpu_backward(prob, t, dtype, losses=True, dX=True, dW=True):
    gd = Guard()
    out = {"label_loss": gd.alloc((prob.rows,), torch.float32) if t["label"] is not None and losses else None,
           "top_loss": gd.alloc((prob.rows,), torch.float32) if t["top_id"] is not None and losses else None,
           "dX": gd.alloc((prob.rows, prob.d), TORCH_DT[dtype]) if dX else None, "dW": gd.alloc((prob.vocab, prob.d), TORCH_DT[dtype]) if dW else None}
    ws, n = workspace(gd, prob, stl.STL_OP_BACKWARD)
    stl.stl_vocab_loss_backward(prob, t["X"], t["W"], t["label"], t["top_id"], t["top_logit"], t["dlabel"], t["dtop"], *out.values(), ws, n)
    gd.check()
    return out


def f64(t):
    return t.double().cpu().numpy()


def check(rows, d, vocab, dtype, tau=1.0, p=None, **kw):
    p = p or problem(rows, d, vocab, dtype, **kw)
    t = to_dev(p, dtype)
    ntop = 0 if p["top_id"] is None else p["top_id"].shape[1]
    prob = stl.VocabProblem(rows, d, vocab, ntop, tau, STL_DT[dtype])
    print(f"vocabulary loss rows={rows} d={d} vocab={vocab} {dtype} tau={tau} ntop={ntop} label={p['label'] is not None}", flush=True)
    tau = tau if ntop else 1.0
    o = lm.vocab_loss(p["X"], p["W"], p["label"], p["top_id"], p["top_logit"], tau, p["dlabel"], p["dtop"])
    e_z = ((d + 16) * U * (np.abs(p["X"]) @ np.abs(p["W"]).T)).max(1)
    big = np.abs(p["X"] @ p["W"].T).max(1) + np.log(vocab)
    E = (2 * e_z + 16 * U * big) / min(tau, 1.0) + (vocab / 8 + 64 + 64 * (ntop > 0)) * U
    ll, tl = gpu_forward(prob, t, dtype)
    got = gpu_backward(prob, t, dtype)
    for name, fwd in (("label_loss", ll), ("top_loss", tl)):
        if got[name] is not None:
            off = np.abs(f64(got[name]) - o[name]) - E
            assert off.max() <= 0, (name, off.max())
            assert torch.equal(got[name], fwd), name                         # the forward call gives the same bits
    # |dz| on absolute values: shares of the softmax and of the teacher count, not their difference
    q, has_t = lm.teacher(p["top_id"], p["top_logit"], vocab, tau) if ntop else (0.0, None)
    z = p["X"] @ p["W"].T
    size = np.zeros((rows, vocab))
    if p["label"] is not None:
        has = (p["label"] >= 0) & (p["label"] < vocab)
        size += (np.abs(p["dlabel"]) * has)[:, None] * np.exp(lm._log_softmax(z))
        size[np.flatnonzero(has), p["label"][has]] += np.abs(p["dlabel"][has])
    if ntop:
        size += (np.abs(p["dtop"]) * has_t)[:, None] / tau * (np.exp(lm._log_softmax(z / tau)) + q)
    step = 0.0 if dtype == "f32" else B + 2.5e-4 * max(1.0, tau / 2, 1 / tau)
    per_row = (E + step)[:, None] * size
    unit = B if dtype == "bf16" else U
    for name, want, bound in (("dX", o["dX"], per_row @ np.abs(p["W"]) + (vocab + 64) * U * (size @ np.abs(p["W"]))),
                              ("dW", o["dW"], per_row.T @ np.abs(p["X"]) + (rows + 64) * U * (size.T @ np.abs(p["X"])))):
        g = f64(got[name])
        assert np.isfinite(g).all(), name
        off = np.abs(g - want) - (bound + unit * np.abs(want))
        assert off.max() <= 0, f"{name}: {off.max()} over the bound at {np.unravel_index(off.argmax(), off.shape)}"
        if dtype == "bf16" and np.linalg.norm(want) > 0:
            rel = np.linalg.norm(g - want) / np.linalg.norm(want)
            assert rel <= 4e-3, f"{name}: relative error {rel:.2e}"
    return prob, t, got


# blocks of 64 and of 256 rows, whole and not; widths with whole stages, with part of one, odd; vocabularies of one column to many blocks
SHAPES = [(1, 64, 64), (1, 32, 1), (2, 8, 3), (5, 40, 100), (16, 128, 1000), (63, 96, 257), (64, 256, 512), (65, 256, 511), (100, 33, 640), (200, 100, 321),
          (256, 512, 1024), (257, 64, 2049), (300, 1000, 777), (513, 129, 255), (700, 256, 4100), (33, 2048, 5000)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_labels(shape, dtype):
    check(*shape, dtype, seed=shape[0])


@pytest.mark.parametrize("shape", SHAPES[3:12])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 0.25])
def test_teacher_alone(shape, dtype, tau):
    check(*shape, dtype, tau=tau, label=False, top=7, seed=shape[0])


@pytest.mark.parametrize("shape", SHAPES[3:12])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [1.0, 4.0, 16.0])
def test_labels_and_teacher(shape, dtype, tau):
    check(*shape, dtype, tau=tau, top=16, ignored=0.3, seed=shape[0])


# few rows and a wide vocabulary: dX's contraction in many runs, whose number is not a divisor of its stages
@pytest.mark.parametrize("shape", [(1, 8, 70000), (34, 64, 66001), (68, 205, 40001), (257, 72, 33000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top", [0, 3])
def test_few_rows_of_a_wide_vocabulary(shape, dtype, top):
    check(*shape, dtype, tau=2.0 if top else 1.0, top=top, seed=sum(shape) + top)


@pytest.mark.parametrize("top", [1, 2, 63, 64, 65, 600, 1024])
def test_lengths_of_the_teachers_lists(top):
    check(40, 64, 1500, "bf16", tau=2.0, top=top, seed=top)
    check(9, 24, 1500, "f32", tau=1.5, top=top, label=False, seed=top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ignored", [0.5, 0.95, 1.0])
def test_rows_without_a_label(dtype, ignored):
    """What an unlabelled row holds is not looked at: not a number in it changes no other bit."""
    p = problem(290, 128, 900, dtype, ignored=ignored, seed=17)
    prob, t, got = check(290, 128, 900, dtype, p=p)
    none = p["label"] < 0
    assert not got["dX"][torch.from_numpy(none).cuda()].any() and not got["label_loss"][torch.from_numpy(none).cuda()].any()
    bad = t["X"].clone()
    bad[torch.from_numpy(none).cuda()] = float("nan")
    again = gpu_backward(prob, dict(t, X=bad), dtype)
    assert all(torch.equal(again[k], got[k]) for k in ("label_loss", "dX", "dW"))
    labels = t["label"].clone()
    labels[torch.from_numpy(none).cuda()] = 900                                # behind the vocabulary: none either
    again = gpu_backward(prob, dict(t, label=labels), dtype)
    assert all(torch.equal(again[k], got[k]) for k in ("label_loss", "dX", "dW"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_of_the_teachers_lists(dtype):
    """Minus infinity and ids outside are no entries; the lowest value of fp32 is one, and alone in its row it is everything."""
    p = problem(6, 64, 300, dtype, label=False, top=4, seed=23)
    low = np.finfo(np.float32).min
    p["top_id"][:] = [[5, 9, 200, 3]] * 6
    p["top_id"][3] = [-1, 300, 2 ** 40, -2 ** 40]
    p["top_logit"][0] = [low, low, low, low]
    p["top_logit"][1] = [1.0, low, -np.inf, 0.0]
    p["top_logit"][2] = [-np.inf] * 4
    p["top_logit"][4] = [low, -np.inf, -np.inf, -np.inf]
    p["top_logit"][5] = [3e38, 3e38, low, -3e38]
    for tau in (0.25, 1.0, 4.0):
        _, _, got = check(6, 64, 300, dtype, tau=tau, p=p)
        assert not got["dX"][2].any() and not got["dX"][3].any() and float(got["top_loss"][2]) == float(got["top_loss"][3]) == 0.0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_confident_and_extreme_logits(dtype):
    """Logits of a deviation of 40: most labels are certain or hopeless, exponentials leave the range of fp32."""
    check(130, 64, 700, dtype, spread=40.0, seed=29)
    check(70, 64, 700, dtype, spread=20.0, top=8, tau=2.0, seed=30)


def test_rows_that_are_not_numbers_stay_alone_in_dx():
    p = problem(80, 64, 500, "bf16", top=5, seed=31)
    prob, t, got = check(80, 64, 500, "bf16", p=p)
    bad = t["X"].clone()
    bad[7, 3], bad[70, 0] = float("nan"), float("inf")
    again = gpu_backward(prob, dict(t, X=bad), "bf16")
    rest = [i for i in range(80) if i not in (7, 70)]
    for k in ("label_loss", "top_loss", "dX"):
        assert torch.equal(again[k][rest], got[k][rest]), k
        assert bool(torch.isnan(again[k][7]).all()), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_on_their_own_and_repeated_bits(dtype):
    prob, t, got = check(270, 192, 1300, dtype, tau=2.0, top=12, ignored=0.2, seed=37)
    for kw in (dict(losses=False), dict(dX=False), dict(dW=False)):
        for _ in range(2):
            again = gpu_backward(prob, t, dtype, **kw)
            assert all(torch.equal(again[k], got[k]) for k in again if again[k] is not None), kw
    # a term without an upstream gradient still gives its loss
    a = gpu_backward(prob, dict(t, dtop=None), dtype)
    b = gpu_backward(prob, dict(t, dtop=torch.zeros(270, device="cuda")), dtype)
    assert torch.equal(a["top_loss"], got["top_loss"]) and torch.equal(a["dX"], b["dX"]) and torch.equal(a["dW"], b["dW"])


def test_more_rows_than_a_chunk():
    """Three chunks: a vocabulary so large that the codes of 512 rows fill one."""
    d, vocab = 32, 4194304
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("not enough free memory")
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = 1100
    X = torch.randn((rows, d), generator=g, device="cuda").bfloat16()
    W = (torch.randn((vocab, d), generator=g, device="cuda") * 0.3).bfloat16()
    label = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    label[::3] = -1
    prob = stl.VocabProblem(rows, d, vocab)
    n = stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    loss, dX, dW = torch.empty(rows, device="cuda"), torch.empty_like(X), torch.empty_like(W)
    w = torch.rand(rows, generator=g, device="cuda") + 0.5
    stl.stl_vocab_loss_backward(prob, X, W, label, None, None, w, None, loss, None, dX, dW, ws, n)
    want_dw = torch.zeros((vocab, d), dtype=torch.float64, device="cuda")
    for at in range(0, rows, 100):
        x, lab = X[at:at + 100].double(), label[at:at + 100]
        has = lab >= 0
        lp = torch.log_softmax(x @ W.double().t(), 1)
        want = torch.where(has, -lp.gather(1, lab.clamp(0)[:, None])[:, 0], 0.0)
        assert float((loss[at:at + 100].double() - want).abs().max()) <= 2e-3 * 1e-1            # (vocab / 8 + ...) u = 0.03 worst, far above what sums of like signs do
        dz = lp.exp()
        dz[torch.arange(len(lab), device="cuda"), lab.clamp(0)] -= 1.0
        dz = dz * torch.where(has, w[at:at + 100].double(), 0.0)[:, None]
        want_dx = dz @ W.double()
        assert float((dX[at:at + 100].double() - want_dx).norm() / want_dx.norm()) <= 4e-3
        want_dw += dz.t() @ x
    assert float((dW.double() - want_dw).norm() / want_dw.norm()) <= 4e-3


def test_more_rows_than_a_chunk_of_many():
    """8192 rows and some, dW in parts (a classifier's vocabulary)."""
    rng = np.random.default_rng(41)
    rows, d, vocab = 8192 + 300, 64, 300
    p = problem(rows, d, vocab, "bf16", ignored=0.02, top=3, seed=41)
    check(rows, d, vocab, "bf16", tau=2.0, p=p)
    assert rng is not None


def test_on_another_stream_and_in_a_captured_graph():
    p = problem(300, 128, 1000, "bf16", top=9, ignored=0.2, seed=43)
    t = to_dev(p, "bf16")
    prob = stl.VocabProblem(300, 128, 1000, 9, 2.0)
    n = stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = [torch.empty(300, device="cuda"), torch.empty(300, device="cuda"), torch.empty_like(t["X"]), torch.empty_like(t["W"])]

    def step():
        stl.stl_vocab_loss_backward(prob, t["X"], t["W"], t["label"], t["top_id"], t["top_logit"], t["dlabel"], t["dtop"], *outs, ws, n)

    step()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for o in outs:
        o.zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        # other inputs, other rows listed: what a replay does is decided on the device
        t["X"].copy_(torch.randn_like(t["X"]))
        t["label"][k::2] = -100 if k == 1 else k + 5
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows(dtype):
    prob = stl.VocabProblem(0, 16, 40, dtype=STL_DT[dtype])
    W = torch.ones((40, 16), dtype=TORCH_DT[dtype], device="cuda")
    dW = torch.ones_like(W)
    assert stl.stl_vocab_loss_workspace_bytes(prob, stl.STL_OP_BACKWARD) == 0
    stl.stl_vocab_loss_forward(prob, None, W, None, None, None, None, None)
    stl.stl_vocab_loss_backward(prob, None, W, None, None, None, None, None, None, None, None, dW)
    assert not dW.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_are_the_losses_differences(dtype):
    """Central differences of the forward call's own losses along a direction, fp32 loss sums: exact to second order in the step."""
    if dtype == "bf16":
        pytest.skip("a step that a bf16 input can hold is far too long")
    p = problem(24, 32, 200, dtype, top=6, seed=47)
    t = to_dev(p, dtype)
    prob = stl.VocabProblem(24, 32, 200, 6, 2.0, STL_DT[dtype])
    got = gpu_backward(prob, t, dtype)

    def value(X, W):
        ll, tl = gpu_forward(prob, dict(t, X=X, W=W), dtype)
        return float((t["dlabel"].double() * ll.double()).sum() + (t["dtop"].double() * tl.double()).sum())

    g = torch.Generator(device="cuda").manual_seed(3)
    for k in ("X", "W"):
        v = torch.randn(t[k].shape, generator=g, device="cuda")
        v /= v.norm()
        h = 2.0 ** -5
        args = {"X": t["X"], "W": t["W"]}
        up, down = (value(**{**args, k: t[k] + sign * h * v}) for sign in (1, -1))
        want = float((got["d" + k].double() * v.double()).sum())
        # rounding of the losses (24 of about 5, 64 u each) over 2 h, and the third derivative (below 1 along a unit direction of these sizes) times h^2 / 6
        assert abs((up - down) / (2 * h) - want) <= 24 * 5 * 64 * U / (2 * h) + 24 * 4 * h * h / 6, k
