"""GPU parity of the residual step (norm, gate, residual sum, norm) and its gradients against the 64-bit oracle.

Tolerances.  An output is rounded to its type once, at most half a unit of its last place: 2^-8 |O| for bf16 (2^-24 |O| for fp32).  The fp32
arithmetic before it: a thread adds 8 to 32 elements, then a tree of 10 steps, then a handful of products, so an entry is off by at most
64 2^-24 times S, the same expression on absolute values.  A sum over rows adds a chain of at most `rows` terms: (rows + 64) 2^-24 S.
"""
import numpy as np
import pytest
import torch

import paper_2503_12211_amd as stl
from gpu_util import STL_DT, TORCH_DT, Guard, dev, host
from oracle import lm

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def _round(a, dtype):
    return torch.from_numpy(np.asarray(a, np.float32)).to(TORCH_DT[dtype]).double().numpy()


def problem(rows, n, dtype, per, post, pre, gate, weights, offsets, seed):
    rng = np.random.default_rng(seed)
    r = lambda *s: _round(rng.standard_normal(s), dtype)  # noqa: E731
    p = {"X": r(rows, n) * 2, "H": _round(rng.standard_normal((rows, n)) * 1.5 + 0.25, dtype), "dXout": r(rows, n), "dZ": r(rows, n) if pre else None,
         "gate": r(-(-rows // per), n) if gate else None, "w_post": r(n) if post and weights else None, "b_post": r(n) if post and offsets else None,
         "w_pre": r(n) if pre and weights else None, "b_pre": r(n) if pre and offsets else None}
    return p


def flags_of(post, pre, center):
    return (stl.STL_FLAG_POST_NORM if post else 0) | (stl.STL_FLAG_PRE_NORM if pre else 0) | (stl.STL_FLAG_CENTER if center else 0)


def to_dev(p, dtype):
    return {k: None if v is None else dev(v, dtype) for k, v in p.items()}


def gpu_forward(prob, t, flags, dtype, in_place=False):
    gd = Guard()
    Xout = t["X"].clone() if in_place else gd.alloc((prob.rows, prob.n), TORCH_DT[dtype])
    Z = gd.alloc((prob.rows, prob.n), TORCH_DT[dtype]) if flags & stl.STL_FLAG_PRE_NORM else None
    stl.stl_residual_norm_forward(prob, Xout if in_place else t["X"], t["H"], t["gate"], t["w_post"], t["b_post"], t["w_pre"], t["b_pre"], Xout, Z, flags)
    gd.check()
    return Xout, Z


def gpu_backward(prob, t, Xout, flags, dtype, accumulate=0, init=None, skip=(), poison=True):
    gd = Guard()
    outs = {"dX": gd.alloc((prob.rows, prob.n), TORCH_DT[dtype]), "dH": gd.alloc((prob.rows, prob.n), TORCH_DT[dtype])}
    if t["gate"] is not None:
        outs["dgate"] = gd.alloc(tuple(t["gate"].shape), torch.float32)
    for k, f in (("dw_post", stl.STL_FLAG_POST_NORM), ("db_post", stl.STL_FLAG_POST_NORM), ("dw_pre", stl.STL_FLAG_PRE_NORM), ("db_pre", stl.STL_FLAG_PRE_NORM)):
        if flags & f:
            outs[k] = gd.alloc((prob.n,), torch.float32)
    for k in skip:
        outs.pop(k, None)
    if init is not None:
        for k in outs:
            if k not in ("dX", "dH"):
                outs[k].fill_(init)
    nbytes = stl.stl_residual_norm_workspace_bytes(prob, flags)
    ws = gd.alloc((max(nbytes, 16),), torch.uint8, fill=0xFF if poison else 0)
    stl.stl_residual_norm_backward(prob, Xout, t["H"], t["gate"], t["w_post"], t["b_post"], t["w_pre"], t["dXout"], t["dZ"], *(
        outs.get(k) for k in ("dX", "dH", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")), accumulate, ws, nbytes, flags)
    gd.check()
    return outs


def close(got, want, size, dtype, chain, name):
    got = host(got) if got.dtype != torch.float32 else got.double().cpu().numpy()
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    off = np.abs(got - want) - (unit * np.abs(want) + chain * EPS * size)
    assert np.isfinite(got).all(), name
    assert off.max(initial=-1.0) <= 0, f"{name}: {off.max()} over the bound at {np.unravel_index(off.argmax(), off.shape)}"


def compare(rows, n, dtype, per=None, post=True, pre=True, center=False, gate=True, weights=True, offsets=False, skip=1.0, scale=1.0, seed=0):
    per = per or rows
    p = problem(rows, n, dtype, per, post, pre, gate, weights, offsets, seed)
    t = to_dev(p, dtype)
    prob = stl.ResidualProblem(rows, n, per, skip, scale, 1e-6, STL_DT[dtype])
    flags = flags_of(post, pre, center)
    kw = dict(gate=p["gate"], per=per, w_post=p["w_post"], b_post=p["b_post"], w_pre=p["w_pre"], post=post, pre=pre, center=center, skip=skip, scale=scale)
    want, want_z = lm.residual_forward(p["X"], p["H"], b_pre=p["b_pre"], **kw)
    Xout, Z = gpu_forward(prob, t, flags, dtype)
    size = np.abs(skip * p["X"]) + np.abs(want - skip * p["X"]) + np.abs(scale) * (np.abs(np.repeat(p["gate"], per, 0)[:rows]) if gate else 1.0) * (
        1.0 + np.abs(p["b_post"]) if p["b_post"] is not None else 1.0)
    close(Xout, want, size, dtype, 64, "Xout")
    if pre:
        hat_size = np.abs(want_z) + (np.abs(p["b_pre"]) if p["b_pre"] is not None else 0.0) + size / np.sqrt(np.mean(want ** 2, 1, keepdims=True)) * (
            np.abs(p["w_pre"]) if p["w_pre"] is not None else 1.0)
        close(Z, want_z, hat_size, dtype, 64, "Z")
    stream = host(Xout) if dtype == "bf16" else Xout.double().cpu().numpy()
    g = lm.residual_backward(stream, p["H"], p["dXout"], p["dZ"], **kw)
    got = gpu_backward(prob, t, Xout, flags, dtype)
    for k, v in got.items():
        sums = k not in ("dX", "dH")
        close(v, g[k], g["size"][k], "f32" if sums else dtype, rows + 64 if sums else 64, k)
    return prob, t, flags, Xout, got


# every shape of a row (threads, chunks), with the last chunk whole and not; rows that fill, and do not fill, a workgroup's turn
WIDTHS = [1, 3, 8, 64, 100, 511, 512, 513, 768, 1000, 1024, 1025, 2047, 2048, 4095, 4096, 4100, 8192, 9000, 16384, 20001, 32768]


@pytest.mark.parametrize("n", WIDTHS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("center", [False, True])
def test_widths(n, dtype, center):
    if center and n == 1:
        pytest.skip("a single element minus its mean is zero")
    compare(9, n, dtype, center=center, offsets=center, seed=n)


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 63, 513, 1030])
@pytest.mark.parametrize("n", [192, 2056])
def test_row_counts(rows, n):
    compare(rows, n, "bf16", seed=rows)
    compare(rows, n, "f32", center=True, offsets=True, seed=rows)


@pytest.mark.parametrize("per", [1, 2, 3, 50, 197, 394])
@pytest.mark.parametrize("center", [False, True])
def test_gates_shared_by_images(per, center):
    compare(394, 320, "bf16", per=per, center=center, offsets=center, scale=0.5, skip=0.75, seed=per)
    compare(101, 2052, "f32", per=min(per, 101), center=center, seed=per + 1)


def test_many_gate_rows():
    """More groups of rows than a launch has rows of workgroups for their sums."""
    compare(70001, 8, "f32", per=2, seed=5)


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("weights", [True, False])
def test_parts_left_out(post, pre, gate, weights):
    compare(37, 1032, "bf16", post=post, pre=pre, gate=gate, weights=weights, seed=11)
    compare(37, 200, "f32", post=post, pre=pre, gate=gate, weights=weights, offsets=True, center=True, skip=0.0 if gate else 1.0, seed=12)


def test_large_rows_as_measured():
    compare(2048, 4096, "bf16", seed=21)
    compare(16 * 197, 768, "bf16", per=197, center=True, offsets=True, seed=22)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_accumulation_and_repeated_bits(dtype):
    prob, t, flags, Xout, got = compare(300, 1100, dtype, per=60, seed=31)
    again, _ = gpu_forward(prob, t, flags, dtype, in_place=True)
    assert torch.equal(again, Xout)
    for _ in range(2):
        same = gpu_backward(prob, t, Xout, flags, dtype)
        assert all(torch.equal(same[k], got[k]) for k in got)
    more = gpu_backward(prob, t, Xout, flags, dtype, accumulate=1, init=2.0)
    for k in got:
        want = got[k] if k in ("dX", "dH") else got[k] + 2.0
        assert torch.equal(more[k], want), k
    # dX in the place of dXout
    t2 = dict(t, dXout=t["dXout"].clone())
    nbytes = stl.stl_residual_norm_workspace_bytes(prob, flags)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    stl.stl_residual_norm_backward(prob, Xout, t["H"], t["gate"], t["w_post"], None, t["w_pre"], t2["dXout"], t["dZ"], t2["dXout"], None, None, None,
                                   None, None, None, 0, ws, nbytes, flags)
    assert torch.equal(t2["dXout"], got["dX"])


def test_gradient_of_every_gate_row_accumulates():
    prob, t, flags, Xout, got = compare(33, 520, "bf16", per=1, seed=41)
    more = gpu_backward(prob, t, Xout, flags, "bf16", accumulate=1, init=-1.5)
    assert torch.equal(more["dgate"], got["dgate"] - 1.5)


def test_missing_upstream_gradients_are_zeros():
    p = problem(20, 640, "bf16", 20, True, True, True, True, False, 51)
    t = to_dev(p, "bf16")
    prob, flags = stl.ResidualProblem(20, 640), flags_of(True, True, False)
    Xout, _ = gpu_forward(prob, t, flags, "bf16")
    zero = torch.zeros_like(Xout)
    for name in ("dXout", "dZ"):
        a, b = (gpu_backward(prob, dict(t, **{name: v}), Xout, flags, "bf16") for v in (None, zero))
        assert all(torch.equal(a[k], b[k]) for k in a), name
    only = gpu_backward(prob, t, Xout, flags, "bf16", skip=("dX", "dgate", "dw_pre"))
    full = gpu_backward(prob, t, Xout, flags, "bf16")
    assert all(torch.equal(only[k], full[k]) for k in only)


def test_rows_that_are_not_numbers_stay_alone():
    p = problem(40, 520, "bf16", 40, True, True, True, True, False, 61)
    t = to_dev(p, "bf16")
    prob, flags = stl.ResidualProblem(40, 520), flags_of(True, True, False)
    Xout, Z = gpu_forward(prob, t, flags, "bf16")
    got = gpu_backward(prob, t, Xout, flags, "bf16")
    bad = {k: t[k].clone() for k in ("X", "H", "dXout", "dZ")}
    bad["X"][3, 5], bad["H"][17, 0] = float("nan"), float("inf")
    X2, Z2 = gpu_forward(prob, {**t, **bad}, flags, "bf16")
    rest = [i for i in range(40) if i not in (3, 17)]
    assert torch.equal(X2[rest], Xout[rest]) and torch.equal(Z2[rest], Z[rest])
    assert bool(torch.isnan(Z2[3]).all()) and bool(torch.isnan(X2[17, 0]))
    bad["dZ"][3, 5] = float("nan")
    again = gpu_backward(prob, {**t, **bad}, Xout, flags, "bf16")
    assert torch.equal(again["dX"][rest], got["dX"][rest]) and torch.equal(again["dH"][rest], got["dH"][rest])
    assert bool(torch.isnan(again["dX"][3]).all())


def test_rows_of_zeros():
    prob, flags = stl.ResidualProblem(3, 256), flags_of(True, True, True)
    z = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda")
    t = {k: None for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
    Xout, Z = gpu_forward(prob, {**t, "X": z, "H": z}, flags, "bf16")
    assert not Xout.any() and not Z.any()


def test_on_another_stream():
    p = problem(500, 1024, "bf16", 500, True, True, True, True, False, 71)
    t = to_dev(p, "bf16")
    prob, flags = stl.ResidualProblem(500, 1024), flags_of(True, True, False)
    want = gpu_forward(prob, t, flags, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        Xout, Z = torch.empty_like(t["X"]), torch.empty_like(t["X"])
        stl.stl_residual_norm_forward(prob, t["X"], t["H"], t["gate"], t["w_post"], None, t["w_pre"], None, Xout, Z, flags)
    s.synchronize()
    assert torch.equal(Xout, want[0]) and torch.equal(Z, want[1])


def test_in_a_captured_graph():
    p = problem(200, 768, "bf16", 50, True, True, True, True, True, 81)
    t = to_dev(p, "bf16")
    prob, flags = stl.ResidualProblem(200, 768, 50), flags_of(True, True, True)
    nbytes = stl.stl_residual_norm_workspace_bytes(prob, flags)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    Xout, Z, dX, dH = (torch.empty_like(t["X"]) for _ in range(4))
    dgate, dw = torch.empty((4, 768), device="cuda"), torch.empty(768, device="cuda")

    def step():
        stl.stl_residual_norm_forward(prob, t["X"], t["H"], t["gate"], t["w_post"], t["b_post"], t["w_pre"], t["b_pre"], Xout, Z, flags)
        stl.stl_residual_norm_backward(prob, Xout, t["H"], t["gate"], t["w_post"], t["b_post"], t["w_pre"], t["dXout"], t["dZ"], dX, dH, dgate, dw, None,
                                       None, None, 0, ws, nbytes, flags)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        t["X"].copy_(torch.randn_like(t["X"]))
        outs = (Xout, Z, dX, dH, dgate, dw)
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), k


def test_no_rows():
    prob = stl.ResidualProblem(0, 64)
    flags = flags_of(True, True, False)
    stl.stl_residual_norm_forward(prob, None, None, None, None, None, None, None, None, None, flags)
    dw = torch.full((64,), 3.0, device="cuda")
    stl.stl_residual_norm_backward(prob, None, None, None, None, None, None, None, None, None, None, None, dw, None, None, None, 1, None, 0, flags)
    assert bool((dw == 3.0).all())
    stl.stl_residual_norm_backward(prob, None, None, None, None, None, None, None, None, None, None, None, dw, None, None, None, 0, None, 0, flags)
    assert not dw.any()


def test_more_elements_than_32_bits_count():
    """Rows behind the 2^31st element: the same bits as those rows alone."""
    rows, n = 140000, 16384
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("not enough free memory")
    p = problem(8, n, "bf16", 8, True, True, True, True, False, 91)
    t = to_dev(p, "bf16")
    flags = flags_of(True, True, False)
    small = stl.ResidualProblem(8, n)
    Xout, Z = gpu_forward(small, t, flags, "bf16")
    got = gpu_backward(small, t, Xout, flags, "bf16")
    big = {k: torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda") for k in ("X", "H", "dXout", "dZ")}
    for k, v in big.items():
        v[-8:] = t[k]
    prob = stl.ResidualProblem(rows, n)
    out, z = torch.empty_like(big["X"]), torch.empty_like(big["X"])
    stl.stl_residual_norm_forward(prob, big["X"], big["H"], t["gate"], t["w_post"], None, t["w_pre"], None, out, z, flags)
    assert torch.equal(out[-8:], Xout) and torch.equal(z[-8:], Z) and not out[:-8].any()
    nbytes = stl.stl_residual_norm_workspace_bytes(prob, flags)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    dX, dH, dw = big["X"], z, torch.empty(n, device="cuda")
    stl.stl_residual_norm_backward(prob, out, big["H"], t["gate"], t["w_post"], None, t["w_pre"], big["dXout"], big["dZ"], dX, dH, None, None, None, dw, None, 0,
                                   ws, nbytes, flags)
    assert torch.equal(dX[-8:], got["dX"]) and torch.equal(dH[-8:], got["dH"])
    # rows of zeros add nothing: the sum of the eight rows, in another order
    assert float((dw - got["dw_pre"]).abs().max()) <= 16 * EPS * float(got["dw_pre"].abs().max()) * 8
