"""The residual step and the vocabulary loss without a GPU: their sources compiled for the host against a stand-in for the HIP runtime that runs a
workgroup's threads as fibers (tests/cpu_emu/), whole calls of the C ABI on buffers that end where their allocation ends, under AddressSanitizer,
and their results against the oracle.  Every access of the real index arithmetic is checked, also where it depends on labels and lists."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import lm
from test_cpu_address_check import CLANG, CSRC, ROOT, _host_source, pytestmark  # noqa: F401


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    work = tmp_path_factory.mktemp("cpu_emu")
    (work / "csrc" / "lm").mkdir(parents=True)
    (work / "include").mkdir()
    shutil.copy(ROOT / "include" / "stl.h", work / "include" / "stl.h")
    # a wavefront's own LDS slabs rely on its lanes moving together: they meet where the compiler is told to keep the order
    meet = {'asm volatile("s_barrier" ::: "memory");': "emu_barrier();", 'asm volatile("" ::: "memory");': "emu_wave();"}
    srcs = []
    for f in sorted(CSRC.glob("**/*.hip")) + sorted(CSRC.glob("**/*.h")):
        to = work / "csrc" / f.relative_to(CSRC)
        to = to.with_suffix(".cpp") if f.suffix == ".hip" else to
        text = f.read_text().replace("../../../include/stl.h", "stl.h")
        for device, host in meet.items():
            text = text.replace(device, host)
        to.write_text(_host_source(text))
        if f.suffix == ".hip" and f.parent.name == "lm":
            srcs.append(to)
    shutil.copy(ROOT / "tests" / "cpu_emu" / "driver.cpp", work / "driver.cpp")
    srcs.append(work / "driver.cpp")
    flags = ["-x", "c++", "-std=c++17", "-O1", "-g", "-fsanitize=address,alignment", "-fno-sanitize-recover=alignment", "-Wno-everything",
             f"-I{ROOT / 'tests' / 'cpu_emu'}", f"-I{work / 'include'}"]
    procs = [(s, subprocess.Popen([str(CLANG), *flags, "-c", str(s), "-o", str(s.with_suffix(".o"))], stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                  text=True)) for s in srcs]
    for s, p in procs:
        out, _ = p.communicate()
        assert p.returncode == 0, f"{s.name}:\n{out[-3000:]}"
    exe = work / "driver"
    res = subprocess.run([str(CLANG), "-fsanitize=address,alignment", *(str(s.with_suffix(".o")) for s in srcs), "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    count = [0]

    def run(call, numbers, inputs, outputs):
        """outputs: name -> (shape, storage type); returns them as float64."""
        count[0] += 1
        d = work / f"case{count[0]}"
        d.mkdir()
        for k, v in inputs.items():
            if v is not None:
                v.tofile(d / f"{k}.in")
        size = {"bf16": 2, "f32": 4}
        args = [f"{k}={v}" for k, v in numbers.items()] + [f"{k}:{int(np.prod(s)) * size[t]}" for k, (s, t) in outputs.items()]
        r = subprocess.run([str(exe), call, str(d), *args], capture_output=True, text=True, timeout=600,
                           env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0"))
        assert r.returncode == 0, (call, numbers, (r.stdout + r.stderr)[-3000:])
        got = {k: _wide(np.fromfile(d / f"{k}.out", np.uint16 if t == "bf16" else np.float32), t).reshape(s) for k, (s, t) in outputs.items()}
        shutil.rmtree(d)
        return got
    return run


def _wide(a, t):
    return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64) if t == "bf16" else a.astype(np.float64)


def _narrow(a, t):
    """values in the storage type (round to nearest even), as stored"""
    a = np.ascontiguousarray(a, np.float32)
    if t == "f32":
        return a
    u = a.view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def rel(g, o):
    return float(np.linalg.norm(g - o) / max(np.linalg.norm(o), 1e-30))


# one rounding of the outputs (1.66e-3 of a bf16 tensor's norm), respectively two and the 16-bit steps between (2.4e-3): bars with the factor that the
# GPU tests' Frobenius bars have; fp32 sums of up to 2000 terms
TOL = {"bf16": 4e-3, "f32": 1e-5}


@pytest.mark.parametrize("rows,n,dtype,per,center,offsets", [
    (3, 1, "bf16", 3, False, False), (9, 100, "bf16", 4, True, True), (17, 513, "f32", 17, False, False), (5, 2050, "bf16", 1, True, False),
    (4, 4096, "f32", 2, False, True), (3, 5001, "bf16", 3, True, True), (2, 17000, "f32", 2, False, False)])
def test_residual(driver, rows, n, dtype, per, center, offsets):
    rng = np.random.default_rng(n)
    groups = -(-rows // per)
    shapes = {"X": (rows, n), "H": (rows, n), "gate": (groups, n), "w_post": (n,), "w_pre": (n,), "dXout": (rows, n), "dZ": (rows, n)}
    if offsets:
        shapes.update(b_post=(n,), b_pre=(n,))
    stored = {k: _narrow(rng.standard_normal(s), dtype) for k, s in shapes.items()}
    v = {k: _wide(a, dtype) for k, a in stored.items()}
    flags = 0xC00 | (0x1000 if center else 0)
    numbers = dict(rows=rows, n=n, per=per, skip=0.75, scale=1.5, dtype=int(dtype == "bf16"), flags=flags)
    kw = dict(gate=v["gate"], per=per, w_post=v["w_post"], b_post=v.get("b_post"), w_pre=v["w_pre"], center=center, skip=0.75, scale=1.5)
    got = driver("residual_forward", numbers, {k: a for k, a in stored.items() if k[0] != "d"}, {"Xout": ((rows, n), dtype), "Z": ((rows, n), dtype)})
    Xo, Z = lm.residual_forward(v["X"], v["H"], b_pre=v.get("b_pre"), **kw)
    assert rel(got["Xout"], Xo) <= TOL[dtype] and rel(got["Z"], Z) <= TOL[dtype]
    outs = {"dX": ((rows, n), dtype), "dH": ((rows, n), dtype), "dgate": ((groups, n), "f32"), "dw_post": ((n,), "f32"), "dw_pre": ((n,), "f32")}
    if offsets:
        outs.update(db_post=((n,), "f32"), db_pre=((n,), "f32"))
    back = driver("residual_backward", numbers, {**{k: stored[k] for k in stored if k != "X"}, "Xout": _narrow(got["Xout"], dtype)}, outs)
    want = lm.residual_backward(got["Xout"], v["H"], v["dXout"], v["dZ"], **kw)
    for k, g in back.items():
        if n > 1 or not center:
            assert np.abs(g - want[k]).max() <= TOL[dtype if k in ("dX", "dH") else "f32"] * max(np.abs(want["size"][k]).max(), 1e-3), k


def vocab_case(driver, rows, d, vocab, dtype, top=0, tau=1.0, label=True, ignored=0.0, seed=0, tol=None):
    rng = np.random.default_rng(seed)
    X, W = _narrow(rng.standard_normal((rows, d)), dtype), _narrow(rng.standard_normal((vocab, d)) * 2 / np.sqrt(d), dtype)
    inputs = {"X": X, "W": W}
    if label:
        inputs["label"] = np.where(rng.random(rows) < ignored, -100, rng.integers(0, vocab, rows)).astype(np.int64)
        inputs["dlabel"] = rng.random(rows).astype(np.float32)
    if top:
        inputs["top_id"] = np.where(rng.random((rows, top)) < 0.2, vocab, rng.integers(0, vocab, (rows, top))).astype(np.int64)
        inputs["top_logit"] = (3 * rng.standard_normal((rows, top))).astype(np.float32)
        inputs["dtop"] = rng.random(rows).astype(np.float32)
    numbers = dict(rows=rows, d=d, vocab=vocab, ntop=top, tau=tau, dtype=int(dtype == "bf16"))
    losses = {**({"label_loss": ((rows,), "f32")} if label else {}), **({"top_loss": ((rows,), "f32")} if top else {})}
    want = lm.vocab_loss(_wide(X, dtype), _wide(W, dtype), inputs.get("label"), inputs.get("top_id"), inputs.get("top_logit"), tau if top else 1.0,
                         inputs.get("dlabel"), inputs.get("dtop"))
    fwd = driver("vocab_forward", numbers, inputs, losses)
    got = driver("vocab_backward", numbers, inputs, {**losses, "dX": ((rows, d), dtype), "dW": ((vocab, d), dtype)})
    for k in losses:
        assert np.array_equal(fwd[k], got[k]) and rel(got[k], want[k]) <= 1e-5, k
    for k in ("dX", "dW"):
        assert rel(got[k], want[k]) <= TOL[dtype], k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,vocab", [(1, 32, 1), (3, 8, 5), (5, 40, 100), (64, 64, 300), (65, 33, 270), (70, 100, 520)])
def test_vocabulary_labels(driver, rows, d, vocab, dtype):
    vocab_case(driver, rows, d, vocab, dtype, ignored=0.2, seed=rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_vocabulary_teacher(driver, dtype):
    vocab_case(driver, 20, 48, 130, dtype, top=6, tau=2.0, label=False, seed=1)
    vocab_case(driver, 70, 32, 260, dtype, top=70, tau=0.5, ignored=0.4, seed=2)


def test_vocabulary_of_many_blocks(driver):
    # more blocks than the stand-in has CUs; contractions of several rounds of the ring
    vocab_case(driver, 300, 288, 1100, "bf16", ignored=0.1, seed=3)
    vocab_case(driver, 40, 256, 1700, "bf16", top=3, tau=4.0, seed=4)
    vocab_case(driver, 20, 40, 2500, "f32", top=2, seed=5)           # dX in parts
