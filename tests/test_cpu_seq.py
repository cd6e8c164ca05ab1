"""The embedding, the norms and rotation of queries and keys, and attention with decay without a GPU: their sources compiled for the host against the stand-in for
the HIP runtime that runs a workgroup's threads as fibers (tests/cpu_emu/, tests/cpu_seq/), whole calls of the C ABI on buffers that end where their allocation
ends, under AddressSanitizer, and their results against the oracle."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import seq
from seq_cases import close, decay_case, decay_check, embed_case, head_case, narrow, turn_error, wide
from test_cpu_address_check import CLANG, CSRC, ROOT, _host_source, pytestmark  # noqa: F401


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    work = tmp_path_factory.mktemp("cpu_seq")
    (work / "include").mkdir()
    shutil.copy(ROOT / "include" / "stl.h", work / "include" / "stl.h")
    meet = {'asm volatile("s_barrier" ::: "memory");': "emu_barrier();", 'asm volatile("" ::: "memory");': "emu_wave();",
            'asm volatile("" : "+s"(out_kind));': ";", '__device__ float fmul_legacy(float a, float b) __asm("llvm.amdgcn.fmul.legacy");': "",
            r'asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(l) : "memory", "m0");': "cpu_touch16(base + off, l);"}
    srcs = []
    package = CSRC.parent
    for f in sorted(package.glob("csrc*/**/*.hip")) + sorted(package.glob("csrc*/**/*.h")):
        to = work / f.relative_to(package)
        to.parent.mkdir(parents=True, exist_ok=True)
        to = to.with_suffix(".cpp") if f.suffix == ".hip" else to
        text = f.read_text().replace("../../../include/stl.h", "stl.h").replace("../../include/stl.h", "stl.h")
        for device, host in meet.items():
            text = text.replace(device, host)
        to.write_text(_host_source(text))
        if f.suffix == ".hip" and (f.parent.name == "csrc_seq" or f.stem in ("lm_residual", "lm_residual_f32")):
            srcs.append(to)
    shutil.copy(ROOT / "tests" / "cpu_seq" / "driver.cpp", work / "driver.cpp")
    srcs.append(work / "driver.cpp")
    flags = ["-x", "c++", "-std=c++17", "-O1", "-g", "-fsanitize=address,alignment", "-fno-sanitize-recover=alignment", "-Wno-everything",
             f"-I{ROOT / 'tests' / 'cpu_seq'}", f"-I{work / 'include'}"]
    procs = [(s, subprocess.Popen([str(CLANG), *flags, "-c", str(s), "-o", str(s.with_suffix(".o"))], stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                  text=True)) for s in srcs]
    for s, p in procs:
        out, _ = p.communicate()
        assert p.returncode == 0, f"{s.name}:\n{out[-3000:]}"
    exe = work / "driver"
    res = subprocess.run([str(CLANG), "-fsanitize=address,alignment", *(str(s.with_suffix(".o")) for s in srcs), "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    count = [0]

    def run(call, numbers, inputs, outputs, was=None):
        """outputs: name -> (shape, storage type); returns them as float64.  was: what outputs hold before."""
        count[0] += 1
        d = work / f"case{count[0]}"
        d.mkdir()
        for end, arrays in (("in", inputs), ("was", was or {})):
            for k, v in arrays.items():
                if v is not None:
                    np.ascontiguousarray(v).tofile(d / f"{k}.{end}")
        size = {"bf16": 2, "f32": 4}
        args = [f"{k}={v}" for k, v in numbers.items()] + [f"{k}:{int(np.prod(s)) * size[t]}" for k, (s, t) in outputs.items()]
        r = subprocess.run([str(exe), call, str(d), *args], capture_output=True, text=True, timeout=600,
                           env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0"))
        assert r.returncode == 0, (call, numbers, (r.stdout + r.stderr)[-3000:])
        got = {k: wide(np.fromfile(d / f"{k}.out", np.uint16 if t == "bf16" else np.float32), t).reshape(s) for k, (s, t) in outputs.items()}
        shutil.rmtree(d)
        return got
    return run


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d,vocab,tokens", [(1, 1, 1, "even"), (7, 9, 5, "even"), (70, 64, 300, "zipf"), (130, 100, 2000, "even"), (300, 40, 50, "zipf"), (200, 24, 9, "one"),
                                                 (33, 2100, 12, "zipf")])
def test_embed(driver, rows, d, vocab, tokens, t):
    c = embed_case(rows, d, vocab, t, seed=rows, tokens=tokens)
    numbers = dict(rows=rows, d=d, vocab=vocab, scale=1.5, dtype=int(t == "bf16"))
    got = driver("embed_forward", numbers, {k: c[k] for k in ("token", "W")}, {"X": ((rows, d), t)})["X"]
    want = seq.embed_forward(c["token"], wide(c["W"], t), 1.5)
    close(got, want, np.abs(want), t, 0, "X")
    for accumulate in (0, 1):
        was = narrow(np.random.default_rng(1).standard_normal((vocab, d)), t)
        got = driver("embed_backward", dict(numbers, accumulate=accumulate), {k: c[k] for k in ("token", "dX")}, {"dW": ((vocab, d), t)}, {"dW": was})["dW"]
        want = seq.embed_backward(c["token"], wide(c["dX"], t), vocab, 1.5, wide(was, t) if accumulate else None)
        close(got, want["dW"], want["size"]["dW"], t, rows + 32, "dW")
        absent = np.setdiff1d(np.arange(vocab), c["token"])
        assert np.array_equal(got[absent], wide(was, t)[absent] if accumulate else np.zeros((len(absent), d)))


def test_embed_of_a_vocabulary_in_wide_ranges(driver):
    """More ids than 256 ranges of the widest have; rows that several segments share."""
    vocab, rows = 256 * 960 + 77, 600
    c = {"token": np.concatenate([np.random.default_rng(0).integers(0, vocab, 300), np.full(300, vocab - 1)]).astype(np.int64), "dX": narrow(np.random.default_rng(1).standard_normal((rows, 3)), "f32")}
    got = driver("embed_backward", dict(rows=rows, d=3, vocab=vocab, scale=1.0, dtype=0), c, {"dW": ((vocab, 3), "f32")})["dW"]
    want = np.zeros((vocab, 3))
    np.add.at(want, c["token"], wide(c["dX"], "f32"))
    assert np.abs(got - want).max() <= (rows + 32) * 2.0 ** -24 * np.abs(wide(c["dX"], "f32")).sum(0).max()
    assert np.array_equal(np.flatnonzero(got.any(1)), np.unique(c["token"]))


HEADS = [(3, 2, 1, 1, 0, 0), (5, 3, 1, 7, 6, 0), (4, 4, 2, 64, 64, 0), (3, 2, 2, 128, 128, 1), (2, 5, 0, 80, 32, 0), (3, 1, 1, 96, 48, 1), (2, 2, 1, 50, 50, 0),
         (2, 1, 1, 1000, 500, 0), (1, 1, 1, 1024, 1024, 1), (9, 3, 2, 16, 16, 0)]


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,kv,d,rot,adjacent", HEADS)
@pytest.mark.parametrize("norm", [1, 0])
def test_head_norm(driver, rows, heads, kv, d, rot, adjacent, norm, t):
    c = head_case(rows, heads, kv, d, t, seed=d)
    numbers = dict(rows=rows, heads=heads, kv_heads=kv, d=d, rot=rot, ld_q=heads * d, ld_k=kv * d, ld_qout=heads * d, ld_kout=kv * d, base=10000.0, dtype=int(t == "bf16"),
                   flags=0x800 * norm | 0x2000 * adjacent)
    kw = dict(position=c["position"], rot=rot, adjacent=bool(adjacent), norm=bool(norm))
    given = {k: c[k] for k in ("w_q", "w_k", "position")}
    shapes = {"Q": (rows, heads, d), "K": (rows, kv, d)}
    sides = "QK" if kv else "Q"
    got = driver("head_forward", numbers, {**given, **{n: c[n] for n in sides}}, {n + "out": (shapes[n], t) for n in sides})
    outs = {"d" + n: (shapes[n], t) for n in sides}
    if norm:
        outs.update({"dw_" + n.lower(): ((d,), "f32") for n in sides})
    back = driver("head_backward", numbers, {**given, **{k: c[k] for n in sides for k in (n, f"d{n}out")}}, outs)
    for n in sides:
        w = wide(c["w_" + n.lower()], t) if norm else None
        want, size = seq.head_forward(wide(c[n], t), w, **kw)
        close(got[n + "out"], want, size, t, d + 32, n, more=turn_error(c["position"], want))
        want = seq.head_backward(wide(c[n], t), wide(c[f"d{n}out"], t), w, **kw)
        close(back["d" + n], want["dx"], want["size"]["dx"], t, 2 * d + 64, "d" + n, more=turn_error(c["position"], want["size"]["dx"]))
        if norm:
            close(back["dw_" + n.lower()], want["dw"], want["size"]["dw"], "f32", rows * shapes[n][1] + d + 64, "dw")


def run_decay(driver, s, t, grads, rows, sequences, length, heads, kv, dk, dv, seq_step, token_step, offset=None, scale=0.7, in_place=0):
    numbers = dict(rows=rows, sequences=sequences, length=length, heads=heads, kv_heads=kv, dk=dk, dv=dv, seq_step=seq_step, token_step=token_step, ld_q=heads * dk, ld_k=kv * dk,
                   ld_v=kv * dv, ld_o=heads * dv, scale=scale, dtype=int(t == "bf16"), in_place=in_place)
    inputs = {k: s[k] for k in ("Q", "K", "V", "log_decay", "state")}
    inputs["offset"] = offset
    state = (sequences, heads, dk, dv)
    if not grads:
        got = driver("decay_forward", numbers, inputs, {"O": ((rows, heads, dv), t), "state_out": (state, "f32")})
        return {"O": got["O"], "state": got["state_out"]}
    inputs.update(dO=s["dO"], dstate_out=s["dstate_out"])
    got = driver("decay_backward", numbers, inputs, {"dQ": ((rows, heads, dk), t), "dK": ((rows, kv, dk), t), "dV": ((rows, kv, dv), t), "dstate_in": (state, "f32")})
    return {**got, "dstate": got.pop("dstate_in")}


DECAYS = [(1, 1, 1, 1, 1, 1), (1, 2, 2, 1, 32, 32), (2, 70, 1, 1, 33, 40), (1, 130, 2, 2, 64, 64), (3, 5, 2, 1, 16, 130), (1, 65, 1, 1, 130, 31), (1, 40, 2, 1, 256, 200)]


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("sequences,length,heads,kv,dk,dv", DECAYS)
def test_decay(driver, sequences, length, heads, kv, dk, dv, t):
    rows = sequences * length
    s = decay_case(rows, sequences, heads, kv, dk, dv, t, seed=length, states=length != 130)
    at = seq.decay_rows(sequences, length, length, 1)
    got = run_decay(driver, s, t, False, rows, sequences, length, heads, kv, dk, dv, length, 1)
    decay_check(got, s, at, t, 0.7, length, ("O", "state"))
    got = run_decay(driver, s, t, True, rows, sequences, length, heads, kv, dk, dv, length, 1)
    decay_check(got, s, at, t, 0.7, length, ("dQ", "dK", "dV", "dstate"))


@pytest.mark.parametrize("t,length,token_step", [("f32", 257, 1), ("bf16", 515, 1), ("bf16", 513, 3)])
def test_decay_in_segments(driver, t, length, token_step):
    """Long enough for several segments of a sequence, whose states are joined; whole pieces and others."""
    for dk, dv in ((16, 24), (9, 17)):
        s = decay_case(length * token_step, 1, 2, 1, dk, dv, t, seed=length + dk)
        at = [list(range(0, length * token_step, token_step))]
        for grads, names in ((False, ("O", "state")), (True, ("dQ", "dK", "dV", "dstate"))):
            got = run_decay(driver, s, t, grads, length * token_step, 1, length, 2, 1, dk, dv, 1, token_step)
            decay_check(got, s, at, t, 0.7, length, names)


def test_decay_by_position_and_packed(driver):
    for t in ("bf16", "f32"):
        s = decay_case(120, 4, 2, 2, 24, 40, t, seed=5)
        got = run_decay(driver, s, t, True, 120, 4, 30, 2, 2, 24, 40, 1, 4)
        decay_check(got, s, seq.decay_rows(4, 30, 1, 4), t, 0.7, 30, ("dQ", "dK", "dV", "dstate"))
        offset = np.array([3, 3, 70, 71, 110], np.int64)                    # rows before, behind and an empty sequence
        s = decay_case(120, 4, 2, 1, 24, 40, t, seed=6)
        at = seq.decay_rows(4, 67, 0, 0, offset, 120)
        got = run_decay(driver, s, t, False, 120, 4, 67, 2, 1, 24, 40, 0, 0, offset, in_place=1)
        _, covered = decay_check(got, s, at, t, 0.7, 67, ("O", "state"))
        assert np.array_equal(got["state"][0], s["state"][0]) and np.isnan(got["O"][~covered]).all()
        got = run_decay(driver, s, t, True, 120, 4, 67, 2, 1, 24, 40, 0, 0, offset)
        _, covered = decay_check(got, s, at, t, 0.7, 67, ("dQ", "dK", "dV", "dstate"))
        assert all(np.isnan(got[n][~covered]).all() for n in ("dQ", "dK", "dV"))


def test_decay_offsets_outside_the_rows(driver):
    """Cut off, and sequences longer than `length` too: no access outside the buffers, which the sanitizer would report."""
    s = decay_case(50, 3, 1, 1, 16, 16, "bf16", seed=7)
    for offset in ([-5, 20, 90, 2 ** 40], [40, 10, 60, 55], [-2 ** 62, -1, 0, 50]):
        offset = np.array(offset, np.int64)
        at = seq.decay_rows(3, 25, 0, 0, offset, 50)
        got = run_decay(driver, s, "bf16", False, 50, 3, 25, 1, 1, 16, 16, 0, 0, offset)
        assert np.isfinite(got["state"]).all()
        run_decay(driver, s, "bf16", True, 50, 3, 25, 1, 1, 16, 16, 0, 0, offset)
        if offset[0] <= offset[1] <= offset[2]:
            decay_check(got, s, at, "bf16", 0.7, 25, ("O", "state"))


@pytest.mark.parametrize("decays", [None, "none left", -0.0, -3e38])
def test_decay_at_its_ends(driver, decays):
    s = decay_case(70, 1, 2, 2, 20, 36, "bf16", seed=8, decays=decays)
    at = [list(range(70))]
    got = run_decay(driver, s, "bf16", False, 70, 1, 70, 2, 2, 20, 36, 70, 1)
    decay_check(got, s, at, "bf16", 0.7, 70, ("O", "state"))
    got = run_decay(driver, s, "bf16", True, 70, 1, 70, 2, 2, 20, 36, 70, 1)
    decay_check(got, s, at, "bf16", 0.7, 70, ("dQ", "dK", "dV", "dstate"))


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("name", ["Q", "K", "V"])
@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_decay_values_that_are_no_numbers(driver, t, name, value):
    """They reach their own and later tokens alone (Q: its own)."""
    s = decay_case(100, 1, 1, 1, 20, 36, t, seed=9)
    clean = run_decay(driver, s, t, False, 100, 1, 100, 1, 1, 20, 36, 100, 1)["O"]
    for at in (0, 70, 99):
        bad = dict(s, **{name: s[name].copy()})
        bad[name][at, 0, 3] = narrow(np.array([value]), t)[0]
        got = run_decay(driver, bad, t, False, 100, 1, 100, 1, 1, 20, 36, 100, 1)["O"]
        assert np.allclose(got[:at], clean[:at], rtol=2.0 ** -7, atol=1e-6)
        if name == "Q":
            assert np.array_equal(got[at + 1:], clean[at + 1:]) and not np.isfinite(got[at]).all()
        else:
            assert not np.isfinite(got[at:][..., 3]).any()
