"""Host check of the rules that cut the products of the layers around the step
(stream_plans.hpp, compiled for the host): plans cover their products, their buffers lie
apart, and the sizes of the GPU tests reach every kernel that the rules choose for sizes
up to those of the tests.  No GPU is used."""
import math
import os
import random
import shutil
import subprocess

import pytest

from tests import test_gpu_model_layers as layers

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = shutil.which("g++") or (HIPCC if os.path.exists(HIPCC) else None)
TYPES = {"float32": 0, "bfloat16": 1}


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if CXX is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("plans") / "stream_plans_check")
    cmd = [CXX, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2002_09018_amd", "csrc"),
           "-I", os.path.join(ROOT, "include"), os.path.join(HERE, "stream_plans_check.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr

    def run(lines):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=300)
        out = r.stdout.split("\n")
        assert r.returncode == 0 and out[len(lines):] == ["ok", ""], r.stdout[-2000:]
        return [[int(x) for x in line.split()] for line in out[:len(lines)]]
    return run


def vocab_kernels(ask, sizes):
    """{(product, type, terms, shape, in parts)} of sizes (rows, dim, vocab, type, gradient's type, copied)."""
    found = set()
    fwd = ask(["vocab %d %d %d %d %d" % (n, d, v, t, c) for n, d, v, t, _, c in sizes])
    bwd = ask(["vgrad %d %d %d %d %d %d" % x for x in sizes])
    for (n, d, v, t, g, c), a, b in zip(sizes, fwd, bwd):
        terms = 3 if t == 0 or g == 0 else 1
        for i in (1, 3):
            found.add(("loss", t, 0, a[i], a[i + 1] > 1))
        for i in (1, 7):
            found |= {("dz", t, 0, b[i], b[i + 1] > 1), ("dX", t, 0, b[i + 2], b[i + 3] > 1),
                      ("dW", t, terms, b[i + 4], b[i + 5] > 1)}
        if b[13]:
            found.add(("dX and dW", t, terms, b[14] > 1, b[15] > 1))
    return found


def ffn_kernels(ask, sizes):
    """The same of sizes (rows, dim, width, type, gradient's type, copied)."""
    found = set()
    for (n, d, w, t, g, _), b in zip(sizes, ask(["fgrad %d %d %d %d %d %d" % x for x in sizes])):
        found |= {("pair", t, 0, b[0], b[1] > 1), ("dX", t, 0, b[2], b[3] > 1),
                  ("dW", t, 3 if t == 0 or g == 0 else 1, b[4], b[5] > 1)}
        if b[6]:
            found.add(("dX and dW", t, 3 if t == 0 else 1, b[7] > 1, b[8] > 1))
    for (n, d, w, t, _, _), a in zip(sizes, ask(["ffn %d %d %d %d %d" % (x[:4] + x[5:]) for x in sizes])):
        found.add(("pair", t, 0, a[0], a[1] > 1))
    return found


def copies(dtype, cols):
    """Whether the tests' layouts of a matrix with rows of `cols` are such that it is copied:
    always, or in some (aligned rows lie as the products read them in the first)."""
    return (1,) if dtype == 0 or cols % 8 else (1, 0)


def drawn(seed, count, hi):
    r = random.Random(seed)

    def size(lo, top):
        return int(math.exp(r.uniform(math.log(lo), math.log(top))))
    out = []
    for _ in range(count):
        x = (size(1, 8192), size(8, 4096), size(8, hi), r.randint(0, 1), r.randint(0, 1))
        out.append(x + (1 if x[3] == 0 else r.randint(0, 1),))
    return out


def test_vocab_sizes_reach_every_kernel(ask):
    tested = [(n, d, v, t, g, c) for n, d, v in layers.VOCAB for t in (0, 1) for g in (0, 1) for c in copies(t, d)]
    tested += [(n, d, v, TYPES[t], g, 1) for n, d, v, t in layers.PIECES for g in (TYPES[t], 0)]
    tested += [(n, d, v, TYPES[t], TYPES[g], int(c)) for n, d, v, t, g, c in layers.VOCAB_MORE]
    missing = vocab_kernels(ask, drawn(1, 20000, 40000)) - vocab_kernels(ask, tested)
    assert not missing


def test_pieces(ask):
    for n, d, v, t in layers.PIECES:
        dt = TYPES[t]
        (fwd,), (bwd,) = ask([f"vocab {n} {d} {v} {dt} 1"]), ask([f"vgrad {n} {d} {v} {dt} {dt} 1"])
        assert fwd[0] > 1 or bwd[0] > 1, (n, d, v, t)
    # a table that is read as it lies is one piece of the loss, whatever its size
    assert ask(["vocab 8192 4096 131072 1 0"])[0][0] == 1


def test_ffn_sizes_reach_every_kernel(ask):
    tested = [(n, d, w, t, g, c) for n, d, w in layers.FFN for t in (0, 1) for g in (0, 1) for c in copies(t, w)]
    tested += [(n, d, w, TYPES[t], TYPES[g], copies(TYPES[t], w)[-1]) for n, d, w, t, g in layers.FFN_MORE]
    missing = ffn_kernels(ask, drawn(2, 20000, 8192)) - ffn_kernels(ask, tested)
    assert not missing
