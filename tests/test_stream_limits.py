"""Host checks of the rules in stream_plans.hpp, compiled for the host.  What a call of the
loss from the last activations refuses: products of 2^22 tiles or more, and nothing else,
wherever the table lies.  The GPU tests' sizes reach every product that forms dX of bf16
inputs from a gradient in terms.  No GPU is used."""
import math
import os
import random
import shutil
import subprocess

import pytest

from tests import test_gpu_model_layer_edges as edges
from tests.test_stream_plans import ask, drawn  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = shutil.which("g++") or (HIPCC if os.path.exists(HIPCC) else None)


def test_many_logits_are_taken(tmp_path):
    if CXX is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path / "stream_limits_check")
    cmd = [CXX, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2002_09018_amd", "csrc"),
           "-I", os.path.join(ROOT, "include"), os.path.join(HERE, "stream_limits_check.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    sizes = [(65536, 1024, 131072), (32768, 1024, 262144), (16384, 1024, 524288), (16777216, 1024, 512),
             (32768, 8, 262144), (4200000, 8, 2000)]
    lines = [(n, d, v, t, c) for n, d, v in sizes for t in (0, 1) for c in (0, 1)]
    # 256 x 256 tiles: one fewer than 2^22 (2047 2049 of them), and 2^22
    lines += [(2047 * 256, 64, 2049 * 256, 1, 0), (2048 * 256, 64, 2048 * 256, 1, 0)]
    r = subprocess.run([exe], input="\n".join(" ".join(map(str, x)) for x in lines) + "\n", capture_output=True,
                       text=True, timeout=300)
    out = r.stdout.split("\n")
    assert r.returncode == 0 and out[len(lines):] == ["ok", ""], r.stdout[-2000:]
    for x, line in zip(lines, out):
        assert int(line.split()[0]) == (x != lines[-1]), (x, line)


def dx_kernels(ask, kind, sizes):  # noqa: F811
    """{(tile, in parts, in pieces of the vocabulary)} of dX, sizes (rows, dim, n, copied)."""
    at = (3, 9) if kind == "vgrad" else (2,)
    found = set()
    for b in ask([f"{kind} %d %d %d 1 0 %d" % x for x in sizes]):
        found |= {(b[i], b[i + 1] > 1, kind == "vgrad" and b[0] > 1) for i in at}
    return found


@pytest.mark.parametrize("kind,tested,top", [("vgrad", edges.VOCAB_TERMS, 40000), ("fgrad", edges.FFN_TERMS, 8192)])
def test_sizes_reach_every_dx_of_terms(ask, kind, tested, top):  # noqa: F811
    tested = [x for x in tested if x[3] or (x[1] if kind == "vgrad" else x[2]) % 8 == 0]
    some = [x[:3] + (x[5],) for x in drawn(9, 20000, top)]
    assert not dx_kernels(ask, kind, some) - dx_kernels(ask, kind, tested)


def test_sizes_reach_every_product_of_few_rows(ask):  # noqa: F811
    """bf16 gradients of up to 32 rows, whose dz has two terms."""
    def kernels(sizes):
        found = set()
        for x, b in zip(sizes, ask(["vgrad %d %d %d 1 1 %d" % x for x in sizes])):
            found |= {("dX", b[3], b[4] > 1), ("dW", b[5], b[6] > 1)}
            if b[13]:
                found.add(("dX and dW", b[14] > 1, b[15] > 1))
        return found
    r = random.Random(5)
    some = [tuple(int(math.exp(r.uniform(math.log(lo), math.log(hi)))) for lo, hi in ((1, 33), (8, 4096), (8, 200000)))
            for _ in range(20000)]
    some = [x + (1 if x[1] % 8 else r.randint(0, 1),) for x in some]
    assert not kernels(some) - kernels(edges.FEW_TERMS)
