"""Host check of the rules that cut the calls from the loss to the gradient
(layer_plans.hpp, compiled for the host): plans cover their sizes, and the sizes
of the GPU tests reach every kernel that the rules choose between.  No GPU is
used."""
import os
import shutil
import subprocess

import pytest

from tests import test_gpu_loss as loss
from tests import test_gpu_weight_grad as wgrad

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = shutil.which("g++") or (HIPCC if os.path.exists(HIPCC) else None)
TYPES = {"float32": 0, "bfloat16": 1}
BLOCK = {0: 1024, 1: 2048}  # entries of a block of logits


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    if CXX is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("plans") / "layer_plans_check")
    cmd = [CXX, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2002_09018_amd", "csrc"),
           "-I", os.path.join(ROOT, "include"), os.path.join(HERE, "layer_plans_check.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr

    def ask(lines):
        r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
        out = r.stdout.split("\n")
        assert r.returncode == 0 and out[len(lines):] == ["ok", ""], r.stdout[-2000:]
        return [tuple(int(x) for x in line.split()) for line in out[:len(lines)]]
    return ask


def test_logprobs_tests_reach_every_kernel(plans):
    """Every number of waves over several blocks to a wave, whole rows and parts,
    with and without alternatives, in both types."""
    cases = [(n, v, k, d) for n, v in loss.LONG for k in loss.LONG_K for d in TYPES.values()]
    reached = set()
    for (n, v, k, d), (waves, parts, per_part) in zip(cases, plans([f"logprobs {n} {v} {k} {d}" for n, v, k, d in cases])):
        if per_part > waves * BLOCK[d] or parts > 1:
            reached.add((d, waves, parts > 1, k > 0))
    for d in TYPES.values():
        for k in (False, True):
            assert {(w, p) for e, w, p, q in reached if e == d and q == k} == {
                (1, False), (2, False), (4, False), (8, False), (4, True)}, (d, k)


def test_gradient_tests_reach_two_blocks_of_a_wave(plans):
    for (n, v, t), (per, segs) in zip(loss.LONG_GRAD, plans([f"grad {n} {v} {TYPES[t]}" for n, v, t in loss.LONG_GRAD])):
        assert per == 2 and segs > 2, (n, v, t)
    assert {t for _, _, t in loss.LONG_GRAD} == set(TYPES)


def test_weight_grad_tests_reach_every_tile(plans):
    cases = [(n, c, o, d) for n, c, o in wgrad.SHAPES + wgrad.LARGE for d in TYPES.values()]
    reached = {(d, m, n, s > 1) for (_, _, _, d), (m, n, s) in zip(
        cases, plans([f"wgrad {n} {c} {o} {d}" for n, c, o, d in cases]))}
    tiles = {0: [(128, 128), (256, 256)], 1: [(128, 128), (128, 256), (256, 256)]}
    assert reached == {(d, m, n, s) for d in tiles for m, n in tiles[d] for s in (False, True)}
