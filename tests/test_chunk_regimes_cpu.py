"""The walk of a chunk step's workgroups on the host, KV heads taken together included, and that the
steps of test_gpu_chunk_regimes.py reach what they are for (tests/c/chunk_regimes.cpp)."""
import os
import subprocess

import pytest

from chunk_regimes import STEPS, max_context
from paper_2608_05326_amd import build as b


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("regimes") / "regimes")
    src = os.path.join(b.ROOT, "tests", "c", "chunk_regimes.cpp")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                        "-fno-sanitize-recover=all", "-I", b.CSRC, src, "-o", out],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return out


def _run(args):
    r = subprocess.run([str(x) for x in args], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr[-2000:]
    return r.stdout.strip()


def test_random_steps(exe):
    assert _run([exe]) == "ok"


@pytest.mark.parametrize("name", STEPS)
def test_steps_reach_their_regime(exe, name):
    hq, hkv, held, lens, least = STEPS[name]
    got = _run([exe, hkv, hq // hkv, max_context(held, lens)] + [x for p in zip(held, lens) for x in p])
    met = dict(zip(("heads", "rounds", "few", "wide", "whole", "keys"), map(int, got.split())))
    assert all(met[k] >= x for k, x in least.items()), met
