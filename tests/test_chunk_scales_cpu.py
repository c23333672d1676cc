"""The scale of a row's logits in the chunk attention (tests/c/chunk_scales.cpp)."""
import os
import subprocess

from paper_2608_05326_amd import build as b


def test_scales_of_every_query_and_softmax_scale(tmp_path):
    exe = str(tmp_path / "scales")
    src = os.path.join(b.ROOT, "tests", "c", "chunk_scales.cpp")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                        "-fno-sanitize-recover=all", "-I", b.CSRC, src, "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr[-2000:]
