"""How a chunk step over the block cache is cut into parts: every key tile of every row tile
once, a slot for every partial result, joins that read all of them (tests/c/chunk_parts.cpp)."""
import os
import subprocess

from paper_2608_05326_amd import build as b


def test_parts_of_random_chunk_steps(tmp_path):
    exe = str(tmp_path / "parts")
    src = os.path.join(b.ROOT, "tests", "c", "chunk_parts.cpp")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                        "-fno-sanitize-recover=all", "-I", b.CSRC, src, "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr[-2000:]
