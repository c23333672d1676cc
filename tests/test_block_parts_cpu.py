"""How a decode step of the block cache is cut into parts: every block once, a slot for every
segment, joins that read all of a pair's segments (tests/c/block_parts.cpp)."""
import os
import subprocess

from paper_2608_05326_amd import build as b


def test_parts_of_random_steps(tmp_path):
    exe = str(tmp_path / "parts")
    src = os.path.join(b.ROOT, "tests", "c", "block_parts.cpp")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined",
                        "-fno-sanitize-recover=all", "-I", b.CSRC, src, "-o", exe],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr[-2000:]
