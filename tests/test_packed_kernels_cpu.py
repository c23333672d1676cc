"""Registers of the prompt-attention and block-cache kernels: compiled for gfx950, none of
them spills to scratch memory, and each fits the waves its launch counts on."""
import re
import subprocess

import pytest

from paper_2608_05326_amd import build as b


@pytest.mark.parametrize("src,kernels,waves", [("prompt_attend.hip", 2, 2), ("block_cache.hip", 5, 2)])
def test_kernels_do_not_spill(tmp_path, src, kernels, waves):
    cmd = [b._hipcc(), "-c", "-x", "hip", f"{b.CSRC}/{src}", "-o", str(tmp_path / "k.o"),
           "--offload-device-only", "-Rpass-analysis=kernel-resource-usage"] + b.FLAGS
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    scratch = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    occupancy = [int(x) for x in re.findall(r"Occupancy \[waves/SIMD\]: (\d+)", r.stderr)]
    assert len(names) == len(scratch) == len(occupancy) == kernels
    assert not {n: x for n, x in zip(names, scratch) if x}
    assert min(occupancy) >= waves
