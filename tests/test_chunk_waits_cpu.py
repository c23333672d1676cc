"""The few-row path of the chunk attention waits for a page's keys by count: eight loads into LDS
may still be on their way, the values'.  That holds if the compiler keeps the keys' eight loads in
front of the values' eight: at the ordering point before the loop, and behind either wait in it
(where the loads of the next page follow the reads of the one before).  Seen in the assembly."""
import re
import subprocess

from paper_2608_05326_amd import build as b

LOAD, POINT, WAIT = "L", "|", "W"


def _sequence(tmp_path):
    """Loads into LDS, ordering points and hand-written waits, in the order of the assembly."""
    out = tmp_path / "k.s"
    cmd = [b._hipcc(), "-S", "-x", "hip", f"{b.CSRC}/block_chunk.hip", "-o", str(out),
           "--offload-device-only"] + b.FLAGS
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    seq, mine = "", False
    for line in out.read_text().splitlines():
        if "#ASMSTART" in line or "#ASMEND" in line:
            mine = "#ASMSTART" in line
        elif "global_load_lds" in line:
            seq += LOAD
        elif mine and "values behind keys" in line:
            seq += POINT
        elif mine and "s_waitcnt vmcnt(8)" in line:
            seq += WAIT
    return seq


def test_a_pages_keys_are_loaded_before_its_values(tmp_path):
    seq = _sequence(tmp_path)
    eight = LOAD * 8
    assert seq.count(LOAD) == 32 and seq.count(POINT) == 1 and seq.count(WAIT) == 2, seq
    assert re.search(rf"(^|[^L]){eight}\{POINT}{eight}($|[^L])", seq), seq
    assert len(re.findall(rf"{WAIT}{eight}(?=$|{WAIT})", seq)) == 2 or \
        re.search(rf"{WAIT}{eight}{WAIT}{eight}{eight}\{POINT}", seq), seq
