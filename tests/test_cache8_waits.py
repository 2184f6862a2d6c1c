"""Waits in front of the barriers that the 8-bit cache attention writes as inline assembly.

A pipeline step writes tiles to LDS that other waves read after the barrier, and leaves its last N LDS reads under
way across it (s_waitcnt lgkmcnt(N)). LDS instructions of a wave complete in order, so every write is there if at
least N LDS instructions follow it. The generated code is read for that.
"""
import os
import re
import subprocess

from paper_2608_01845_amd import build

WAIT = re.compile(r"\s*s_waitcnt lgkmcnt\((\d+)\)\s*$")


def steps(text):
    """(N, LDS instructions since the barrier before) of every written wait of N > 0 with a barrier behind it."""
    lds, ours, n = [], False, None
    for line in text.split("\n"):
        raw = line.strip()
        if raw.startswith(";;#ASM"):
            ours = raw.startswith(";;#ASMSTART")
            continue
        name = raw.split(" ")[0].split("\t")[0]
        m = WAIT.match(line)
        if ours and m:
            n = int(m[1])
        elif name == "s_barrier":
            if ours and n:
                yield n, lds
            lds, n = [], None
        elif name.startswith("ds_"):
            lds.append(name)


def late(n, lds):
    """Writes that the wait does not cover."""
    return [x for x in lds[len(lds) - n:] if "write" in x]


def test_the_reader_sees_a_late_write():
    wait = "\t;;#ASMSTART\n\ts_waitcnt lgkmcnt(2)\n\ts_barrier\n\t;;#ASMEND\n"
    for reads, bad in ((0, 1), (1, 1), (2, 0), (3, 0)):
        text = "\tds_write_b128 v0, v[0:3]\n" + "\tds_read_b128 v[4:7], v9\n" * reads + wait
        assert [len(late(*s)) for s in steps(text)] == [bad]


def test_tiles_are_written_before_their_barrier(tmp_path):
    out = str(tmp_path / "a.s")
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, "cache8_attention.hip"),
                        "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found = list(steps(open(out).read()))
    assert sum(any("write" in x for x in lds) for _, lds in found) >= 32   # four steps of each of eight kernels
    assert all(len(lds) >= n and not late(n, lds) for n, lds in found)
