"""Wait states in front of the memory instructions that the kernels write as inline assembly.

The compiler keeps its own instructions apart but does not look into an assembly string. The generated code of
every source that holds such a load is read for two rules of the CDNA instruction set: a scalar register that a
vector instruction wrote may be read by a memory instruction five wait states later, and M0 by a load to LDS one
wait state after its write. Every instruction is one wait state, s_nop n is n + 1.
"""
import glob
import os
import re
import subprocess

import pytest

from paper_2608_01845_amd import build

SOURCES = [os.path.basename(p) for p in sorted(glob.glob(os.path.join(build.CSRC, "*.hip")))
           if re.search(r"\basm\b[^;]*(buffer|global|flat|scratch)_(load|store|atomic)", open(p).read())]
LABEL = re.compile(r"^([.\w$]+):")


def scalars(operand):
    """Scalar registers of an operand, as numbers and names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.fullmatch(r"s(\d+)", operand)
    if m:
        return {int(m[1])}
    return {"vcc"} if operand.startswith("vcc") else {"m0"} if operand == "m0" else set()


class Code:
    """Instructions of one assembly file: (name, operands, within an assembly string)."""

    def __init__(self, text):
        self.ins, self.labels, ours = [], {}, False
        for line in text.split("\n"):
            raw = line.strip()
            if raw.startswith(";;#ASM"):
                ours = raw.startswith(";;#ASMSTART")
                continue
            line = raw.split(";")[0].split("//")[0].strip()
            m = LABEL.match(line)
            if m:
                self.labels[m[1]] = len(self.ins)
                continue
            if not line or line.startswith("."):
                continue
            name, _, rest = line.partition(" ")
            if "\t" in name:
                name, _, rest = line.partition("\t")
            self.ins.append((name, [x.strip() for x in re.split(r",(?![^\[]*\])", rest.strip())], ours))
        self.at = {}                                   # instruction -> branches that arrive there
        for i, (name, ops, _) in enumerate(self.ins):
            if name.startswith(("s_branch", "s_cbranch")) and ops[0] in self.labels:
                self.at.setdefault(self.labels[ops[0]], []).append(i)

    def before(self, i, left):
        """Instructions that can run up to `left` wait states before instruction i: (index, wait states between)."""
        todo, seen = [(i, 0)], set()
        while todo:
            j, gap = todo.pop()
            if (j, gap) in seen or gap >= left:
                continue
            seen.add((j, gap))
            prev = list(self.at.get(j, ()))
            if j > 0 and self.ins[j - 1][0] not in ("s_branch", "s_endpgm", "s_setpc_b64"):
                prev.append(j - 1)
            for k in prev:
                yield k, gap
                name, ops, _ = self.ins[k]
                todo.append((k, gap + (int(ops[0], 0) + 1 if name == "s_nop" else 1)))


def written(name, ops):
    """Scalar registers that a vector instruction writes."""
    n = 2 if "_co_" in name or name.startswith("v_div_scale") else 1
    return set().union(*(scalars(x) for x in ops[:n])) if name.startswith("v_") else set()


def hazards(text):
    code = Code(text)
    loads, bad = 0, []
    for i, (name, ops, ours) in enumerate(code.ins):
        if not ours or not name.startswith(("buffer_", "global_", "flat_", "scratch_")):
            continue
        loads += 1
        reads = set().union(*(scalars(x.split(" ")[0]) for x in ops))
        lds = any(re.search(r"\blds\b", x) for x in ops)
        for k, gap in code.before(i, 5):
            kn, ko, _ = code.ins[k]
            if reads & written(kn, ko):
                bad.append((i, gap, f"{kn} {', '.join(ko)}"))
            elif lds and gap < 1 and kn.startswith("s_") and "m0" in scalars(ko[0]):
                bad.append((i, gap, f"{kn} {', '.join(ko)}"))
    return loads, bad


def test_the_reader_sees_hazards():
    load = "\t;;#ASMSTART\n\ts_mov_b32 m0, s9\n\ts_nop {}\n\tbuffer_load_dwordx4 v3, s[4:7], 0 offen lds\n\t;;#ASMEND\n"
    for n, bad in ((0, 1), (2, 1), (3, 0)):
        assert hazards("\tv_readfirstlane_b32 s6, v204\n" + load.format(n)) == (1, [(3, n + 2, "v_readfirstlane_b32 s6, v204")] * bad)
    assert hazards("\tv_readfirstlane_b32 s8, v204\n" + load.format(0))[1] == []
    assert hazards("\tv_cmp_gt_i32_e64 s[6:7], v0, v1\n\ts_mov_b32 s4, 0\n" + load.format(1))[1]
    jump = "\tv_readfirstlane_b32 s4, v1\n\ts_cbranch_scc1 .LBB0_2\n\ts_endpgm\n.LBB0_1:\n\ts_nop 9\n.LBB0_2:\n"
    assert len(hazards(jump + load.format(1))[1]) == 1 and not hazards(jump + load.format(3))[1]
    bare = "\t;;#ASMSTART\n\ts_mov_b32 m0, s9\n\tbuffer_load_dword v3, s[4:7], 0 offen lds\n\t;;#ASMEND\n"
    assert len(hazards(bare)[1]) == 1


@pytest.mark.parametrize("src", SOURCES)
def test_written_memory_instructions_keep_their_distance(src, tmp_path):
    out = str(tmp_path / "a.s")
    r = subprocess.run([build.HIPCC, *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, src), "-o", out],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    loads, bad = hazards(open(out).read())
    assert loads > 0
    assert not bad, (len(bad), bad[:8])


def test_sources_with_written_loads_are_found():
    assert "cache_attention.hip" in SOURCES
