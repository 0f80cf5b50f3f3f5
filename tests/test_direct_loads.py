"""What the compiler makes around the direct loads into LDS of csrc/fp8_matmul.hip, which are inline assembly (CPU: the
source is compiled to assembly and read). A scalar register that a vector instruction wrote may be read by a load five wait
states later; the compiler counts them for its own loads, not for those. And m0 belongs to them alone."""
import os
import re
import shutil
import subprocess
import sys
from collections import defaultdict

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STATES = 5


def functions(text):
    """Instructions and labels of each function, without comments and directives."""
    out, name = defaultdict(list), None
    for line in text.splitlines():
        line = line.split(";")[0].strip()
        m = re.match(r"(_Z\w+):$", line)
        if m:
            name = m[1]
        elif name and line and (not line.startswith((".", "#")) or line.startswith(".LBB")):
            out[name].append(line)
    return out


def scalars(operand):
    """Scalar registers of an operand: s5, s[4:7], vcc, vcc_lo."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return {"s%d" % i for i in range(int(m[1]), int(m[2]) + 1)}
    if re.fullmatch(r"s\d+|vcc_lo|vcc_hi", operand):
        return {operand}
    return {"vcc_lo", "vcc_hi"} if operand == "vcc" else set()


def operands(line):
    return [x.strip().split()[0] for x in line.split(None, 1)[1].split(",")] if " " in line else []


def written_by_vector(line):
    op = line.split()[0]
    if not op.startswith("v_"):
        return set()
    ops = operands(line)
    two = op.startswith(("v_cmp", "v_div_scale", "v_add_co", "v_addc", "v_sub_co", "v_subb", "v_mad_u64", "v_mad_i64"))
    r = set().union(*(scalars(x) for x in ops[:2 if two else 1]))
    return r | ({"vcc_lo", "vcc_hi"} if op.startswith("v_cmp") and op.endswith("_e32") else set())


def hazards(lines):
    """(direct loads, pairs of a vector write and the load that reads it too early), over every way through the code."""
    at, ins = {}, []
    for line in lines:
        if line.startswith(".LBB"):
            at[line.rstrip(":")] = len(ins)
        else:
            ins.append(line)
    before = defaultdict(list)
    for i, line in enumerate(ins):
        op = line.split()[0]
        if op.startswith("s_cbranch") or op == "s_branch":
            before[at[line.split()[-1]]].append(i)
        if op not in ("s_branch", "s_endpgm"):
            before[i + 1].append(i)
    loads, early = 0, []
    for i, line in enumerate(ins):
        if not (line.startswith("buffer_load") and line.endswith(" lds")):
            continue
        loads += 1
        reads = set().union(*(scalars(x) for x in operands(line)))
        seen, todo = set(), [(j, 0) for j in before[i]]
        while todo:
            j, states = todo.pop()
            if states >= STATES or (j, states) in seen:
                continue
            seen.add((j, states))
            if written_by_vector(ins[j]) & reads:
                early.append((ins[j], line))
                continue
            wait = re.fullmatch(r"s_nop (\d+)", ins[j])
            todo += [(k, states + (int(wait[1]) + 1 if wait else 1)) for k in before[j]]
    return loads, early


def strays(lines):
    """Uses of m0 other than as the direct loads set it."""
    bad = []
    for i, line in enumerate(lines):
        if re.search(r"\bm0\b", line):
            after = [x for x in lines[i + 1:i + 3]]
            if not (line.startswith("s_mov_b32 m0,") and after[0] == "s_nop 0" and after[1].endswith(" lds")):
                bad.append(line)
    return bad


def test_planted():
    load = "buffer_load_dwordx4 v1, s[4:7], s9 offen lds"
    for lines, bad in ((["v_readfirstlane_b32 s9, v0", "s_mov_b32 m0, s1", "s_nop 0", load], 1),
                       (["v_readfirstlane_b32 s9, v0", "s_nop 2", "s_mov_b32 m0, s1", "s_nop 0", load], 0),
                       (["v_readfirstlane_b32 s8, v0", "s_mov_b32 m0, s1", "s_nop 0", load], 0),
                       (["v_readlane_b32 s6, v0, 3", "s_branch .LBB0_2", ".LBB0_1:", "s_nop 7", ".LBB0_2:", "s_nop 0", load], 1),
                       (["v_cmp_eq_u32_e64 s[8:9], v0, v1", "s_nop 3", load], 1), (["s_mov_b32 s9, s3", load], 0)):
        loads, early = hazards(lines)
        assert loads == 1 and len(early) == bad, lines
    mine = ["s_mov_b32 m0, s1", "s_nop 0", load]
    assert not strays(mine) and strays(["s_mov_b32 m0, s1", "v_movrels_b32 v1, v2", load]) and strays(mine + ["s_add_u32 s1, m0, 4"])


def test_compiled(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2604_22312_amd import build
    if not (os.path.exists(build.hipcc()) or shutil.which(build.hipcc())):
        pytest.skip("no hipcc")
    out = tmp_path / "fp8_matmul.s"
    source = os.path.join(ROOT, "paper_2604_22312_amd", "csrc", "fp8_matmul.hip")
    subprocess.run([build.hipcc()] + build.HIPCC_FLAGS + ["-I" + build.INCLUDE, "--cuda-device-only", "-S", source, "-o", str(out)],
                   check=True, capture_output=True)
    found = functions(out.read_text())
    tiles = {n: f for n, f in found.items() if "tile_kernel" in n}
    assert len(tiles) == 22   # (three shapes by two kinds of scales by three types, the largest in 16 bits)
    for name, lines in found.items():
        loads, early = hazards(lines)
        assert not early, (name, early[:3])
        assert not strays(lines), (name, strays(lines)[:3])
        assert (loads > 0) == (name in tiles), name
