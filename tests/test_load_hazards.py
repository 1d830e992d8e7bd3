"""What vector loads written in assembly need of the instructions before them (no GPU needed: hipcc cross-compiles for gfx950).  The compiler leaves a block of
assembly as it is and sees no load in it, so it puts no wait before one: a scalar register that a vector instruction wrote may be read by a vector load 5 wait states
later, m0 by a load into LDS 1 after a scalar instruction wrote it.  A load that comes sooner may read from the address before: of other values, or of nothing."""
import os
import re
import subprocess

import pytest


def blocks_of_assembly(tmp_path, source):
    """Every block with the instructions before it: (function, lines, index of the first line of the block, index behind the last)."""
    from paper_2112_08541_amd import buildlib
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is not installed")
    out = str(tmp_path / "x.s")
    p = subprocess.run([hipcc, *buildlib.HIPCC_FLAGS, "--cuda-device-only", "-S", os.path.join(buildlib.CSRC, source), "-o", out],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert p.returncode == 0, p.stdout[-2000:]
    found, function, lines, begin = [], None, [], None
    for line in open(out):
        if "#ASMSTART" in line:
            begin = len(lines)
        elif "#ASMEND" in line:
            found.append((function, lines, begin, len(lines)))
            begin = None
        line = line.split(";")[0].strip()
        m = re.match(r"(_Z\w+):$", line)
        if m:
            function, lines = m.group(1), []
        elif line and (not line.startswith(".") or line.startswith(".LBB")):
            lines.append(line)
    return found


def scalars_written_by_vector(line):
    """The scalar registers that a vector instruction writes (its first operand, and a carry behind it)."""
    if not line.startswith("v_"):
        return set()
    out = set()
    for operand in line.split(None, 1)[1].split(",")[:2]:
        m = re.match(r"\s*s\[(\d+):(\d+)\]$", operand) or re.match(r"\s*s(\d+)$", operand)
        if m:
            out |= set(range(int(m.group(1)), int(m.group(m.lastindex)) + 1))
        if not re.match(r"v_(readfirstlane|readlane|cmp|add_co|sub_co|addc|subb|div_scale|mad_u64|mad_i64)", line):
            return set()
        if not re.match(r"v_(add_co|sub_co|addc|subb|div_scale|mad_u64|mad_i64)", line):
            break
    return out


def states(line):
    m = re.match(r"s_nop (\w+)", line)
    return int(m.group(1), 0) + 1 if m else 1


@pytest.mark.parametrize("source", ["bgl_classes.hip"])
def test_loads_in_assembly_wait_for_their_scalars(tmp_path, source):
    seen, wrong = 0, []
    for function, lines, begin, end in blocks_of_assembly(tmp_path, source):
        for i in range(begin, end):
            if not re.match(r"(buffer|global)_load", lines[i]):
                continue
            seen += 1
            m = re.search(r"s\[(\d+):(\d+)\]", lines[i])
            used, waited, j = set(range(int(m.group(1)), int(m.group(2)) + 1)), 0, i - 1
            while waited < 5:
                if j < 0 or lines[j].startswith(".LBB") or lines[j].startswith("s_cbranch") or lines[j].startswith("s_branch"):
                    wrong.append((function, f"{waited} wait states behind a branch", lines[max(0, j):i + 1]))
                    break
                if scalars_written_by_vector(lines[j]) & used:
                    wrong.append((function, f"{waited} wait states", lines[j:i + 1]))
                    break
                if waited < 1 and re.match(r"s_\w+ m0,", lines[j]):
                    wrong.append((function, "m0", lines[j:i + 1]))
                waited += states(lines[j])
                j -= 1
    assert seen > 0 and not wrong, (seen, len(wrong), wrong[:6])


@pytest.mark.parametrize("source", ["bgl_classes.hip"])
def test_assembly_leaves_m0_as_it_was(tmp_path, source):
    """The compiler keeps m0 to itself and cannot be told that a block writes it."""
    for function, lines, begin, end in blocks_of_assembly(tmp_path, source):
        block = lines[begin:end]
        if any(re.match(r"s_\w+ m0,", line) for line in block):
            first, last = re.match(r"s_mov_b32 (s\d+), m0$", block[0]), re.match(r"s_mov_b32 m0, (s\d+)$", block[-1])
            assert first and last and first.group(1) == last.group(1), (function, block)
            assert not any(re.search(rf"\b{first.group(1)}\b", line) for line in block[1:-1])
