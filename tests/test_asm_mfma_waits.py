"""Built-code check of the distance between a matrix instruction and what uses its result
(CPU, needs hipcc).

The machine does not hold back a vector, LDS or memory instruction that reads (or
writes) a register which a matrix instruction has still to write: the compiler keeps
them apart by wait states, s_nop among them.  It searches the paths back through a
block's predecessors, each block once, and so may take a longer path for the
shortest: where a branch that skips a few instructions follows a matrix
instruction, what comes after the join may be too early on the path that skips.
This test compiles the kernels that have such branches to gfx950 assembly and
walks every path.  A planted hazard in a synthetic listing checks the walk itself.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2506_20686_amd import build as hipbuild

HIPCC = hipbuild.HIPCC
SOURCES = ("fwd.hip", "xat_fwd.hip", "xat_bwd.hip", "glu.hip")
needs_hipcc = pytest.mark.skipif(not (os.path.exists(HIPCC) or shutil.which("hipcc")),
                                 reason="hipcc not available")


def regs(text):
    """Vector and accumulation registers named in an operand list."""
    found = set()
    for kind, lo, hi, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        for r in range(int(lo or one), int(hi or one) + 1):
            found.add((kind, r))
    return found


def needed(op):
    """Wait states after a matrix instruction: its passes (8 of the bf16 ones used here, 16
    of the fp32 one) and 4, or 2 for fp32, as the compiler keeps in straight code."""
    if "32x32x16_bf16" in op:
        return 12
    if "32x32x2_f32" in op:
        return 18
    raise AssertionError("passes of " + op + " unknown")


def functions(text):
    """(name, [block: (label, [(line, op, operands)])]) of each function."""
    name, blocks = None, None
    for i, raw in enumerate(text.splitlines()):
        m = re.match(r"^(_Z\w+):", raw)
        if m:
            name, blocks = m.group(1), [("entry", [])]
            continue
        if name is None:
            continue
        m = re.match(r"^(\.LBB\w+):", raw)
        if m:
            blocks.append((m.group(1), []))
            continue
        body = raw.split(";")[0].strip()
        if re.match(r"^\.Lfunc_end", body):
            yield name, blocks
            name = None
        elif body and not body.startswith("."):
            op, _, rest = body.partition(" ")
            if "\t" in op:
                op, _, rest = body.partition("\t")
            blocks[-1][1].append((i + 1, op, rest))
            if op.startswith(("s_cbranch", "s_branch")):
                blocks.append((f"after{i}", []))


def scan(text):
    """(matrix instructions walked, [hazards])."""
    walked, bad = 0, []
    for name, blocks in functions(text):
        at = {label: n for n, (label, _) in enumerate(blocks)}
        after = []
        for n, (_, code) in enumerate(blocks):
            s = [n + 1] if n + 1 < len(blocks) else []
            if code and code[-1][1] == "s_endpgm":
                s = []
            elif code and code[-1][1] == "s_branch":
                s = [at[code[-1][2].strip()]]
            elif code and code[-1][1].startswith("s_cbranch"):
                s.append(at[code[-1][2].strip()])
            after.append(s)
        for n, (_, code) in enumerate(blocks):
            for k, (line, op, rest) in enumerate(code):
                if not op.startswith("v_mfma"):
                    continue
                walked += 1
                want = needed(op)
                dst = regs(rest.split(",")[0])
                best, todo = {}, [(n, k + 1, 0)]
                while todo:
                    b, start, waited = todo.pop()
                    if start == 0:
                        if best.get(b, 1 << 30) <= waited:
                            continue
                        best[b] = waited
                    left = dst
                    for line2, op2, rest2 in blocks[b][1][start:]:
                        if waited >= want:
                            break
                        if op2.startswith("v_mfma"):
                            if regs(rest2.split(",")[0]) & left:
                                waited = want  # its own wait begins
                                break
                        elif regs(rest2) & left:
                            bad.append(f"{name}: line {line2} {op2} {rest2} is {waited} states "
                                       f"after line {line} {op}, {want} needed")
                            waited = want
                            break
                        waited += int(rest2.split()[0], 0) + 1 if op2 == "s_nop" else 1
                    if waited < want:
                        todo += [(s, 0, waited) for s in after[b]]
    return walked, bad


MFMA = "\tv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], 0"


def listing(*lines):
    return "\n".join(["_Zk:", MFMA, *lines, "\ts_endpgm", ".Lfunc_end0:"])


def test_scanner_finds_a_planted_hazard():
    # the branch skips to the join at once
    short = ["\ts_cbranch_vccnz .LBB0_2", "\ts_nop 3", ".LBB0_2:", "\ts_nop 6",
             "\tv_add_f32_e32 v30, v3, v4"]
    walked, bad = scan(listing(*short))
    assert walked == 1 and len(bad) == 1 and "is 8 states" in bad[0]
    short[3] = "\ts_nop 10"
    assert scan(listing(*short)) == (1, [])
    # a loop: the use comes round, and another matrix instruction takes the result over
    loop = [".LBB0_1:", "\tv_mov_b32_e32 v40, v41", "\ts_cbranch_scc1 .LBB0_1", "\ts_nop 10",
            "\tds_write_b32 v50, v7"]
    assert scan(listing(*loop)) == (1, [])
    loop[3] = "\ts_nop 1"
    assert len(scan(listing(*loop))[1]) == 1
    assert scan(listing("\tv_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]",
                        "\ts_nop 11", "\tv_mov_b32_e32 v60, v0")) == (2, [])


@needs_hipcc
@pytest.mark.parametrize("src", SOURCES)
def test_results_are_waited_for_on_every_path(tmp_path, src):
    out = tmp_path / (src + ".s")
    ilp = hipbuild.ILP_FLAGS if src in hipbuild.MAX_ILP else []
    cmd = [HIPCC, *hipbuild.FLAGS, *ilp, "--cuda-device-only", "-S",
           "-I", os.path.join(hipbuild.ROOT, "include"), "-I", hipbuild.CSRC,
           os.path.join(hipbuild.CSRC, src), "-o", str(out)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    walked, bad = scan(out.read_text())
    assert walked > 0
    assert not bad, "\n".join(bad[:20])
