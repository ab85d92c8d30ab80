"""Built-code check, as test_asm_mfma_waits.py makes it, of matrix instructions that read
another's unfinished result, and of every source that has matrix instructions (CPU, needs
hipcc).

A matrix instruction may take the result of the one before as its C at once where it is the
same registers.  As its A or B, or as a C that only overlaps it, the result has to be
finished, as for any other reader: an operand is read at the start, and nothing holds it back."""
import concurrent.futures
import os
import re
import subprocess

import pytest

from paper_2506_20686_amd import build as hipbuild
from test_asm_mfma_waits import HIPCC, functions, listing, needed, needs_hipcc, regs

SOURCES = sorted(os.path.basename(s) for s in hipbuild.sources())
WITH = ("bwd.hip", "dkdv.hip", "dkdv_end.hip", "fwd.hip", "glu.hip", "lin.hip", "lnl.hip",
        "trn.hip", "xat_bwd.hip", "xat_fwd.hip")


def states(op):
    """Wait states until a result is there: 4 passes and 4 for the 16 x 16 x 32 products."""
    return 8 if "16x16x32_bf16" in op else needed(op)


def reads_early(op, dst, want, op2, rest2, waited):
    """Whether the matrix instruction op2 reads what op (to dst) has not finished; None where
    op2 goes on with the result itself."""
    d, a, b, c = (x.strip() for x in rest2.split(",")[:4])
    if waited < want and (regs(a) | regs(b)) & regs(dst):
        return True
    if regs(c) & regs(dst) and (c != dst or op2 != op):
        return waited < want - 2  # read two states later than A and B
    return None if regs(d) & regs(dst) else False


def scan(text):
    """(matrix instructions walked, [hazards])."""
    walked, bad = 0, []
    for name, blocks in functions(text):
        at = {label: n for n, (label, _) in enumerate(blocks)}
        after = []
        for n, (_, code) in enumerate(blocks):
            s = [n + 1] if n + 1 < len(blocks) else []
            last = code[-1][1] if code else ""
            if last == "s_endpgm":
                s = []
            elif last == "s_branch":
                s = [at[code[-1][2].strip()]]
            elif last.startswith("s_cbranch"):
                s.append(at[code[-1][2].strip()])
            after.append(s)
        for n, (_, code) in enumerate(blocks):
            for k, (line, op, rest) in enumerate(code):
                if not op.startswith("v_mfma"):
                    continue
                walked += 1
                want, dst = states(op), rest.split(",")[0].strip()
                left, best, todo = regs(dst), {}, [(n, k + 1, 0)]
                while todo:
                    b, start, waited = todo.pop()
                    if start == 0:
                        if best.get(b, 1 << 30) <= waited:
                            continue
                        best[b] = waited
                    for line2, op2, rest2 in blocks[b][1][start:]:
                        if waited >= want:
                            break
                        if op2.startswith("v_mfma"):
                            early = reads_early(op, dst, want, op2, rest2, waited)
                            if early is None:  # its own wait begins
                                waited = want
                                break
                        else:
                            early = bool(regs(rest2) & left)
                        if early:
                            bad.append(f"{name}: line {line2} {op2} {rest2} is {waited} states "
                                       f"after line {line} {op}, {want} needed")
                            waited = want
                            break
                        waited += int(rest2.split()[0], 0) + 1 if op2 == "s_nop" else 1
                    if waited < want:
                        todo += [(s, 0, waited) for s in after[b]]
    return walked, bad


def mfma(d, a, b, c, kind="32x32x16_bf16"):
    return f"\tv_mfma_f32_{kind} {d}, {a}, {b}, {c}"


def test_scanner_finds_planted_operands():
    # listing() starts with a product to v[0:15]
    a, b, other = "v[20:23]", "v[24:27]", "v[32:47]"
    assert scan(listing(mfma("v[0:15]", a, b, "v[0:15]"))) == (2, [])  # the chain of a sum
    for early in (mfma(other, "v[4:7]", b, "0"), mfma(other, a, "v[12:15]", "0"),
                  mfma(other, a, b, "v[8:23]"), mfma("v[0:15]", "v[0:3]", b, "v[0:15]")):
        assert len(scan(listing(early))[1]) == 1, early
        assert len(scan(listing("\ts_nop 8", early))[1]) == 1, early
        assert scan(listing("\ts_nop 11", early)) == (2, []), early
    # around a branch
    skip = ["\ts_cbranch_vccnz .LBB0_2", "\ts_nop 9", ".LBB0_2:", "\ts_nop 2",
            mfma(other, "v[4:7]", b, "0")]
    walked, bad = scan(listing(*skip))
    assert walked == 2 and len(bad) == 1 and "is 4 states" in bad[0]
    # other registers, and another kind's chain of the same ones
    assert scan(listing(mfma(other, a, b, other))) == (2, [])
    assert len(scan(listing(mfma("v[0:15]", "v20", "v21", "v[0:15]", "32x32x2_f32")))[1]) == 1
    # the short products
    short = [mfma("v[60:63]", a, b, "0", "16x16x32_bf16"), "\ts_nop 6", "\tv_mov_b32_e32 v70, v61"]
    assert len(scan(listing(*short))[1]) == 1
    short[1] = "\ts_nop 7"
    assert scan(listing(*short)) == (2, [])


def assembly(src, to):
    ilp = hipbuild.ILP_FLAGS if src in hipbuild.MAX_ILP else []
    cmd = [HIPCC, *hipbuild.FLAGS, *ilp, "--cuda-device-only", "-S",
           "-I", os.path.join(hipbuild.ROOT, "include"), "-I", hipbuild.CSRC,
           os.path.join(hipbuild.CSRC, src), "-o", str(to)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return to.read_text()


@needs_hipcc
def test_no_result_of_any_source_is_read_early(tmp_path):
    with concurrent.futures.ThreadPoolExecutor(8) as pool:
        texts = list(pool.map(lambda s: assembly(s, tmp_path / (s + ".s")), SOURCES))
    for src, text in zip(SOURCES, texts):
        walked, bad = scan(text)
        assert walked == len(re.findall(r"^\s+v_mfma", text, re.M)), src
        assert walked > 0 or src not in WITH, src
        assert not bad, src + "\n" + "\n".join(bad[:20])
