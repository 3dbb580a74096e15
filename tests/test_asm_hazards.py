"""The LDS copies and the MFMAs of the GEMM kernels are inline asm, so the compiler's
hazard recognizer does not see them.  A VMEM instruction may read a scalar register
that a vector instruction wrote only after 5 wait states, and a vector instruction
read or write an MFMA's result only after 16 (more than the 11 of an 8-pass MFMA; each later MFMA
counts as four), and nothing inserts them there.  These tests check the distances
in the assembly of every source with such copies, in program order: a loop's exit
is the code after it."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

from paper_2507_23387_amd import build

WAIT_STATES = 5
COPY = re.compile(r"global_load_lds_\w+\s+v\d+, s\[(\d+):(\d+)\]")
VECTOR_TO_SCALAR = re.compile(r"(?:v_readfirstlane_b32|v_readlane_b32)\s+s(\d+)")
VECTOR_MASK = re.compile(r"v_\w+\s+s\[(\d+):(\d+)\]")


def too_close(assembly):
    """(function, line number, copy) of each copy that comes too soon."""
    found, copies, function, written, clock = [], 0, "", {}, 0
    for number, line in enumerate(assembly.splitlines(), 1):
        code = line.split(";")[0].strip()
        label = re.match(r"^(_Z\w+):", code)
        if label:
            function, written = label.group(1), {}
        if not code or code.endswith(":") or code.startswith("."):
            continue
        copy = COPY.search(code)
        if copy:
            copies += 1
            for r in range(int(copy.group(1)), int(copy.group(2)) + 1):
                if clock - written.get(r, -100) - 1 < WAIT_STATES:
                    found.append((function, number, code))
                    break
        one, pair = VECTOR_TO_SCALAR.match(code), VECTOR_MASK.match(code)
        if one:
            written[int(one.group(1))] = clock
        elif pair:
            for r in range(int(pair.group(1)), int(pair.group(2)) + 1):
                written[r] = clock
        nop = re.match(r"s_nop\s+(\d+)", code)
        clock += 1 + (int(nop.group(1)) if nop else 0)
    return found, copies


MFMA_WAIT = 16


def _vector_registers(operand):
    many = re.match(r"([av])\[(\d+):(\d+)\]", operand)
    if many:
        return {(many.group(1), r) for r in range(int(many.group(2)), int(many.group(3)) + 1)}
    one = re.match(r"([av])(\d+)$", operand)
    return {(one.group(1), int(one.group(2)))} if one else set()


def touched_early(assembly):
    """(function, line number, instruction) that read an inline-asm MFMA's result, or
    write to it, too soon."""
    found, mfmas, function, written, clock, inline = [], 0, "", {}, 0, False
    for number, line in enumerate(assembly.splitlines(), 1):
        if "#ASMSTART" in line or "#ASMEND" in line:
            inline = "#ASMSTART" in line
        code = line.split(";")[0].strip()
        label = re.match(r"^(_Z\w+):", code)
        if label:
            function, written = label.group(1), {}
        if not code or code.endswith(":") or code.startswith("."):
            continue
        name, _, rest = code.partition(" ")
        operands = [o.split()[0] if o.split() else "" for o in rest.split(",")]
        if name.startswith("v_mfma"):
            clock += 4
            if inline:
                mfmas += 1
                written.update((r, clock) for r in _vector_registers(operands[0]))
            continue
        if name.startswith(("v_", "ds_", "global_", "scratch_")):
            touched = set().union(*map(_vector_registers, operands))
            if any(clock - written.get(r, -100) < MFMA_WAIT for r in touched):
                found.append((function, number, code))
            if name.startswith("v_"):
                for r in _vector_registers(operands[0]):
                    written.pop(r, None)
        nop = re.match(r"s_nop\s+(\d+)", code)
        clock += 1 + (int(nop.group(1)) if nop else 0)
    return found, mfmas


def test_the_checks_themselves():
    loop = ("_Zk:\n;;#ASMSTART\n v_mfma_f32_16x16x32_f16 a[252:255], v[0:3], v[4:7], a[252:255]\n"
            ";;#ASMEND\n s_cbranch_scc0 .L1\n.L2:\n v_accvgpr_read_b32 v2, a254\n")
    assert len(touched_early(loop)[0]) == 1
    assert not touched_early(loop.replace(".L2:\n", ".L2:\n s_nop 7\n s_nop 7\n"))[0]
    assert not touched_early(loop.replace("a254", "a251"))[0]
    assert len(touched_early(loop.replace("read_b32 v2, a254", "write_b32 a254, v2"))[0]) == 1
    assert not touched_early(loop.replace("#ASMSTART", ""))[0]  # the compiler's own MFMA
    bad = "_Zk:\n v_readfirstlane_b32 s10, v6\n global_load_lds_dwordx4 v1, s[10:11]\n"
    assert len(too_close(bad)[0]) == 1
    assert len(too_close(bad.replace("v6\n", "v6\n s_nop 3\n"))[0]) == 1
    assert not too_close(bad.replace("v6\n", "v6\n s_nop 4\n"))[0]
    assert not too_close(bad.replace("s10, v6", "s12, v6"))[0]


def test_copies_and_results_keep_their_distances(tmp_path):
    sources = [s for s in build.sources() if "dma16s(" in open(s).read()]
    assert {os.path.basename(s) for s in sources} >= {"gemm.hip", "gemm_small.hip", "gemm_tile.hip"}

    def assemble(src):
        out = str(tmp_path / (os.path.basename(src) + ".s"))
        flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
        subprocess.run([build.HIPCC, *flags, *build.FILE_FLAGS.get(os.path.basename(src), []),
                        *build._includes(), "-S", "--cuda-device-only", src, "-o", out],
                       check=True, capture_output=True)
        return open(out).read()

    with ThreadPoolExecutor(4) as pool:
        for src, text in zip(sources, pool.map(assemble, sources)):
            found, copies = too_close(text)
            assert copies > 0, src
            assert not found, (os.path.basename(src), found[:5])
            found, mfmas = touched_early(text)
            assert mfmas > 0 or os.path.basename(src) != "gemm.hip"  # the others use builtins
            assert not found, (os.path.basename(src), found[:5])
