"""The LDS copies of the GEMM kernels are inline asm, so the compiler's hazard
recognizer does not see them: a VMEM instruction may read a scalar register that
a vector instruction wrote only after 5 wait states, and nothing inserts them
there.  This checks the distance in the assembly of every source with such
copies, block by block in program order (a branch target starts anew from the
block before it, the one case that falls through)."""
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


def test_the_check_itself():
    bad = "_Zk:\n v_readfirstlane_b32 s10, v6\n global_load_lds_dwordx4 v1, s[10:11]\n"
    assert len(too_close(bad)[0]) == 1
    assert len(too_close(bad.replace("v6\n", "v6\n s_nop 3\n"))[0]) == 1
    assert not too_close(bad.replace("v6\n", "v6\n s_nop 4\n"))[0]
    assert not too_close(bad.replace("s10, v6", "s12, v6"))[0]


def test_scalar_bases_of_copies_are_written_early(tmp_path):
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
