"""A launch with more than 64 KiB of dynamic LDS asks the runtime for it first, and
looks at the answer: every launch with dynamic LDS in the sources either calls set_lds
in the same function or shows at compile time that it needs no more."""
import os
import re

import pytest

from paper_2507_23387_amd import build


def arguments(text, start):
    """The arguments of the call whose opening parenthesis is at `start`."""
    depth, args, at = 0, [], start + 1
    for i in range(start, len(text)):
        c = text[i]
        if c in "([{":
            depth += 1
        elif c in ")]}":
            depth -= 1
        if depth == 1 and c == ",":
            args.append(text[at:i].strip())
            at = i + 1
        if depth == 0:
            return [*args, text[at:i].strip()]
    raise AssertionError("no closing parenthesis")


def unguarded(source):
    """(line number, LDS argument) of each launch that neither asks nor shows."""
    code = re.sub(r"//[^\n]*", "", source)
    found = []
    for call in re.finditer(r"hipLaunchKernelGGL\(", code):
        lds = arguments(code, call.end() - 1)[3]
        # Back to the start of the function: the last brace at the start of a line.
        body = code[max(0, code.rfind("\n}", 0, call.start())):call.start()]
        shown = re.search(r"static_assert\(\s*(\w+) <= 64 \* 1024", body)
        if lds != "0" and "set_lds(" not in body and not (shown and shown.group(1) == lds):
            found.append((code.count("\n", 0, call.start()) + 1, lds))
    return found


def test_the_check_itself():
    launch = "void f() {\n%s  hipLaunchKernelGGL((k<1, 2>), dim3(a, b), dim3(64), %s, stream, g);\n}\n"
    assert not unguarded(launch % ("", "0"))
    assert unguarded(launch % ("", "kBytes")) == [(2, "kBytes")]
    assert not unguarded(launch % ("  const hipError_t e = set_lds(&k, kBytes, done);\n", "kBytes"))
    assert not unguarded(launch % ('  static_assert(kBytes <= 64 * 1024, "");\n', "kBytes"))
    assert unguarded(launch % ('  static_assert(kOther <= 64 * 1024, "");\n', "kBytes"))
    asked = "void g() {\n  set_lds(&k, kBytes, done);\n}\n"
    assert unguarded(asked + launch % ("", "4 * n"))


@pytest.mark.parametrize("path", build.sources(), ids=os.path.basename)
def test_launches_ask_for_their_lds(path):
    assert not unguarded(open(path).read())
