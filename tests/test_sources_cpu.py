"""What holds for every kernel's source."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_23429_gb300", "csrc")


def statements():
    """(file, line, text) of every asm statement, from its name to the parenthesis that closes it."""
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh", ".h")):
            continue
        text = open(os.path.join(CSRC, name)).read()
        for m in re.finditer(r"\basm\b(\s+volatile)?\s*\(", text):
            depth, at, quoted = 1, m.end(), False
            while depth:
                c = text[at]
                if c == '"' and text[at - 1] != "\\":
                    quoted = not quoted
                depth += 0 if quoted else (c == "(") - (c == ")")
                at += 1
            yield name, text.count("\n", 0, m.start()) + 1, text[m.start():at]


def test_loads_of_memory_stay_behind_the_wait_for_the_previous_kernel():
    """after_previous() is volatile asm, which other volatile asm is kept in order with; asm that is neither volatile nor names memory may
    be moved ahead of it, to where the kernel before may not have written yet what is loaded."""
    every = list(statements())
    assert len(every) > 50
    loads = [s for s in every if re.search(r"\bld\.(global|shared)|cp\.async|tcgen05\.ld\b", s[2])]
    assert len(loads) > 15
    free = [s for s in loads if not re.match(r"asm\s+volatile", s[2])]
    assert {s[0] for s in free} <= {"linear.cuh"} and len(free) == 2, [s[:2] for s in free]  # lin_ld1's


def test_epilogues_take_their_pointers_behind_the_wait():
    """lin_ld1 is not volatile: each kernel that uses it has the epilogue's pointers from from_here(), volatile asm behind the wait."""
    users = [n for n in sorted(os.listdir(CSRC)) if n.endswith((".cu", ".cuh")) and n != "linear.cuh" and "lin_ld1(" in open(os.path.join(CSRC, n)).read()]
    assert users == ["linear_few.cu", "linear_join.cu", "linear_tc.cuh"]
    for name in users:
        text = open(os.path.join(CSRC, name)).read()
        kernel = text[text.index("__global__"):]
        assert kernel.index("after_previous();") < kernel.index("const LinearEpilogue E = from_here(A.e);")
        assert not re.search(r"LinearEpilogue&? E = A\.e|A\.e\.(x_scale|w_scale|bias|resid|gate)\b", kernel)
    assert 'asm volatile("" : "+l"(e.x_scale)' in open(os.path.join(CSRC, "linear.cuh")).read()
