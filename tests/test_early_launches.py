"""The rule for kernels that may start before the ones ahead of them have finished (launch.h),
read off the sources of those that launch_early starts: each is named in the rule, has one
wait, and reads nothing of memory before it."""
import os
import re

import pytest

from test_dependent_launches import CSRC, source

EARLY = {"pages_kernel": "pages.cu", "page_slots_kernel": "pages.cu", "pages_init_kernel": "pages.cu",
         "rope_kernel": "rope.cu", "rope_one_kernel": "rope.cu", "rope_write_kernel": "rope.cu"}
# what reads or writes global memory in these kernels
TOUCHES = re.compile(r"\bload\(|\*a\.|a\.\w+\[|an\.positions|set_input|set_need|make_angles|find_span|atomic|"
                     r"raise_status|__ldg|__ldcg|__ldcs")


def body(kernel):
    text = source(EARLY[kernel])
    start = re.search(r"\b%s\((?=const)" % kernel, text)
    at = text.index("{", text.index(") {", start.start()))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i]
    raise AssertionError(kernel)


def test_every_early_launch_is_listed():
    names = set()
    for file in os.listdir(CSRC):
        if file.endswith((".cu", ".cuh")):
            text = source(file)
            for m in re.finditer(r"\blaunch_early\(\s*(\w+)", text):
                local = re.findall(r"auto %s = (\w+)" % m.group(1), text[:m.start()])
                names.add(local[-1] if local else m.group(1))
    names.discard("kern")              # launch_dependent's own call of it
    assert names == set(EARLY)
    rule = open(os.path.join(CSRC, "launch.h")).read()
    for name in EARLY:
        assert re.search(r"\b%s\b" % name, rule), name


@pytest.mark.parametrize("kernel", sorted(EARLY))
def test_nothing_is_touched_before_the_wait(kernel):
    text = body(kernel)
    assert text.count("griddep_wait()") == 1
    before = text[:text.index("griddep_wait()")]
    # bodies of local functions are not run there
    before = re.sub(r"auto load = \[&\]\(.*?\n    \};", "", before, flags=re.S)
    found = TOUCHES.search(before)
    assert found is None, found.group(0)
    # what another kernel may have written is not read through the read-only path
    assert "__ldg(" not in text
