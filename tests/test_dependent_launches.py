"""The rule for kernels that may start before the ones ahead of them have finished
(launch.h), read off the sources: such a kernel has a wait, and in the order of its
source no copy into shared memory, no atomic on global memory and no read of rows
comes before the first one."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2606_03075_gb300", "csrc")
DEPENDENTS = {
    "score_tc_kernel": "score_tc.cu", "tpr_select_kernel": "select.cu", "tpr_select_warp_kernel": "select.cu",
    "decode_merge_kernel": "decode.cu", "cache_write_kernel": "cache_rows.cu",
    "cache_read_kernel": "cache_rows.cu", "chunk_stream_kernel": "chunk_stream.cu",
    "chunk_stream_merge": "chunk_stream.cu", "chunk_tile_kernel": "chunk_tile.cuh",
    "chunk_tile_merge": "chunk_merge.cu"}
# (issue() is the row streams' copies)
EARLY = re.compile(r"\b(tma_load_\w+|bulk_load|issue\s*<|refill\s*\(\)|cp\.async\.bulk\.tensor|"
                   r"take_share|atomicAdd\(work_counter|copy_rows|__ldcs|__ldcg)")


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def body(kernel, file):
    text = source(file)
    at = text.index("{", re.search(r"\b%s\(const\b|\b%s\(Problem\b" % (kernel, kernel), text).start())
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i]
    raise AssertionError(kernel)


def test_every_dependent_launch_is_listed():
    """As many kernels are named in calls of launch_dependent as the rule lists."""
    names = set()
    for file in os.listdir(CSRC):
        text = source(file)
        for m in re.finditer(r"(?<!cudaError_t )launch_dependent\(([^;]*?)dim3", text, re.S):
            arg = m.group(1)
            found = set(re.findall(r"\b(\w+_kernel|chunk_\w+_merge)\b", arg))
            if not found:                      # a local: auto kern = name<...>
                local = re.match(r"\s*(\w+)", arg).group(1)
                found = set(re.findall(r"auto %s = (\w+)" % local, text[:m.start()]))
            assert found, (file, arg)
            names |= found
    names.discard("tpr_select_general_kernel")   # same name of the local, an ordinary launch
    assert names == set(DEPENDENTS)


@pytest.mark.parametrize("kernel", sorted(DEPENDENTS))
def test_nothing_is_read_before_the_wait(kernel):
    text = body(kernel, DEPENDENTS[kernel])
    wait = text.find("griddep_wait()")
    assert wait >= 0
    early = EARLY.search(text[:wait])
    assert early is None, early.group(0)
    # rows that another kernel may have written: never through the read-only path
    assert not re.search(r"__ldg\((k|v|scores|budgets|offsets|idx|part|lens|page_table)\b", text)
