"""The follow-up example: eviction, paged cache, question, answer, read-back.

Both attentions see the same rows.  The paged one rounds its weights and its output
to bf16 (2^-9 relative each), so they differ by at most
2^-9 (sum_j A_ij |v_j| + |o|), besides the fp32 accumulation.  The values have a
standard deviation of about 1 (sum_j A_ij |v_j| below 2 for averages over tens of
rows) and the largest of the outputs is above 0.25: at most 9 * 2^-9 of it."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    from paper_2606_03075_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location(
        "follow_up", os.path.join(os.path.dirname(HERE), "examples", "follow_up.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("fmt,share", [("bf16", 1.0), ("int8", 33 / 64), ("int4", 17 / 64)])
def test_follow_up(example, fmt, share):
    from paper_2606_03075_gb300 import synth
    wl = synth.WORKLOADS["tiny"]
    held, rows, err = example.follow_up(wl, wl.ratios[0], fmt, question=20, answer=3)
    assert err <= 9 * 2.0 ** -9
    # whole pages of stored rows: 2 d, d + d / 32 or d / 2 + d / 32 bytes a row
    slots = held / (2 * 2 * wl.d * share)
    assert slots == int(slots) and slots % 64 == 0 and slots >= rows / (2 * 2 * wl.d)
