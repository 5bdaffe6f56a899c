"""The follow-up example over 4-bit floats, and its pages: taken for what the sets hold, and
for that alone.  The tolerance is that of the other formats (test_follow_up_gpu.py): weights
and output in bf16 against the same rows."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("name,question,answer", [("tiny", 20, 3), ("tiny", 1, 130)])
def test_follow_up_over_4_bit_floats(name, question, answer):
    from paper_2606_03075_gb300 import build, synth
    build.build()
    spec = importlib.util.spec_from_file_location(
        "follow_up", os.path.join(os.path.dirname(HERE), "examples", "follow_up.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    wl = synth.WORKLOADS[name]
    held, rows, err = example.follow_up(wl, wl.ratios[0], "fp4", question=question, answer=answer)
    # two roundings of 2^-8 each, of weights and output: at most 2^-7 sum_j A_ij |v_j|, whose
    # sum is below 2 and the largest output above 0.25
    assert err <= 8 * 2.0 ** -7
    slots = held / (2 * 2 * wl.d * 17 / 64)
    assert slots == int(slots) and slots % 64 == 0 and slots >= rows / (2 * 2 * wl.d)
