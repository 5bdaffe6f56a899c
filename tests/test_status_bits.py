"""The package's names of the device status bits are those of include/tgvkv.h."""
import os
import re

import paper_2606_03075_gb300 as tgvkv


def test_every_status_bit_has_its_name(repo_root):
    text = open(os.path.join(repo_root, "include", "tgvkv.h")).read()
    bits = {int(value, 16): name
            for name, value in re.findall(r"^#define TGVKV_STATUS_(\w+)\s+(0x[0-9A-Fa-f]+)u", text, re.M)}
    bits.pop(0, None)
    assert len(bits) >= 8 and all(b & (b - 1) == 0 for b in bits)
    assert tgvkv.STATUS_BITS == bits
