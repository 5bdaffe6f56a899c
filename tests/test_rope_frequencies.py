"""The frequencies that a rotary plan holds, against 50-digit arithmetic, within the bound that
include/tgvkv.h states for them (no GPU).

The bound, in units u = 2^-53 of f: the exponent -2 i / rot_dim is off by u / 2, which pow takes
times ln base <= 18.5, and pow is within 2 u: 11.3 u; the division by 2 pi and its constant, 1.4 u;
LINEAR's division 1 u; BASE's base 3 u for its own pow and product and u ln(factor^..) <= 9.3 u
for that one's exponent (bases from 10^4 to 10^8).  PARTS: t is off by 13.7 u of itself, g by
13.7 u (g + r), r = low / (high - low), and 3 u g, and f (g + (1 - g) / factor) by as much over
g + (1 - g) / factor, which is largest at an end: 13.7 u times r (factor - 1) <= 3, or times
r + 1 <= 2 (r <= 1); with 4 u of its own operations 62 u in all, where 2^-47 is 64 u."""
import os
import re
from decimal import Decimal as D
from decimal import localcontext

import pytest

PI = D("3.14159265358979323846264338327950288419716939937510582097494")


@pytest.fixture(scope="module")
def api():
    from paper_2606_03075_gb300 import build
    build.build()
    from paper_2606_03075_gb300 import api as _api
    return _api


def turns(rot, base, scaling="none", factor=1.0, original=0, low=1.0, high=32.0):
    """f_i / (2 pi) of every pair, by the definition."""
    b = D(base)
    if scaling == "base" and rot > 2:
        b *= D(factor) ** (D(rot) / D(rot - 2))
    log, out = b.ln(), []
    for i in range(rot // 2):
        f = (log * D(-2 * i) / D(rot)).exp()
        if scaling == "linear":
            f /= D(factor)
        if scaling == "parts":
            t = D(original) * f / (2 * PI)
            g = min(max((t - D(low)) / (D(high) - D(low)), D(0)), D(1))
            f *= g + (1 - g) / D(factor)
        out.append(f / (2 * PI))
    return out


@pytest.mark.parametrize("rot", [2, 20, 24, 80, 96, 112, 128, 254])
@pytest.mark.parametrize("base", [1e4, 1e6])
@pytest.mark.parametrize("o", [dict(), dict(scaling="linear", factor=3.0),
                               dict(scaling="base", factor=8.0), dict(scaling="base", factor=40.0),
                               dict(scaling="parts", factor=40.0, original=4096),
                               dict(scaling="parts", factor=8.0, original=8192, high=4.0)])
def test_frequencies_are_within_the_stated_bound(api, repo_root, rot, base, o):
    header = open(os.path.join(repo_root, "include", "tgvkv.h")).read()
    stated, = re.findall(r"2\^-(\d+)\s+(?:\*\s+)?of\s+(?:\*\s+)?p f_i", header)
    plan = api.make_rope(256, rot_dim=rot, base=base, **o)
    with localcontext() as c:
        c.prec = 50
        for i, want in enumerate(turns(rot, base, **o)):
            got = D(int(plan.turns[i])) / 2 ** 64
            # a fraction of 2^64, below which it is cut off
            assert abs(got - want) <= want * D(2) ** -int(stated) + D(2) ** -64, (i, float(got / want - 1))
