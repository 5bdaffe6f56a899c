"""Plain reference of rotary positions and of the page list, written from the definitions
in include/tgvkv.h; shares no code with the CUDA path."""
import math
from fractions import Fraction

import numpy as np

TWO_PI = 2 * math.pi


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=0, low=1.0, high=32.0):
    """Radians a position of every pair."""
    out = []
    for i in range(rot // 2):
        b = base
        if scaling == "base" and rot > 2:
            b = base * factor ** (rot / (rot - 2))
        f = b ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            t = original * f / TWO_PI
            if t <= low:
                f /= factor
            elif t < high:
                g = (t - low) / (high - low)
                f *= g + (1 - g) / factor
        out.append(f)
    return out


def angle(p, f):
    """p f modulo 2 pi: whole turns taken off exactly, of the double f / (2 pi)."""
    return float(Fraction(f / TWO_PI) * int(p) % 1) * TWO_PI


def turned(x, positions, freqs, rot, layout="half", sections=None, attention=1.0, mode="forward"):
    """Rows x, fp64 [T, heads, d], positions [axes, T]."""
    y = np.array(x, np.float64)
    half = rot // 2
    sections = [half] if sections is None else sections
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    a = 1.0 if mode == "move" else attention
    for t in range(x.shape[0]):
        for i in range(half):
            th = angle(positions[axis[i]][t], freqs[i])
            c, s = math.cos(th) * a, math.sin(th) * a
            if mode == "gradient":
                s = -s
            j, k = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
            y[t, :, j] = x[t, :, j] * c - x[t, :, k] * s
            y[t, :, k] = x[t, :, k] * c + x[t, :, j] * s
    return y


def partner_magnitude(x, rot, layout="half"):
    """|x1| + |x2| of every value's pair (0 for values that do not turn): what the error of
    c and s is relative to."""
    m, half = np.zeros(x.shape), rot // 2
    for i in range(half):
        j, k = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        m[..., j] = m[..., k] = np.abs(x[..., j]) + np.abs(x[..., k])
    return m


class Pages:
    """The page list, a list operation at a time."""

    def __init__(self, sets, max_pages, n_pages, page):
        self.page, self.max_pages = page, max_pages
        self.table = np.full((sets, max_pages), -1, np.int64)
        self.stack = list(range(n_pages - 1, -1, -1))

    def held(self, n):
        return -(-int(n) // self.page)

    def grow(self, lens, new):
        """False, and nothing done, where the stack holds too few."""
        want = [max(self.held(b) - self.held(a), 0) for a, b in zip(lens, new)]
        if sum(want) > len(self.stack):
            return False
        for s, n in enumerate(want):
            for i in range(n):
                self.table[s, self.held(lens[s]) + i] = self.stack.pop()
        return True

    def shrink(self, lens, new):
        for s in reversed(range(len(lens))):
            for j in reversed(range(self.held(new[s]), self.held(lens[s]))):
                self.stack.append(int(self.table[s, j]))
                self.table[s, j] = -1

    def slots(self, lens, news, H_kv, tokens):
        """[tokens, H_kv]; -1 past the last sequence's."""
        out = np.full((tokens, H_kv), -1, np.int64)
        t = 0
        for b, n in enumerate(news):
            for i in range(n):
                for g in range(H_kv):
                    j = int(lens[b * H_kv + g]) + i
                    out[t, g] = self.table[b * H_kv + g, j // self.page] * self.page + j % self.page
                t += 1
        return out
