"""Refusals of the paged-cache calls that concern the layout of their integer arrays
(no GPU: nothing is launched)."""
import ctypes

import pytest

from test_paged_cache_abi import FAKE, FAKE2, P, desc, lib, pools  # noqa: F401 (lib: the fixture)

INVALID = 1
OFF_BY_TWO = P(0x10002)


@pytest.mark.parametrize("name", ["table", "lens", "off", "out"])
def test_misaligned_integers_of_a_write(lib, name):
    """A pointer that the kernels could not load 4 bytes through is refused."""
    a = dict(table=FAKE, lens=FAKE, off=FAKE, out=FAKE2)
    a[name] = P(0x200002) if name == "out" else OFF_BY_TWO
    d = ctypes.byref(desc())
    assert lib.tgvkv_cache_write(d, pools(), a["table"], a["lens"], FAKE, 256, 128, FAKE, 256, 128, 3, a["off"],
                                 a["out"], FAKE, None) == INVALID
    assert b"aligned" in lib.tgvkv_last_error()
    if name != "off":
        assert lib.tgvkv_cache_write_rows(d, pools(), a["table"], a["lens"], FAKE, FAKE, 3, FAKE, a["out"], FAKE,
                                          None) == INVALID
        assert b"aligned" in lib.tgvkv_last_error()


@pytest.mark.parametrize("name", ["table", "first"])
def test_misaligned_integers_of_a_read(lib, name):
    a = dict(table=FAKE, first=FAKE)
    a[name] = OFF_BY_TWO
    assert lib.tgvkv_cache_read(ctypes.byref(desc()), pools(), a["table"], a["first"], FAKE, FAKE, FAKE, 3, FAKE,
                                None) == INVALID
    assert b"aligned" in lib.tgvkv_last_error()


@pytest.mark.parametrize("name", ["table", "lens", "off"])
def test_misaligned_integers_of_the_attention(lib, name):
    a = dict(table=FAKE, lens=FAKE, off=FAKE)
    a[name] = OFF_BY_TWO
    # (max_q = 0: a call that got past its checks would launch nothing)
    assert lib.tgvkv_chunk_attention(ctypes.byref(desc()), pools(), a["table"], a["lens"], FAKE, 1024, 128, 3,
                                     a["off"], 0, FAKE, FAKE, None) == INVALID
    assert b"aligned" in lib.tgvkv_last_error()
