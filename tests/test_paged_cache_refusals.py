"""Refusals of the paged-cache calls that concern the layout of their integer arrays
(no GPU: nothing is launched)."""
import ctypes

import pytest
import torch

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


class Calls(Exception):
    """Raised in the library's place: the binding's own checks are through."""


@pytest.mark.parametrize("call", ["write", "write_rows", "read", "attend"])
def test_a_page_table_of_another_width(lib, call, monkeypatch):
    """A table with more columns than max_pages holds enough entries, but its rows would
    be taken from the wrong places."""
    from paper_2606_03075_gb300 import api
    cd = api.make_cache_desc(2, 8, 2, 64, 16, 64, 8, "int8")
    real = api._dev
    # CPU tensors in the place of the GPU's: only their shapes are looked at
    monkeypatch.setattr(api, "_dev", lambda t, dtype, numel, name: real(t, dtype, numel, name) if t is None else 1)
    monkeypatch.setattr(api, "_ptr", lambda t, dtypes, numel, name: 1)
    monkeypatch.setattr(api, "_tokens", lambda t, heads, d, name: (1, 1, 1, 3))

    def stop(stream):
        raise Calls

    monkeypatch.setattr(api, "_stream", stop)
    cache = api.alloc_cache(cd, device="cpu")
    x, i = torch.zeros(3, 64), torch.zeros(5, dtype=torch.int32)

    def run(table):
        if call == "write":
            api.tgvkv_cache_write(cd, cache, table, i, x, x, i, i, i)
        elif call == "write_rows":
            api.tgvkv_cache_write_rows(cd, cache, table, i, x, x, i, i, i)
        elif call == "read":
            api.tgvkv_cache_read(cd, cache, table, None, i, x, x, i)
        else:
            api.tgvkv_chunk_attention(cd, cache, table, i, x, i, 1, x, i)

    for shape in ((4, 8), (2, 2, 8), (32,)):
        with pytest.raises(Calls):
            run(torch.zeros(shape, dtype=torch.int32))
    for shape in ((4, 9), (4, 16), (8, 4), (2, 2, 10)):
        with pytest.raises(ValueError, match="max_pages = 8"):
            run(torch.zeros(shape, dtype=torch.int32))
