"""Limits of a token's step on the host (the pointers are fake, never dereferenced; every call here is refused before any
HIP call or is a workspace query)."""

import ctypes

import pytest

from test_step_abi import FAKE, UNSUPPORTED, _attend, _cache, lib  # noqa: F401

CHUNK = 4096                     # the most positions of a workgroup


@pytest.mark.parametrize("page,width", [(16, 2 ** 27 - 1), (64, 2 ** 25 - 1), (2048, 2 ** 20 - 1)])
@pytest.mark.parametrize("type_", [0, 1])
def test_attention_keeps_positions_and_a_range_below_2_31(lib, page, width, type_):  # noqa: F811
    """A workgroup's positions run up to a range past the last visible one, in 32 bits: with max_len within a range of 2^31
    the count of ranges came out negative and the output was not written."""
    big = _cache(page_size=page, table_width=width, type=type_, k_scale=FAKE, v_scale=FAKE)
    most = 2 ** 31 - CHUNK
    for n in (most + 1, page * width):
        assert n <= page * width
        assert _attend(lib, big, max_len=n) == UNSUPPORTED
        assert b"max_len" in lib.qwam_last_error()
        assert lib.qwam_paged_attention_workspace(ctypes.byref(big), 4, n) == -1
    assert lib.qwam_paged_attention_workspace(ctypes.byref(big), 4, most) > 0
