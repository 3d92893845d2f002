"""Sizes past what the kernels count in are refused on the host; none of these calls reaches a device."""
import ctypes

import pytest

from .test_spatial_host import FAKE, att, lib  # noqa: F401

MOST = 1 << 30


@pytest.mark.parametrize("over", [dict(rows_q=MOST + 1), dict(rows_k=MOST + 1), dict(sequences=MOST + 1), dict(rows_k=2 ** 31 - 1), dict(heads=4098)], ids=str)
def test_rows_past_the_kernels_counts(lib, over):  # noqa: F811
    a = ctypes.byref(att(head_dim=8, **{"heads": 2, "kv_heads": 2, **over}))
    assert lib.dchag_attend(1, a, *[FAKE] * 6, 1 << 60, None) == -2
    assert lib.dchag_attend_backward(1, a, *[FAKE] * 9, None, FAKE, 1 << 60, None) == -2
    assert lib.dchag_attend_workspace_bytes(1, a, 0) == 0 == lib.dchag_attend_workspace_bytes(1, a, 1)


def test_most_rows_are_taken(lib):  # noqa: F811
    """Up to the limit there is a workspace for the call."""
    a = ctypes.byref(att(heads=1, kv_heads=1, head_dim=8, rows_q=MOST, rows_k=MOST, sequences=3))
    assert lib.dchag_attend_workspace_bytes(1, a, 0) > 0 and lib.dchag_attend_workspace_bytes(1, a, 1) > 0


@pytest.mark.parametrize("over", [
    dict(sequences=1 << 21, rows_q=1 << 21, rows_k=1 << 21, heads=16, kv_heads=16),     # single tokens: a workgroup a sequence and key head
    dict(sequences=1 << 20, rows_q=1 << 25, rows_k=1 << 25, heads=32, kv_heads=32),
], ids=["few", "tiles"])
def test_more_threads_than_a_launch_can_have(lib, over):  # noqa: F811
    a = ctypes.byref(att(head_dim=8, **over))
    assert lib.dchag_attend(1, a, *[FAKE] * 6, 1 << 60, None) == -2
    assert lib.dchag_attend_backward(1, a, *[FAKE] * 9, None, FAKE, 1 << 60, None) == -2


def test_more_blocks_than_a_launch_can_take(lib):  # noqa: F811
    for rows, D in ((1 << 25, 1024), ((1 << 30) - 255, 32), ((1 << 30) - 255, 8)):
        assert lib.dchag_unpack8(1, rows, D, 0, FAKE, FAKE, FAKE, None) == -2
    for rows, D in ((1 << 27, 1024), ((1 << 32) - 1023, 32)):
        assert lib.dchag_pack8(0, rows, D, 0, FAKE, FAKE, FAKE, None) == -2
