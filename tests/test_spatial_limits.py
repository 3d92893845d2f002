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
