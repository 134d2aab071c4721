"""Refusals of the attention call beside those of test_kv_cpu.py (no device needed)."""
import ctypes as C

import pytest

from tests.test_kv_cpu import B, _cache, _tree  # noqa: F401


@pytest.mark.parametrize("stride", [0, 1, 31, -31])
def test_rows_of_lse_that_share_their_places_are_refused(B, stride):  # noqa: F811
    lib, c = B.load(), C.byref(_cache(B))
    assert lib.conqur_tree_attention(c, _tree(B, lse_t=stride), None) == -1
    # without lse, or with one row, the stride does not matter: the call gets as far as its workspace
    assert lib.conqur_tree_attention(c, _tree(B, lse=0, lse_t=stride, wsb=1), None) == -2
    assert lib.conqur_tree_attention(c, _tree(B, rows=1, lse_t=stride, wsb=1), None) == -2


def test_wider_rows_of_lse_are_taken(B):  # noqa: F811
    for stride in (32, 33, -32):
        assert B.load().conqur_tree_attention(C.byref(_cache(B)), _tree(B, lse_t=stride, wsb=1), None) == -2
