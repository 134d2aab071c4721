"""Refusals of the attention call that loses a wait (no device needed)."""
import ctypes as C

import pytest

from tests.test_kv_cpu import B, P, _cache, _tree  # noqa: F401


@pytest.mark.parametrize("block,site,index", [(-1, 1, 0), (0, 0, 0), (0, 6, 0), (0, 1, -1), (0, 1, 4), (0, 2, 4), (0, 3, 2), (0, 5, 2)])
def test_what_is_not_a_wait_is_refused(B, block, site, index):  # noqa: F811
    assert B.load().conqur_debug_tree_attention(C.byref(_cache(B)), _tree(B, group=8, nodes=8, lse_t=64), block, site, index, None) == -1


def test_few_rows_have_no_such_waits(B):  # noqa: F811
    lib = B.load()
    assert lib.conqur_debug_tree_attention(C.byref(_cache(B)), _tree(B, group=4, nodes=4), 0, 1, 0, None) == -10
    assert lib.conqur_debug_tree_attention(C.byref(_cache(B)), _tree(B, group=8, nodes=8, lse_t=64, ws=0), 0, 1, 0, None) == -1
    assert lib.conqur_debug_tree_attention(C.byref(_cache(B)), _tree(B, group=8, nodes=8, lse_t=64, wsb=1), 0, 1, 0, None) == -2
