"""Sizes of selective state-space layers next to what a launch can take.  No GPU needed."""
import ctypes

import pytest

import paper_2606_27748_amd as F


@pytest.mark.parametrize("chunks,status", [(504, F.FLEX_OK), (505, F.FLEX_ERR_INVALID_ARG), (511, F.FLEX_ERR_INVALID_ARG),
                                           (512, F.FLEX_ERR_INVALID_ARG)])
def test_gradients_of_as_many_groups_as_heads(chunks, status):
    """512 threads for each chunk and group, and chunks by eights: 2^14 groups of 512 chunks are 2^32 threads."""
    d, n = F.make_scan_desc(1, 1 << 14, 1 << 14, 64, 64, 64 * (chunks - 1)), ctypes.c_size_t()
    assert F.load().flex_scan_workspace_size(ctypes.byref(d), F.FLEX_PASS_BWD, ctypes.byref(n)) == status


@pytest.mark.parametrize("chunks,status", [(511, F.FLEX_OK), (512, F.FLEX_ERR_INVALID_ARG)])
def test_gradients_of_one_group(chunks, status):
    """Fewer workgroups than heads: the sweeps' threads are the limit, as before."""
    d, n = F.make_scan_desc(1, 1, 1 << 14, 64, 64, 64 * (chunks - 1)), ctypes.c_size_t()
    assert F.load().flex_scan_workspace_size(ctypes.byref(d), F.FLEX_PASS_BWD, ctypes.byref(n)) == status
