"""Refusals of mkv_chunk_attention that need no device: nothing is launched."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paper_2608_23834_b200 as M
from conftest import ROOT


@pytest.mark.parametrize("name", ["chunk_attention.cu", "tensor_ptx.cuh"])
def test_no_read_only_loads_in_kernels_that_start_early(name):
    """The plan, scan and merge kernels start while their predecessors still write (as in test_early_launch_loads)."""
    with open(os.path.join(ROOT, "paper_2608_23834_b200", "csrc", name)) as f:
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", f.read(), flags=re.S)
    assert not re.findall(r"__ldg\b|ld\.global\.nc|\bconst\s+\w+\s*\*\s*__restrict__", code)


def test_workspace_grows_with_the_table_and_bad_sizes_are_refused():
    cfg = M.make_config(256, 4, 24, 10, 10, np.ones(256, np.int8))
    size = C.c_size_t()
    call = lambda B, pages: M.lib().mkv_chunk_workspace_bytes(C.byref(cfg), B, pages, C.byref(size))
    assert call(2, 100) == M.OK
    small = size.value
    assert call(64, 65536) == M.OK and size.value - small >= 8 * (64 * 65536 - 200) and size.value % 256 == 0
    for B, pages in ((0, 10), (-1, 10), (1, 0), (1, -3)):
        assert call(B, pages) == M.E_INVALID
    assert M.lib().mkv_chunk_workspace_bytes(C.byref(cfg), 1, 1, None) == M.E_INVALID
    cfg.head_dim = 96
    assert call(1, 1) == M.E_INVALID


def test_a_bookkeeping_pool_takes_no_chunk():
    hp = M.HostPool(128, 2, 8, 4, 4)
    f = M.lib().mkv_chunk_attention
    assert f(hp.handle, None, 1024, 4, None, None, None, None, 1, 1, 1.0, None, None, None, 0, None) == M.E_INVALID
    assert f(None, None, 1024, 4, None, None, None, None, 1, 1, 1.0, None, None, None, 0, None) == M.E_INVALID
    hp.close()
