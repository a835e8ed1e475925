"""Checks of the sequence operators' arguments that need no GPU, in Python and in the library."""
import ctypes as C

import pytest
import torch

from test_memory_boundary import CONFIG, GOOD, M, dims, view  # noqa: F401  (M: the fixture)


def test_workspace_in_host_memory(M):  # noqa: F811
    """The one pointer of a call that a kernel writes without any other tensor's shape: it has to lie on the GPU too, needed or not."""
    for need in (0, 64):
        with pytest.raises(M.MarlError, match="on the GPU"):
            M.binding._workspace(torch.empty(256, dtype=torch.uint8), need)
    assert M.binding._workspace(None, 0) is None
