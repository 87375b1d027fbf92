"""Sizes that pass 32 bits are refused by the calls that go through ctypes too, which takes integers modulo 2^32.  No GPU is needed."""
import os

import pytest
import torch

import paper_2405_16883_amd as sp


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1])
@pytest.mark.parametrize("place", [0, 1, 2])
def test_sizes_beyond_32_bits(big, place):
    if not os.path.exists(sp.LIB_PATH):
        pytest.skip("library not built")
    sizes = [5, 5, 5]
    sizes[place] = big
    for call in (lambda: sp.scorch_embedding_gradient_workspace_bytes(*sizes), lambda: sp.scorch_spmm_plan_workspace_bytes(*sizes, 5),
                 lambda: sp.scorch_spmm_plan(*sizes, torch.zeros(6, dtype=torch.int32), 5, workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_sizes_of_32_bits_are_taken():
    if not os.path.exists(sp.LIB_PATH):
        pytest.skip("library not built")
    assert sp.scorch_embedding_gradient_workspace_bytes(2 ** 31 - 1, 2 ** 31 - 1, 4) > 2 ** 35
