"""The table's gradient on a stream that is given refuses the same things with the same errors as on the current one.  No GPU is needed."""
import os

import pytest
import torch

import paper_2405_16883_amd as sp


class Stream:
    cuda_stream = 0


@pytest.mark.parametrize("which", ["dout", "dE"])
@pytest.mark.parametrize("wrong,error", [([1.0], TypeError), (None, TypeError), (torch.zeros(2), ValueError), (torch.zeros(()), ValueError)])
@pytest.mark.parametrize("stream", [None, Stream()])
def test_what_is_no_matrix_is_refused(which, wrong, error, stream):
    if not os.path.exists(sp.LIB_PATH):
        pytest.skip("library not built")
    good = torch.zeros(2, 2)
    if which == "dE" and error is TypeError:
        error = (TypeError, ValueError)  # the first of the two operands is on the CPU, which is found first
    a = {"dout": good, "dE": good, which: wrong}
    with pytest.raises(error):
        sp.scorch_embedding_gradient(torch.zeros(2, dtype=torch.int32), a["dout"], a["dE"], stream=stream)
