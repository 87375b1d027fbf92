"""Grammar masks whose rows are further apart than 32 bits reach."""
import pytest
import torch

import paper_2405_16883_amd as sp
from vocab_util import pack_mask

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("stride", [2 ** 31 + 7, 2 ** 32 + 5])
def test_masks_with_rows_far_apart(stride):
    """A stride taken modulo 2^32 would read words of the first row's neighbourhood, which allow the opposite."""
    rows, vocab, words = 2, 100, 4
    g = torch.Generator().manual_seed(stride % 1000)
    allowed = (torch.rand((rows, vocab), generator=g) < 0.5).numpy()
    buf = torch.empty(stride + words, dtype=torch.int32, device="cuda")
    buf[:64] = ~pack_mask(allowed)[1].repeat(16)
    mask = buf.as_strided((rows, words), (stride, 1))
    mask.copy_(pack_mask(allowed))
    x = torch.randn((rows, vocab), device="cuda")
    out = torch.empty_like(x)
    sp.scorch_logits_process(x, out, mask=mask)
    assert torch.equal(out, torch.where(torch.from_numpy(allowed).cuda(), x, -float("inf")))
