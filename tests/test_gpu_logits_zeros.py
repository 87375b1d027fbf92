"""Columns that no list names keep their bits, negative zeros too."""
import pytest
import torch

import paper_2405_16883_amd as sp
from vocab_util import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lists", ["history", "bias", "both"])
def test_columns_that_no_list_names_keep_their_bits(kind, lists):
    vocab = 1000
    x = torch.full((1, vocab), -0.0, dtype=TYPES[kind], device="cuda")
    x[:, 500:] = torch.randn(500, device="cuda").to(TYPES[kind])
    tokens = torch.arange(3, vocab, 5, dtype=torch.int32, device="cuda")
    rowptr = torch.tensor([0, tokens.numel()], dtype=torch.int32, device="cuda")
    one = torch.ones(1, device="cuda")
    a = {}
    if lists != "bias":
        a.update(history_rowptr=rowptr, history=tokens, repetition=2 * one, presence=one, frequency=one)
    if lists != "history":
        a.update(bias_rowptr=rowptr, bias_tokens=tokens, bias_vals=torch.ones(tokens.numel(), device="cuda"))
    out = torch.empty_like(x)
    sp.scorch_logits_process(x, out, **a)
    rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
    rest[tokens.long()] = False
    bits = torch.int32 if kind == "f32" else torch.int16
    assert torch.equal(out.view(bits)[:, rest], x.view(bits)[:, rest])
    assert (out[:, ~rest] != x[:, ~rest]).any()
