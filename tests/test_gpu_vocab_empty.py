"""Vocabulary calls without columns, rows, tokens or entries: nothing outside the outputs is touched, and what the definitions give is written."""
import pytest
import torch

import paper_2405_16883_amd as sp
from vocab_util import TYPES

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(0, 0), (0, 7), (3, 0), (2050, 0), (300, 0)])
def test_distillation(rows, vocab, kind):
    Z = torch.empty((rows, vocab), dtype=TYPES[kind], device="cuda")
    rowptr = torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    colidx, vals = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.ones(rows, device="cuda")  # column 0 is outside
    loss, both, stats, dZ = (torch.full(s, 7.0, device="cuda") for s in ((rows,), (rows,), (rows, 2), (rows, vocab)))
    sp.scorch_distill_loss(Z, rowptr, colidx, vals, 1.0, loss, stats)
    sp.scorch_distill_gradient(Z, rowptr, colidx, vals, 1.0, stats, None, dZ.to(Z.dtype))
    sp.scorch_distill_loss_gradient(Z, rowptr, colidx, vals, 1.0, None, both, dZ.to(Z.dtype))
    assert (loss == 0).all() and (both == 0).all()
    assert (stats[:, 0] == -float("inf")).all() and (stats[:, 1] == 0).all()


@pytest.mark.parametrize("rows,vocab", [(0, 0), (0, 7), (3, 0), (3, 7)])
def test_logits_with_empty_lists(rows, vocab):
    x = torch.randn((rows, vocab), device="cuda")
    out = torch.full_like(x, 7.0)
    rowptr, none = torch.zeros(rows + 1, dtype=torch.int32, device="cuda"), ints()
    one = torch.ones(rows, device="cuda")
    mask = torch.full((rows, (vocab + 31) // 32), -1, dtype=torch.int32, device="cuda")
    sp.scorch_logits_process(x, out, rowptr, none, repetition=2 * one, presence=one, frequency=one, bias_rowptr=rowptr, bias_tokens=none,
                             bias_vals=torch.empty(0, device="cuda"), mask=mask)
    assert torch.equal(out, x)


@pytest.mark.parametrize("vocab,d", [(0, 0), (0, 8), (5, 0), (5, 8)])
@pytest.mark.parametrize("tokens", [0, 3, 300])
def test_lookup_and_gradient(tokens, vocab, d):
    ids = torch.full((tokens,), 2, dtype=torch.int32, device="cuda")
    E, X = torch.ones((vocab, d), device="cuda"), torch.full((tokens, d), 7.0, device="cuda")
    sp.scorch_embedding_lookup(ids, E, X, 3.0)
    assert (X == (3 if vocab else 0)).all()
    dE = torch.full((vocab, d), 7.0, device="cuda")
    sp.scorch_embedding_gradient(ids, X, dE)
    want = torch.zeros_like(dE)
    want[2:3] = 3 * tokens
    assert torch.equal(dE, want)
    sp.scorch_embedding_gradient(ids, X, dE, accumulate=True)
    assert torch.equal(dE, 2 * want)
