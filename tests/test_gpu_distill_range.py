"""Distillation over the whole range of logits and temperatures: where differences of logits pass the largest number of 32 bits, the results
that are numbers are right."""
import numpy as np
import pytest
import torch

from test_gpu_distill import check, problem, run
from vocab_util import TYPES, assert_within, distill_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [2, 33, 5000, 140001])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("inv_t", [0.25, 1e-3, 1e-37, 2e-38])
def test_differences_of_logits_beyond_the_largest_number(kind, vocab, inv_t):
    """Logits from -3e38 to 3e38: the largest scaled differences are 1.5e38, 6e35, 60 and 12."""
    rng = np.random.default_rng(vocab)
    Z = torch.from_numpy(rng.uniform(-3e38, 3e38, (4, vocab)).astype(np.float32)).to(TYPES[kind])
    Z[:, 0], Z[:, 1] = 3e38, -3e38
    lists = [([1], [0.0]), ([0, 1], [3e38, -3e38]), ([1, 0], [2e38, -1e38]), ([0], [5.0])]
    check(Z, lists, inv_t=inv_t, dloss=[0.5 / inv_t] * 4)


@pytest.mark.parametrize("vocab", [2, 5000, 140001])
@pytest.mark.parametrize("inv_t", [1.0, 8.0])
def test_a_share_of_a_loss_beyond_the_largest_number(vocab, inv_t):
    """A teacher's probability of e^-60 on a logit that is 6e38 below the largest: 60 + 6e38 inv_t times it is a number."""
    Z = torch.zeros((2, vocab))
    Z[:, 0], Z[:, 1] = 3e38, -3e38
    lists = [([0, 1], [60.0 / inv_t, 0.0]), ([1, 0], [-60.0 / inv_t, 0.0])]
    check(Z, lists, inv_t=inv_t)


@pytest.mark.parametrize("scale,inv_t", [(1e30, 1.0), (1e4, 100.0), (1.0, 1e-6), (1e-37, 2e38), (1e37, 1e-37)])
def test_large_and_small_logits_and_temperatures(scale, inv_t):
    Z, lists = problem(3, 5000, 10, 6, spread=1.0)
    lists = [(c, (t * np.float32(scale)).astype(np.float32)) for c, t in lists]
    Z = Z * scale
    loss, stats, apart, both, dZ = run(Z, lists, inv_t)
    ref, tol = distill_ref(Z, lists, inv_t)[:2]
    assert_within(loss, ref, tol, "loss")
    assert_within(both, ref, tol, "loss with gradient")
    assert dZ.isfinite().all() and apart.isfinite().all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab,k", [(9, 12), (3001, 1500)])
@pytest.mark.parametrize("in_place", [False, True])
def test_temperatures_so_high_that_all_columns_are_alike(kind, vocab, k, in_place):
    """Entries that repeat, more of them than threads, rows without entries and rows that are not numbers."""
    Z, lists = problem(6, vocab, k, vocab, repeats=True)
    lists[1] = ([], [])
    Z[2], Z[4, vocab - 1] = -float("inf"), float("nan")
    lists[2] = lists[4] = ([1], [0.0])
    Z, weights = Z.to(TYPES[kind]), [1e37 * (i + 1) for i in range(6)]
    loss, stats, apart, both, dZ = run(Z, lists, 2e-37, weights, in_place=in_place)
    for x in (loss, both, apart, dZ):
        assert x[[2, 4]].isnan().all() and (x[1] == 0).all()
    rest = [0, 1, 3, 5]
    check(Z[rest], [lists[i] for i in rest], 2e-37, [weights[i] for i in rest], pad=3, in_place=in_place)
