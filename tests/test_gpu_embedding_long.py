"""The table's gradient of long lists: every number of ids per thread and step, parts of one step and of several, one to four passes of the sort."""
import numpy as np
import pytest
import torch

import paper_2405_16883_amd as sp
from test_gpu_embedding import zipf

pytestmark = pytest.mark.gpu

# Up to 131 072 ids a thread of the 128 workgroups has one, then 2, 4 and 8; from 1 048 577 on a workgroup has several steps.
TOKENS = [131072, 131073, 262145, 300000, 524289, 600000, 1048576, 1048577, 1100000, 3000001]


@pytest.mark.parametrize("tokens", TOKENS)
@pytest.mark.parametrize("vocab", [700, 50257, 2 ** 20 + 3, 2 ** 30 + 1])  # one, two, three and four passes
@pytest.mark.parametrize("law", ["uniform", "zipf"])
def test_long_lists(tokens, vocab, law):
    """Whole numbers, at most 4 x 3 000 001 in a sum: exact in any order."""
    rng = np.random.default_rng(tokens + vocab)
    ids = zipf(tokens, vocab, rng, 0.1) if law == "zipf" else torch.from_numpy(rng.integers(-2, vocab + 2, tokens).astype(np.int32)).cuda()
    d = 1 if vocab > 2 ** 29 else 1 + tokens % 8
    dout = torch.randint(-4, 5, (tokens, d), device="cuda").to(torch.bfloat16)
    order = torch.argsort(ids)
    seen, counts = torch.unique_consecutive(ids[order], return_counts=True)
    sums = dout[order].double().cumsum(0)[counts.cumsum(0) - 1]
    want = torch.cat([sums[:1], sums[1:] - sums[:-1]])
    inside = (seen >= 0) & (seen < vocab)
    seen, want = seen[inside].long(), want[inside]
    dE = torch.zeros((vocab, d), device="cuda")
    for accumulate in (True, False) if vocab < 2 ** 29 else (True,):
        if not accumulate:
            dE.fill_(float("nan"))
        sp.scorch_embedding_gradient(ids, dout, dE, accumulate=accumulate)
        assert torch.equal(dE[seen].double(), want)
        dE[seen] = 0
        assert dE.count_nonzero() == 0


@pytest.mark.parametrize("tokens", [200000, 600000, 2000003])
def test_rows_of_one_id_are_added_in_the_order_of_their_positions(tokens):
    """Runs of one to seven rows, each the work of one wavefront: the bits of a sum one by one."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    vocab = tokens // 4
    order = torch.randperm(tokens, device="cuda", generator=g)
    ids = torch.empty(tokens, dtype=torch.int32, device="cuda")
    run = torch.arange(tokens, device="cuda") // 7 * 2 + (torch.arange(tokens, device="cuda") % 7 >= 3).long()  # of 3 and 4
    ids[order] = (run % vocab).to(torch.int32)
    dout = torch.randn((tokens, 2), device="cuda", generator=g)
    dE = torch.empty((vocab, 2), device="cuda")
    sp.scorch_embedding_gradient(ids, dout, dE)
    by_id = torch.sort(ids.long(), stable=True)
    first = torch.searchsorted(by_id.values, torch.arange(vocab + 1, device="cuda"))
    want = torch.zeros((vocab, 2), device="cuda")
    longest = int((first[1:] - first[:-1]).max())
    assert longest <= 8
    for k in range(longest):
        at = first[:-1] + k
        more = at < first[1:]
        want[more] += dout[by_id.indices[at[more]]]
    assert torch.equal(dE, want)
