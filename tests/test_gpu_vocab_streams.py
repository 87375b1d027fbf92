"""Every vocabulary call runs on the stream that it is given: it sees inputs that are produced there, late, while the current stream has nothing to wait for."""
import pytest
import torch

import paper_2405_16883_amd as sp

pytestmark = pytest.mark.gpu


def operands(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def ints(n, hi):
        return torch.randint(0, hi, (n,), dtype=torch.int32, device="cuda", generator=g)

    def floats(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    rowptr = torch.arange(0, 301, dtype=torch.int32, device="cuda") * (seed + 2)
    return {"ids": ints(300, 40), "E": floats(40, 24), "X": floats(300, 24), "Z": floats(300, 40), "dZ": floats(300, 40), "rowptr": rowptr,
            "colidx": ints(1500, 40), "vals": floats(1500), "loss": floats(300), "stats": floats(300, 2).exp(), "row": floats(300).exp(),
            "mask": ints(600, 2 ** 31 - 1).view(300, 2)}


CALLS = {
    "lookup": lambda a, s: sp.scorch_embedding_lookup(a["ids"], a["E"], a["X"], stream=s),
    "gradient": lambda a, s: sp.scorch_embedding_gradient(a["ids"], a["X"], a["E"], stream=s),
    "gradient added": lambda a, s: sp.scorch_embedding_gradient(a["ids"], a["X"], a["E"], 2.0, accumulate=True, stream=s),
    "loss": lambda a, s: sp.scorch_distill_loss(a["Z"], a["rowptr"], a["colidx"], a["vals"], 0.5, a["loss"], a["stats"], stream=s),
    "distill gradient": lambda a, s: sp.scorch_distill_gradient(a["Z"], a["rowptr"], a["colidx"], a["vals"], 0.5, a["stats"], a["row"], a["dZ"], stream=s),
    "both": lambda a, s: sp.scorch_distill_loss_gradient(a["Z"], a["rowptr"], a["colidx"], a["vals"], 0.5, a["row"], a["loss"], a["dZ"], stream=s),
    "logits": lambda a, s: sp.scorch_logits_process(a["Z"], a["dZ"], a["rowptr"], a["colidx"], repetition=a["row"], bias_rowptr=a["rowptr"],
                                                    bias_tokens=a["colidx"], bias_vals=a["vals"], mask=a["mask"], stream=s),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_inputs_that_the_stream_produces_late_are_seen(name):
    """With several streams: some may share a queue of the hardware with the current one and would be in order all the same."""
    call = CALLS[name]
    late, want, stale = operands(1), operands(1), operands(2)
    call(want, None)  # the right results
    call(stale, None)  # what a call that does not wait for the inputs comes to
    assert any(not torch.equal(stale[k], want[k]) for k in want)
    big = torch.ones((8192, 8192), device="cuda")
    product = torch.mm(big, big)  # the library is loaded
    for side in [torch.cuda.Stream() for _ in range(4)]:
        got, ready = operands(2), torch.cuda.Event()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(4):
                torch.mm(big, big, out=product)  # some 40 ms
            for k in late:
                got[k].copy_(late[k])
            ready.record()
        call(got, side)
        assert not ready.query(), "the inputs were there before the call, which shows nothing"
        side.synchronize()
        for k in want:
            assert torch.equal(got[k], want[k]), k
