"""What the vocabulary operators refuse in Python, with real tensors: the outputs keep what they held."""
import pytest
import torch

import paper_2405_16883_amd as sp

pytestmark = pytest.mark.gpu


def args():
    i = dict(dtype=torch.int32, device="cuda")
    return {"ids": torch.zeros(4, **i), "E": torch.ones(5, 8, device="cuda"), "X": torch.full((4, 8), 7.0, device="cuda"),
            "Z": torch.ones(4, 5, device="cuda"), "dZ": torch.full((4, 5), 7.0, device="cuda"), "rowptr": torch.tensor([0, 1, 1, 2, 2], **i),
            "colidx": torch.zeros(2, **i), "vals": torch.ones(2, device="cuda"), "loss": torch.full((4,), 7.0, device="cuda"),
            "stats": torch.full((4, 2), 7.0, device="cuda"), "row": torch.ones(4, device="cuda"), "mask": torch.full((4, 1), -1, **i)}


CALLS = {
    "lookup": (lambda a: sp.scorch_embedding_lookup(a["ids"], a["E"], a["X"]), ("ids", "E", "X")),
    "gradient": (lambda a: sp.scorch_embedding_gradient(a["ids"], a["X"], a["E"]), ("ids", "X", "E")),
    "loss": (lambda a: sp.scorch_distill_loss(a["Z"], a["rowptr"], a["colidx"], a["vals"], 1.0, a["loss"], a["stats"]),
             ("Z", "rowptr", "colidx", "vals", "loss", "stats")),
    "distill gradient": (lambda a: sp.scorch_distill_gradient(a["Z"], a["rowptr"], a["colidx"], a["vals"], 1.0, a["stats"], a["row"], a["dZ"]),
                         ("Z", "rowptr", "colidx", "vals", "stats", "row", "dZ")),
    "both": (lambda a: sp.scorch_distill_loss_gradient(a["Z"], a["rowptr"], a["colidx"], a["vals"], 1.0, a["row"], a["loss"], a["dZ"]),
             ("Z", "rowptr", "colidx", "vals", "row", "loss", "dZ")),
    "logits": (lambda a: sp.scorch_logits_process(a["Z"], a["dZ"], a["rowptr"], a["colidx"], repetition=a["row"], bias_rowptr=a["rowptr"],
                                                  bias_tokens=a["colidx"], bias_vals=a["vals"], mask=a["mask"]),
               ("Z", "dZ", "rowptr", "colidx", "row", "vals", "mask")),
}
SWAPS = {
    "another type": lambda t: t.to(torch.float64 if t.is_floating_point() else torch.int64),
    "on the CPU": lambda t: t.cpu(),
    "every other element": lambda t: torch.stack([t, t], -1)[..., 0],
    "one too many": lambda t: torch.cat([t, t[:1]]),
    "no tensor": lambda t: [1.0],
}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("swap", sorted(SWAPS))
def test_an_argument_that_does_not_fit_is_refused(name, swap):
    call, names = CALLS[name]
    call(args())
    for which in names:
        if swap == "one too many" and (name, which) in (("lookup", "E"), ("gradient", "E"), ("logits", "Z")):
            continue  # a table of six rows is as good; the others are then too few
        a = args()
        keep = {k: v.clone() for k, v in a.items()}
        a[which] = SWAPS[swap](a[which])
        if swap == "one too many" and which in ("colidx", "vals") and name != "logits":
            a["vals" if which == "colidx" else "colidx"] = keep["vals" if which == "colidx" else "colidx"]  # of different lengths
        with pytest.raises((ValueError, TypeError, sp.ScorchError)):
            call(a)
        torch.cuda.synchronize()
        for k in keep:
            if k != which:
                assert torch.equal(a[k], keep[k]), k


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs a second GPU")
def test_tensors_of_another_device_are_refused():
    for name, (call, names) in CALLS.items():
        for which in names:
            a = args()
            a[which] = a[which].to("cuda:1")
            with pytest.raises(ValueError, match="current device"):
                call(a)


def test_negated_views_are_refused():
    for name, which in (("lookup", "E"), ("gradient", "X"), ("loss", "Z"), ("both", "vals"), ("logits", "row")):
        b = args()
        b[which] = torch._neg_view(b[which])
        with pytest.raises(ValueError, match="negated"):
            CALLS[name][0](b)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_every_call_runs_on_the_stream_that_it_is_given(name, monkeypatch):
    """Waiting for that stream alone is enough to see the results."""
    call, names = CALLS[name]
    want = args()
    call(want)
    got = args()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    import functools
    for f in ("scorch_embedding_lookup", "scorch_embedding_gradient", "scorch_distill_loss", "scorch_distill_gradient", "scorch_distill_loss_gradient",
              "scorch_logits_process"):
        monkeypatch.setattr(sp, f, functools.partial(getattr(sp, f), stream=side))
    call(got)
    side.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k
