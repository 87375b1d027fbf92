"""What the vocabulary operators refuse, before anything reaches a GPU: no GPU is needed."""
import ctypes
import math
import os

import pytest
import torch

import paper_2405_16883_amd as sp
from test_binding_errors import run

BAD, UNSUPPORTED, SMALL = sp.binding.SCORCH_ERR_INVALID_ARG, sp.binding.SCORCH_ERR_UNSUPPORTED, sp.binding.SCORCH_ERR_WORKSPACE_TOO_SMALL
F32, BF16 = 0, 1
P = 4096  # stands for a pointer: nothing is read from it


@pytest.fixture()
def lib():
    if not os.path.exists(sp.LIB_PATH):
        pytest.skip("library not built")
    return sp.load_library()


def refused(lib, status, word, got):
    assert got == status, lib.scorch_last_error()
    if word:
        assert word in lib.scorch_last_error().decode()


def test_lookup(lib):
    def call(tokens=2, vocab=3, d=4, ids=P, E=P, e_type=F32, lde=4, scale=1.0, out=P, out_type=F32, ldo=4):
        return lib.scorch_embedding_lookup(tokens, vocab, d, ids, E, e_type, lde, scale, out, out_type, ldo, None)
    for change, word in (({"tokens": -1}, "negative"), ({"vocab": -1}, "negative"), ({"d": -1}, "negative"), ({"ids": None}, "ids"),
                         ({"E": None}, "E"), ({"out": None}, "out"), ({"lde": 3}, "stride"), ({"ldo": 3}, "stride"), ({"e_type": 3}, "type"),
                         ({"out_type": -1}, "type"), ({"E": P + 2}, "aligned"), ({"out": P + 1, "out_type": BF16}, "aligned")):
        refused(lib, BAD, word, call(**change))
    refused(lib, UNSUPPORTED, "d =", call(d=2 ** 23 + 1, lde=2 ** 24, ldo=2 ** 24))
    assert call(tokens=0, ids=None, out=None) == 0 and call(d=0, E=None) == 0


def test_gradient(lib):
    need = sp.scorch_embedding_gradient_workspace_bytes(2, 3, 4)

    def call(tokens=2, vocab=3, d=4, ids=P, dout=P, t=F32, lddo=4, add=0, dE=P, e=F32, ldde=4, ws=P, size=need):
        return lib.scorch_embedding_gradient(tokens, vocab, d, ids, dout, t, lddo, 1.0, add, dE, e, ldde, ws, size, None)
    for change, word in (({"tokens": -1}, "negative"), ({"vocab": -2}, "negative"), ({"d": -1}, "negative"), ({"ids": None}, "ids"),
                         ({"dout": None}, "dout"), ({"dE": None}, "dE"), ({"lddo": 3}, "stride"), ({"ldde": 0}, "stride"), ({"t": 7}, "type"),
                         ({"e": 3}, "type"), ({"ws": None}, "workspace"), ({"ws": P + 128}, "256"), ({"dE": P + 2}, "aligned")):
        refused(lib, BAD, word, call(**change))
    refused(lib, SMALL, str(need), call(size=need - 1))
    refused(lib, UNSUPPORTED, "d =", call(d=2 ** 23 + 1, lddo=2 ** 24, ldde=2 ** 24))
    assert call(vocab=0, dE=None) == 0 and call(d=0) == 0 and call(tokens=0, add=1, ids=None, dout=None) == 0


def test_gradient_workspace(lib):
    size = sp.scorch_embedding_gradient_workspace_bytes
    assert 0 < size(0, 0, 0) <= size(1, 10, 8) <= size(10_000, 10, 8) < size(10_000, 10, 4096)
    # order of the tokens and partial rows: less than dout and four integers a token
    for tokens, d in ((16384, 4096), (262144, 768), (10 ** 7, 64)):
        assert size(tokens, 1000, d) < tokens * d * 2 + tokens * 16 + 2 ** 21
    assert size(2 ** 31 - 1, 2 ** 31 - 1, 8) > 2 ** 35  # sizes beyond 32 bits
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, -1)):
        with pytest.raises(sp.ScorchError) as e:
            size(*bad)
        assert e.value.status == BAD
    refused(lib, BAD, "bytes_out", lib.scorch_embedding_gradient_workspace_bytes(1, 1, 1, None))


def test_distillation(lib):
    big = sp.DISTILL_VOCAB_MAX + 1
    base = dict(rows=2, vocab=3, Z=P, t=F32, ldz=3, rowptr=P, x=1.0, loss=P, stats=P, dZ=P + 64, lddz=3)

    def loss(**change):
        a = {**base, **change}
        return lib.scorch_distill_loss(a["rows"], a["vocab"], a["Z"], a["t"], a["ldz"], a["rowptr"], P, P, a["x"], a["loss"], a["stats"], None)

    def gradient(**change):
        a = {**base, **change}
        return lib.scorch_distill_gradient(a["rows"], a["vocab"], a["Z"], a["t"], a["ldz"], a["rowptr"], P, P, a["x"], a["stats"], None, a["dZ"], a["lddz"], None)

    def both(**change):
        a = {**base, **change}
        return lib.scorch_distill_loss_gradient(a["rows"], a["vocab"], a["Z"], a["t"], a["ldz"], a["rowptr"], P, P, a["x"], None, a["loss"], a["dZ"], a["lddz"], None)

    for call in (loss, gradient, both):
        for change, word in (({"rows": -1}, "negative"), ({"vocab": -1}, "negative"), ({"Z": None}, "Z"), ({"t": 5}, "type"), ({"ldz": 2}, "stride"),
                             ({"rowptr": None}, "rowptr"), ({"x": 0.0}, "temperature"), ({"x": -1.0}, "temperature"),
                             ({"x": math.nan}, "temperature"), ({"x": math.inf}, "temperature")):
            refused(lib, BAD, word, call(**change))
        assert call(rows=0, rowptr=None) == 0
        refused(lib, UNSUPPORTED, "launch", call(rows=2 ** 22, lddz=3))
    for call in (gradient, both):
        refused(lib, BAD, "dZ", call(dZ=None))
        refused(lib, BAD, "stride", call(lddz=2))
        refused(lib, BAD, "another row stride", call(dZ=P, lddz=4))
        refused(lib, UNSUPPORTED, str(sp.DISTILL_VOCAB_MAX), call(vocab=big, ldz=big, lddz=big))
    refused(lib, BAD, "stats", gradient(stats=None))
    refused(lib, BAD, "stats", loss(stats=None))
    refused(lib, BAD, "loss", loss(loss=None))
    refused(lib, BAD, "loss", both(loss=None))
    assert gradient(vocab=0, Z=None, dZ=None) == 0


def test_logits(lib):
    rules = sp.LogitsRules()

    def call(rows=2, vocab=40, x=P, t=F32, ldl=40, rules=rules, out=P + 64, o=F32, ldo=40):
        return lib.scorch_logits_process(rows, vocab, x, t, ldl, ctypes.byref(rules) if rules is not None else None, out, o, ldo, None)
    for change, word in (({"rows": -1}, "negative"), ({"vocab": -1}, "negative"), ({"x": None}, "logits"), ({"out": None}, "out"), ({"t": 3}, "type"),
                         ({"o": -1}, "type"), ({"ldl": 39}, "stride"), ({"ldo": 39}, "stride"), ({"rules": None}, "rules"),
                         ({"out": P, "ldo": 41}, "out is logits"), ({"out": P, "o": BF16}, "out is logits"), ({"x": P + 1}, "aligned")):
        refused(lib, BAD, word, call(**change))
    masked = sp.LogitsRules(mask=P, ldm=1)
    refused(lib, BAD, "mask", call(rules=masked))
    refused(lib, UNSUPPORTED, "launch", call(rows=2 ** 23, vocab=1))
    assert call(rows=0, x=None, out=None) == 0 and call(vocab=0) == 0


def test_binding_refuses_what_does_not_fit_together():
    if not os.path.exists(sp.LIB_PATH):
        pytest.skip("library not built")
    i, f, m = torch.zeros(2, dtype=torch.int32), torch.zeros(2), torch.zeros(2, 2)
    for call in (lambda: sp.scorch_embedding_lookup(i, m, m), lambda: sp.scorch_embedding_gradient(i, m, m),
                 lambda: sp.scorch_distill_loss(m, i, i, f, 1.0, f, m), lambda: sp.scorch_distill_gradient(m, i, i, f, 1.0, m, f, m),
                 lambda: sp.scorch_distill_loss_gradient(m, i, i, f, 1.0, f, f, m), lambda: sp.scorch_logits_process(m, m)):
        with pytest.raises(ValueError):  # not on a GPU
            call()


CALLS = {
    "embedding_lookup": ["native.embedding_lookup(i, {x}, d, 1.0, None)", "native.embedding_lookup({x}, d, d, 1.0, None)"],
    "embedding_gradient": ["native.embedding_gradient(i, {x}, d, 1.0, 0, b, None)", "native.embedding_gradient(i, d, {x}, 1.0, 0, b, None)"],
    "distill_loss": ["native.distill_loss({x}, i, i, f, 1.0, f, d, None)", "native.distill_loss(d, {x}, i, f, 1.0, f, d, None)"],
    "distill_gradient": ["native.distill_gradient(d, i, i, f, 1.0, d, f, {x}, None)", "native.distill_gradient({x}, i, i, f, 1.0, d, f, d, None)"],
    "distill_loss_gradient": ["native.distill_loss_gradient({x}, i, i, f, 1.0, f, f, d, None)",
                              "native.distill_loss_gradient(d, i, i, {x}, 1.0, f, f, d, None)"],
    "logits_process": ["native.logits_process({x}, d, None, None, None, None, None, None, None, None, None, None, None)",
                       "native.logits_process(d, d, i, {x}, None, None, None, None, None, None, None, None, None)"],
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_tensors_without_memory_wrong_things_and_counts_are_python_errors(name):
    body = """
with FakeTensorMode():
    i, f, b = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(9, dtype=torch.uint8, device="cuda")
    h = torch.zeros(2, 2, device="cuda", dtype=torch.float64)
def attempt(call):
    try:
        call()
        print("nothing")
    except Exception as e:
        print("raised")
"""
    want = 0
    for call in CALLS[name]:
        for x in ("sparse", "d", "h", "None", "3", "'text'"):
            body += f"attempt(lambda: {call.format(x=x)})\n"
            want += 1
    body += f"attempt(lambda: native.{name}())\n"
    assert run(body) == ["raised"] * (want + 1)
