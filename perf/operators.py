"""Performance cases of the operators at the two ends of a language model's vocabulary, where lists of token ids meet dense rows.

A case is a dict of plain values.  `op` names what runs, the rest are sizes and types ("f32", "bf16", "f16"):

    lookup         rows of a table by token id, scaled; ids outside the table (padding) give zeros
    gradient       gradient of the table: rows of the same token added up; it overwrites the table's gradient or is added to it
    distill_loss   Kullback-Leibler divergence of the student's logits from a teacher's top logits, which are stored as a CSR matrix
    distill_apart  the loss, and in a second call its gradient by the logits
    distill_both   the loss and its gradient in one call
    logits         penalties for tokens of the history, biases and grammar masks on the logits of the next token

All inputs are synthetic and drawn on the GPU from a seed.  Ids follow Zipf's law (probability about 1 / (id + 1)), as those of a vocabulary
sorted by frequency do.  `own` False: elementary torch operations in 32 bits, rounded once; True: the library's entry points.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # the tokens of one decoding step for a batch of 16: launch latency
        {"name": "lookup decode 16", "op": "lookup", "tokens": 16, "vocab": 131072, "d": 4096, "table": "bf16", "out": "bf16", "pads": 0.0, "pad": 0},
        # a training batch: 32-bit master table, 16-bit activations
        {"name": "lookup train 16k", "op": "lookup", "tokens": 16384, "vocab": 131072, "d": 4096, "table": "f32", "out": "bf16", "pads": 0.0, "pad": 0},
        # a padded batch of odd length and width, the table a block of columns of a wider array
        {"name": "lookup ragged odd", "op": "lookup", "tokens": 50021, "vocab": 50257, "d": 1001, "table": "f16", "out": "f16", "pads": 0.1, "pad": 3},
        # fine-tuning on a few sequences, 16-bit gradient that overwrites
        {"name": "gradient finetune 2k", "op": "gradient", "tokens": 2048, "vocab": 32000, "d": 1024, "type": "bf16", "grad": "bf16", "add": False, "pads": 0.0, "pad": 0},
        # a training batch added to the gradient that the tied output layer has left in the same table
        {"name": "gradient tied 16k", "op": "gradient", "tokens": 16384, "vocab": 131072, "d": 4096, "type": "bf16", "grad": "f32", "add": True, "pads": 0.0, "pad": 0},
        # many short padded sequences of a narrow model, odd vocabulary; the most frequent ids have thousands of rows each
        {"name": "gradient long 256k", "op": "gradient", "tokens": 262144, "vocab": 50257, "d": 768, "type": "bf16", "grad": "f32", "add": False, "pads": 0.1, "pad": 0},
        # evaluation of a student on a few sequences: only the loss, odd vocabulary, teacher rows of 0 to 32 entries
        {"name": "distill loss odd", "op": "distill_loss", "rows": 1023, "vocab": 50257, "k": 32, "ragged": True, "type": "f32", "inv_t": 1.0, "pad": 0},
        # training with the loss and its gradient in separate calls, as an engine of automatic differentiation makes them
        {"name": "distill apart 2k", "op": "distill_apart", "rows": 2048, "vocab": 32000, "k": 64, "ragged": False, "type": "bf16", "inv_t": 0.5, "pad": 0},
        # training on a large vocabulary, both at once
        {"name": "distill both 4k", "op": "distill_both", "rows": 4096, "vocab": 131072, "k": 64, "ragged": False, "type": "bf16", "inv_t": 0.5, "pad": 0},
        # one sequence's next token under a grammar
        {"name": "logits single", "op": "logits", "rows": 1, "vocab": 131072, "history": 512, "bias": 8, "mask": True, "type": "bf16", "out": "f32", "pad": 0},
        # a serving batch, half of its rows under a grammar
        {"name": "logits batch 256", "op": "logits", "rows": 256, "vocab": 131072, "history": 2048, "bias": 64, "mask": True, "type": "bf16", "out": "f32", "pad": 0},
        # a few long conversations over an odd vocabulary, no grammar
        {"name": "logits long history", "op": "logits", "rows": 33, "vocab": 50257, "history": 32768, "bias": 300, "mask": False, "type": "f32", "out": "f32", "pad": 5},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _even(rng, n, to):
    """Half of the sizes are multiples of `to`, the others any number."""
    return n // to * to if n > to and rng.random() < 0.5 else n


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["lookup", "gradient", "gradient", "distill_loss", "distill_apart", "distill_both", "logits", "logits"])
        case = {"op": op, "vocab": _even(rng, _log(rng, 1000, 262144), 64), "pad": rng.choice([0, 0, 0, 8, 3])}
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op in ("lookup", "gradient"):
            case.update(tokens=_even(rng, _log(rng, 1, 65536 if op == "lookup" else 262144), 256), d=_even(rng, _log(rng, 64, 8192), 64),
                        pads=rng.choice([0.0, 0.0, 0.1, 0.5]))
            if op == "lookup":
                case.update(table=rng.choice([kind, "f32"]), out=kind)
            else:
                case.update(type=kind, grad=rng.choice([kind, "f32"]), add=rng.random() < 0.5)
        elif op == "logits":
            case.update(rows=_log(rng, 1, 512), history=_log(rng, 1, 32768) * (rng.random() < 0.9), bias=_log(rng, 1, 300) * (rng.random() < 0.7),
                        mask=rng.random() < 0.6, type=kind, out=rng.choice([kind, "f32"]))
        else:
            case.update(rows=_even(rng, _log(rng, 1, 8192), 64), k=_log(rng, 1, 256), ragged=rng.random() < 0.5, type=kind,
                        inv_t=rng.choice([1.0, 0.5, 0.25, 1.25]))
        if work(case)["bytes"] <= most:
            return case


def _distinct(tokens, vocab):
    """How many different ids so many draws of Zipf's law have: a sum over blocks of the vocabulary, a factor of 1.25 wide each."""
    lo, got = 1.0, 0.0
    while lo < vocab + 1:
        hi = min(vocab + 1.0, max(lo + 1, lo * 1.25))
        each = math.log(hi / lo) / math.log(vocab + 1) / (hi - lo)
        got += (hi - lo) * -math.expm1(tokens * math.log1p(-min(each, 0.999)))
        lo = hi
    return got


def work(case):
    op, v = case["op"], case["vocab"]
    if op in ("lookup", "gradient"):
        t, d = case["tokens"], case["d"]
        real = t * (1 - case["pads"])
        rows = _distinct(real, v)
        if op == "lookup":
            return {"bytes": 4 * t + rows * d * SIZE[case["table"]] + t * d * SIZE[case["out"]], "flops": real * d}
        table = 2 * rows if case["add"] else v
        return {"bytes": 4 * t + real * d * SIZE[case["type"]] + table * d * SIZE[case["grad"]], "flops": real * d}
    r = case["rows"]
    if op == "logits":
        mean = 0.75 * case["history"]
        extra = 4 * mean + 8 * case["bias"] + (v / 8 if case["mask"] else 0)
        return {"bytes": r * (v * (SIZE[case["type"]] + SIZE[case["out"]]) + extra), "flops": r * (4 * mean + case["bias"])}
    nnz = r * case["k"] * (0.5 if case["ragged"] else 1)
    writes = 0 if op == "distill_loss" else 1
    return {"bytes": r * v * SIZE[case["type"]] * (1 + writes) + 8 * nnz + 8 * r, "flops": r * v * (4 + 4 * writes)}


def _block(rows, cols, pad, dtype, g, spread=1.0):
    """A matrix of normal values whose rows are `pad` elements further apart than they are long."""
    x = torch.randn((rows, cols + pad), device="cuda", generator=g)
    return x.mul_(spread).to(dtype)[:, :cols]


def _ids(shape, vocab, g):
    u = torch.rand(shape, device="cuda", generator=g, dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1).to(torch.int32)


def _pointers(lengths):
    p = torch.zeros(lengths.numel() + 1, dtype=torch.int32, device="cuda")
    p[1:] = lengths.cumsum(0)
    return p


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, v, pad = case["op"], case["vocab"], case["pad"]
    s = dict(case)
    if op in ("lookup", "gradient"):
        t, d = case["tokens"], case["d"]
        ids = _ids(t, v, g)
        if case["pads"]:
            ids[torch.rand(t, device="cuda", generator=g) < case["pads"]] = -1
        s.update(ids=ids, scale=math.sqrt(d) if op == "lookup" else 1 / math.sqrt(d))
        if op == "lookup":
            s["E"] = _block(v, d, pad, TYPES[case["table"]], g, 0.02)
        else:
            s["dout"] = _block(t, d, pad, TYPES[case["type"]], g, 0.1)
            if case["add"]:
                s["dE"] = _block(v, d, 0, TYPES[case["grad"]], g, 0.01)
        return s
    r = case["rows"]
    if op == "logits":
        s["logits"] = _block(r, v, pad, TYPES[case["type"]], g, 3.0)
        if case["history"]:
            n = case["history"]
            lengths = torch.randint(n // 2, n + 1, (r,), device="cuda", generator=g)
            s["history_rowptr"] = _pointers(lengths)
            s["history"] = _ids(int(lengths.sum()), v, g)
            s["generated_from"] = (lengths * torch.rand(r, device="cuda", generator=g)).to(torch.int32)  # the prompt lies before it
            s["repetition"] = 1 + 0.3 * torch.rand(r, device="cuda", generator=g)
            s["presence"] = 0.5 * torch.rand(r, device="cuda", generator=g)
            s["frequency"] = 0.2 * torch.rand(r, device="cuda", generator=g)
        if case["bias"]:
            n = case["bias"]
            s["bias_rowptr"] = torch.arange(r + 1, device="cuda", dtype=torch.int32) * n
            s["bias_tokens"] = _ids(r * n, v, g)
            s["bias_vals"] = 4 * torch.randn(r * n, device="cuda", generator=g)
        if case["mask"]:  # a grammar allows few tokens or most; every other row has none
            words = (v + 31) // 32
            share = torch.rand((r, 1, 1), device="cuda", generator=g) ** 2
            share[1::2] = 1.0
            bits = torch.rand((r, words, 32), device="cuda", generator=g) < share
            s["mask"] = (bits.to(torch.int64) << torch.arange(32, device="cuda")).sum(-1).to(torch.int32)
        return s
    k = min(case["k"], v)
    s["Z"] = _block(r, v, pad, TYPES[case["type"]], g, 2.0)
    lengths = torch.randint(0, k + 1, (r,), device="cuda", generator=g) if case["ragged"] else torch.full((r,), k, device="cuda")
    s["rowptr"] = _pointers(lengths)
    gaps = 1 + (torch.rand((r, k), device="cuda", generator=g) * (v // k)).long().clamp_(max=v // k - 1)
    cols = gaps.cumsum(1) - 1  # distinct, below v
    there = torch.arange(k, device="cuda") < lengths[:, None]
    s["colidx"] = cols[there].to(torch.int32)
    top = 8 + 4 * torch.rand((r, k), device="cuda", generator=g)
    s["vals"] = top[there]
    # the student has learnt some of it
    rows = torch.arange(r, device="cuda")[:, None].expand(r, k)
    s["Z"][rows[there], cols[there]] = (top[there] + torch.randn(s["vals"].shape, device="cuda", generator=g)).to(s["Z"].dtype)
    # the mean of the rows' losses times the temperature squared; with 16-bit floats of small range a scaled sum, so that gradients stay normal numbers
    s["dloss"] = torch.full((r,), 64.0 if case["type"] == "f16" else 1.0 / r, device="cuda") / case["inv_t"] ** 2
    return s


# ---------------------------------------------------------------- plain forms

def _plain_lookup(s):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < s["vocab"])
    rows = s["E"][ids.clamp(0, s["vocab"] - 1)].float() * s["scale"]
    return torch.where(there[:, None], rows, 0.0).to(TYPES[s["out"]])


def _plain_gradient(s):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < s["vocab"])
    rows = torch.where(there[:, None], s["dout"].float(), 0.0)
    total = torch.zeros((s["vocab"], s["d"]), device="cuda").index_add_(0, ids.clamp(0, s["vocab"] - 1), rows)
    total *= s["scale"]
    if not s["add"]:
        return total.to(TYPES[s["grad"]])
    s["dE"].copy_(s["dE"].float() + total)
    return s["dE"]


def _row_of(rowptr, n):
    """The row of each stored entry."""
    return torch.repeat_interleave(torch.arange(rowptr.numel() - 1, device="cuda"), (rowptr[1:] - rowptr[:-1]).long(), output_size=n)


def _plain_teacher(s, row):
    """Probabilities and logarithms of them of the stored entries, over each row's own."""
    x = s["vals"] * s["inv_t"]
    top = torch.full((s["rows"],), -math.inf, device="cuda").scatter_reduce_(0, row, x, "amax")
    e = torch.exp(x - top[row])
    total = torch.zeros(s["rows"], device="cuda").index_add_(0, row, e)
    return e / total[row], x - top[row] - torch.log(total[row])


def _plain_distill(s, with_gradient):
    row, col = _row_of(s["rowptr"], s["colidx"].numel()), s["colidx"].long()
    p, log_p = _plain_teacher(s, row)
    z = s["Z"].float()
    top = z.amax(1)
    e = torch.exp((z - top[:, None]) * s["inv_t"])
    total = e.sum(1)
    log_q = (s["Z"][row, col].float() - top[row]) * s["inv_t"] - torch.log(total[row])
    # differences of like numbers: 64 bits until they are added up
    loss = torch.zeros(s["rows"], device="cuda", dtype=torch.float64).index_add_(0, row, p.double() * (log_p.double() - log_q.double())).float()
    if not with_gradient:
        return {"loss": loss, "stats": torch.stack([top, total], 1)}
    some = (s["rowptr"][1:] > s["rowptr"][:-1]).float()
    dz = e * (some / total)[:, None]
    dz.index_put_((row, col), -p, accumulate=True)
    return {"loss": loss, "dZ": (dz * (s["dloss"] * s["inv_t"])[:, None]).to(s["Z"].dtype)}


def _plain_logits(s):
    r, v = s["rows"], s["vocab"]
    x = s["logits"].float()
    if "history_rowptr" in s:
        row = _row_of(s["history_rowptr"], s["history"].numel())
        at = row * v + s["history"].long()
        place = torch.arange(at.numel(), device="cuda") - s["history_rowptr"][:-1].long()[row]
        seen = torch.zeros(r * v, dtype=torch.bool, device="cuda").index_fill_(0, at, True).view(r, v)
        count = torch.zeros(r * v, device="cuda").index_add_(0, at, (place >= s["generated_from"][row]).float()).view(r, v)
        rep = s["repetition"][:, None]
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if "bias_rowptr" in s:
        row = _row_of(s["bias_rowptr"], s["bias_tokens"].numel())
        x = x + torch.zeros(r * v, device="cuda").index_add_(0, row * v + s["bias_tokens"].long(), s["bias_vals"]).view(r, v)
    if s["mask"] is not False:
        allowed = (s["mask"][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = torch.where(allowed.view(r, -1)[:, :v] == 1, x, -math.inf)
    return x.to(TYPES[s["out"]])


# ---------------------------------------------------------------- the library's entry points

def _own(s):
    import paper_2405_16883_amd as sp

    op = s["op"]
    if op == "lookup":
        out = torch.empty((s["tokens"], s["d"]), dtype=TYPES[s["out"]], device="cuda")
        sp.scorch_embedding_lookup(s["ids"], s["E"], out, s["scale"])
        return out
    if op == "gradient":
        dE = s["dE"] if s["add"] else torch.empty((s["vocab"], s["d"]), dtype=TYPES[s["grad"]], device="cuda")
        sp.scorch_embedding_gradient(s["ids"], s["dout"], dE, s["scale"], accumulate=s["add"])
        return dE
    if op == "logits":
        out = torch.empty((s["rows"], s["vocab"]), dtype=TYPES[s["out"]], device="cuda")
        more = {}
        if "history_rowptr" in s:
            more.update({k: s[k] for k in ("history_rowptr", "history", "generated_from", "repetition", "presence", "frequency")})
        if "bias_rowptr" in s:
            more.update({k: s[k] for k in ("bias_rowptr", "bias_tokens", "bias_vals")})
        if s["mask"] is not False:
            more["mask"] = s["mask"]
        sp.scorch_logits_process(s["logits"], out, **more)
        return out
    loss = torch.empty(s["rows"], device="cuda")
    teacher = (s["rowptr"], s["colidx"], s["vals"])
    if op == "distill_both":
        dZ = torch.empty((s["rows"], s["vocab"]), dtype=s["Z"].dtype, device="cuda")
        sp.scorch_distill_loss_gradient(s["Z"], *teacher, s["inv_t"], s["dloss"], loss, dZ)
        return {"loss": loss, "dZ": dZ}
    stats = torch.empty((s["rows"], 2), device="cuda")
    sp.scorch_distill_loss(s["Z"], *teacher, s["inv_t"], loss, stats)
    if op == "distill_loss":
        return {"loss": loss, "stats": stats}
    dZ = torch.empty((s["rows"], s["vocab"]), dtype=s["Z"].dtype, device="cuda")
    sp.scorch_distill_gradient(s["Z"], *teacher, s["inv_t"], stats, s["dloss"], dZ)
    return {"loss": loss, "dZ": dZ}


def run(state):
    if own:
        return _own(state)
    op = state["op"]
    if op == "lookup":
        return _plain_lookup(state)
    if op == "gradient":
        return _plain_gradient(state)
    if op == "logits":
        return _plain_logits(state)
    return _plain_distill(state, op != "distill_loss")


# ---------------------------------------------------------------- 64 bits, from the definitions

def _exact_gradient(s):
    """Rows in the order of their ids; the sum of a run is the difference of running sums at its ends."""
    order = torch.argsort(s["ids"], stable=True)
    order = order[int((s["ids"] < 0).sum()):]
    ids = s["ids"][order].long()
    edge = torch.searchsorted(ids, torch.arange(s["vocab"] + 1, device="cuda"))
    out = []
    for c in range(0, s["d"], 512):
        run_sum = torch.zeros((ids.numel() + 1, min(512, s["d"] - c)), dtype=torch.float64, device="cuda")
        torch.cumsum(s["dout"][:, c:c + 512][order].double(), 0, out=run_sum[1:])
        out.append((run_sum[edge[1:]] - run_sum[edge[:-1]]) * s["scale"])
    total = torch.cat(out, 1)
    return total + s["dE"].double() if s["add"] else total


def _exact_distill(s, with_gradient):
    p = s["rowptr"].tolist()
    loss = torch.zeros(s["rows"], dtype=torch.float64, device="cuda")
    stats = torch.empty((s["rows"], 2), dtype=torch.float64, device="cuda")
    dZ = torch.empty((s["rows"], s["vocab"]), dtype=torch.float64, device="cuda") if with_gradient else None
    for i in range(s["rows"]):
        z, c = s["Z"][i].double(), s["colidx"][p[i]:p[i + 1]].long()
        log_q = torch.log_softmax(z * s["inv_t"], 0)
        log_p = torch.log_softmax(s["vals"][p[i]:p[i + 1]].double() * s["inv_t"], 0)
        if c.numel():
            loss[i] = (log_p.exp() * (log_p - log_q[c])).sum()
        if with_gradient:
            if c.numel():
                g = log_q.exp()
                g[c] -= log_p.exp()  # the columns of a row are distinct here
                dZ[i] = g * (s["dloss"][i].double() * s["inv_t"])
            else:
                dZ[i] = 0
        else:
            stats[i, 0] = z.max()
            stats[i, 1] = torch.exp((z - z.max()) * s["inv_t"]).sum()
    return {"loss": loss, "dZ": dZ} if with_gradient else {"loss": loss, "stats": stats}


def _exact_logits(s):
    out = s["logits"].double().clone()
    v = s["vocab"]
    hp = s["history_rowptr"].tolist() if "history_rowptr" in s else None
    bp = s["bias_rowptr"].tolist() if "bias_rowptr" in s else None
    for i in range(s["rows"]):
        x = out[i]
        if hp:
            tokens, start = s["history"][hp[i]:hp[i + 1]].long(), int(s["generated_from"][i])
            for_all = torch.bincount(tokens, minlength=v) > 0
            count = torch.bincount(tokens[start:], minlength=v).double()
            r = s["repetition"][i].double()
            x = torch.where(for_all & (x > 0), x / r, torch.where(for_all, x * r, x))
            x = x - count * s["frequency"][i].double() - s["presence"][i].double() * (count != 0)
        if bp:
            x = x + torch.bincount(s["bias_tokens"][bp[i]:bp[i + 1]].long(), weights=s["bias_vals"][bp[i]:bp[i + 1]].double(), minlength=v)
        if s["mask"] is not False:
            words = s["mask"][i].long() & 0xFFFFFFFF
            forbidden = torch.stack([(words >> b) & 1 for b in range(32)], 1).reshape(-1)[:v] == 0
            x = x.masked_fill(forbidden, -math.inf)
        out[i] = x
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "lookup":
        out = torch.zeros((s["tokens"], s["d"]), dtype=torch.float64, device="cuda")
        real = torch.nonzero(s["ids"] >= 0)[:, 0]
        out[real] = s["E"].index_select(0, s["ids"][real]).double() * s["scale"]
        return out
    if op == "gradient":
        return _exact_gradient(s)
    if op == "logits":
        return _exact_logits(s)
    return _exact_distill(s, op != "distill_loss")
