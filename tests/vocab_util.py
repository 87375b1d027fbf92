"""Plain 64-bit forms of the vocabulary operators on the CPU, with bounds for what 32-bit arithmetic and one rounding may be off.

A rounding to a type is off by at most half a step, relative to the value; u(t) is that half step, and one 32-bit operation is off
by U = 2^-24 of its result.  exp2 and log are taken as off by 2 U."""
import numpy as np
import torch

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SENTINEL = -77.0


def u(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half the distance between the smallest numbers of a type; results of 32 bits below 2^-126 may be flushed."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2 if dtype == torch.float16 else 2.0 ** -126


def padded(rows, cols, pad, dtype, fill=SENTINEL):
    """A matrix whose rows are `pad` further apart than they are long, and the buffer around it."""
    buf = torch.full((max(rows, 1), cols + pad), fill, dtype=dtype, device="cuda")
    return buf[:rows, :cols], buf


def csr(lists):
    """Row pointers and the joined lists, on the GPU."""
    rowptr = torch.tensor(np.concatenate([[0], np.cumsum([len(x) for x in lists])]), dtype=torch.int32, device="cuda")
    return rowptr, np.concatenate([np.asarray(x) for x in lists]) if len(lists) else np.zeros(0)


def assert_within(got, ref, tol, what=""):
    got, ref, tol = got.double().cpu().numpy(), np.asarray(ref), np.asarray(tol)
    same = (got == ref) | (np.isnan(got) & np.isnan(ref))  # infinities too
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - ref) <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off; first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[bad][0]} +- {np.broadcast_to(tol, bad.shape)[bad][0]}"


def gradient_ref(ids, dout, vocab, scale, old=None):
    """(value, bound without the result's rounding): a sum of n rows in 32 bits is off by at most n U of the sum of magnitudes."""
    ids, x = ids.cpu().numpy(), dout.double().cpu().numpy()
    ok = (ids >= 0) & (ids < vocab)
    ref, mag = np.zeros((vocab, x.shape[1])), np.zeros((vocab, x.shape[1]))
    np.add.at(ref, ids[ok], x[ok])
    np.add.at(mag, ids[ok], np.abs(x[ok]))
    n = np.bincount(ids[ok], minlength=vocab)[:, None]
    scale = float(np.float32(scale))
    ref, mag = ref * scale, mag * abs(scale)
    if old is not None:
        old = old.double().cpu().numpy()
        ref, mag = ref + old, mag + np.abs(old)
    return ref, (n + 3) * U * mag


def distill_ref(Z, lists, inv_t, dloss=None):
    """Z: CPU tensor; lists: per row (columns, values).  Loss, stats and gradient in 64 bits, with their bounds.

    S is a sum of V terms: every thread of 256 or more adds its share one by one and may rescale it, the partial sums go through a tree of
    ten levels; a term's argument y is off by 3 U y, which is at most 3 U / e of a sum that is at least 1."""
    z_all = Z.double().numpy()
    x = float(np.float32(inv_t))
    rows, vocab = z_all.shape
    loss, loss_tol = np.zeros(rows), np.zeros(rows)
    stats = np.zeros((rows, 2))
    dz, dz_tol = np.zeros((rows, vocab)), np.zeros((rows, vocab))
    s_err = (vocab / 256 + 60) * U
    for i in range(rows):
        c, t = np.asarray(lists[i][0], dtype=np.int64), np.asarray(lists[i][1], dtype=np.float32).astype(np.float64)
        keep = (c >= 0) & (c < vocab) & (t != -np.inf)
        c, t = c[keep], t[keep]
        z = z_all[i]
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            top = z.max() if vocab else -np.inf
            w = x * (z - top)
            e = np.exp(w)
            s = e.sum()
            q = e / s
            stats[i] = top, s
            if not len(c):
                continue
            y = x * (t - t.max())
            p = np.exp(y) / np.exp(y).sum()
            term = y - np.log(np.exp(y).sum()) - (w[c] - np.log(s))
            loss[i] = np.where(p == 0, 0, p * term).sum()
            p_err = (len(c) / 256 + 60 + 4 * np.abs(y)) * U
            loss_tol[i] = np.where(p == 0, 0, p * (p_err * np.abs(term) + 4 * U * (np.abs(y) + np.abs(w[c]) + 40))).sum() + s_err + len(c) * U * np.abs(p * term).max()
            g = q.copy()
            np.add.at(g, c, -p)
            weight = x * (1.0 if dloss is None else float(dloss[i]))
            dz[i] = g * weight
            err = np.where(q > 0, (s_err + (8 + 4 * np.abs(w)) * U) * q, 0)
            np.add.at(err, c, (p_err + 8 * U) * p)
            dz_tol[i] = abs(weight) * err + 4 * U * np.abs(dz[i])
    return loss, loss_tol, stats, s_err, dz, dz_tol


def logits_ref(logits, history=None, start=None, rep=None, pres=None, freq=None, bias=None, mask=None):
    """(value, bound without the result's rounding).  history: lists of tokens; bias: lists of (tokens, values); mask: truth values."""
    x = logits.double().cpu().numpy()
    rows, vocab = x.shape
    out, tol = np.zeros_like(x), np.zeros_like(x)
    for i in range(rows):
        y, err = x[i].copy(), np.zeros(vocab)
        f32 = lambda a: float(np.float32(a[i])) if a is not None else None  # noqa: E731
        if history is not None:
            tokens = np.asarray(history[i], dtype=np.int64)
            place = np.arange(len(tokens))
            inside = (tokens >= 0) & (tokens < vocab)
            seen = np.zeros(vocab, dtype=bool)
            seen[tokens[inside]] = True
            late = inside & (place >= (start[i] if start is not None else 0))
            count = np.bincount(tokens[late], minlength=vocab)
            if rep is not None:
                y = np.where(seen, np.where(y > 0, y / f32(rep), y * f32(rep)), y)
                err += np.where(seen & np.isfinite(y), 2 * U * np.abs(y), 0)
            for part in ((count * f32(freq)) if freq is not None else None, np.where(count > 0, f32(pres), 0) if pres is not None else None):
                if part is not None:
                    y = y - part
                    err += np.where(np.isfinite(y), U * (np.abs(part) + np.abs(y)), 0)
        if bias is not None:
            tokens, values = np.asarray(bias[i][0], dtype=np.int64), np.asarray(bias[i][1], dtype=np.float32).astype(np.float64)
            inside = (tokens >= 0) & (tokens < vocab)
            add, mag, n = np.zeros(vocab), np.zeros(vocab), np.bincount(tokens[inside], minlength=vocab)
            np.add.at(add, tokens[inside], values[inside])
            np.add.at(mag, tokens[inside], np.abs(values[inside]))
            y = np.where(n > 0, y + add, y)
            with np.errstate(invalid="ignore"):
                err += np.where((n > 0) & np.isfinite(y), U * (n * mag + np.abs(y)), 0)
        if mask is not None:
            y, err = np.where(mask[i], y, -np.inf), np.where(mask[i], err, 0)
        out[i], tol[i] = y, err
    return out, tol


def pack_mask(mask):
    """Truth values (rows x vocab) as int32 words, a bit per column; the bits behind the last column are set."""
    rows, vocab = mask.shape
    bits = np.ones((rows, (vocab + 31) // 32 * 32), dtype=np.uint8)
    bits[:, :vocab] = mask
    return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32).copy()).cuda()
