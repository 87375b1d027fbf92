"""Distillation of many rows: every number of threads per row and of vectors held, against the definition in 64 bits on some of the rows."""
import numpy as np
import pytest
import torch

import paper_2405_16883_amd as sp
from vocab_util import SENTINEL, TYPES, U, assert_within, distill_ref, tiny, u

pytestmark = pytest.mark.gpu
INF = float("inf")


class Problem:
    """Rows of random logits with a short list each; some rows have what goes wrong most easily: no entries, columns that repeat, more entries
    than threads, a column throughout, entries outside, logits that are -infinity or not a number."""

    def __init__(self, rows, vocab, kind, seed, pad=0, offset=0):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        dtype, ld = TYPES[kind], vocab + pad
        self.rows, self.vocab, self.pad, self.offset = rows, vocab, pad, offset
        self.Z = self.matrix(dtype)
        self.Z.copy_(torch.randn((rows, vocab), device="cuda", generator=g).mul_(3))
        special = sorted(rng.permutation(rows)[:9].tolist())
        self.lists = [None] * rows
        for i in range(rows):
            n = int(rng.integers(1, 41))
            self.lists[i] = (rng.integers(0, vocab, n) if i % 5 == 0 else rng.permutation(min(vocab, 4096))[:n] * (vocab // min(vocab, 4096)), None)
        a, b, c, d, e, f, h, i, j = special
        self.lists[a] = (np.zeros(0, dtype=np.int64), None)
        self.lists[b] = (rng.integers(0, vocab, 1500), None)
        self.lists[c] = (np.full(70, vocab - 1), None)
        self.lists[d] = (np.array([-1, vocab, 3, 2 ** 31 - 1, 3]), None)
        self.Z[e, vocab - 1] = float("nan")
        self.Z[f] = -INF
        self.Z[h, ::2] = -INF
        self.lists[h] = (np.array([1, 3, 1]), None)
        self.Z[i, 0] = INF
        self.lists[j] = (np.array([0, vocab - 1, vocab // 2]), None)
        self.lists = [(cols, rng.normal(5, 3, len(cols)).astype(np.float32)) for cols, _ in self.lists]
        self.numbers = [r for r in range(rows) if r not in (e, f, i)]
        self.sample = sorted({0, rows - 1, rows // 2, *special, *rng.permutation(rows)[:6].tolist()})
        self.rowptr = torch.from_numpy(np.concatenate([[0], np.cumsum([len(x) for x, _ in self.lists])]).astype(np.int32)).cuda()
        self.colidx = torch.from_numpy(np.concatenate([x for x, _ in self.lists]).astype(np.int32)).cuda()
        self.vals = torch.from_numpy(np.concatenate([t for _, t in self.lists])).cuda()
        self.dloss = torch.from_numpy(rng.uniform(0.5, 2, rows).astype(np.float32)).cuda()

    def matrix(self, dtype):
        """rows x vocab, beginning `offset` elements into a buffer whose rows are `pad` further apart."""
        ld = self.vocab + self.pad
        self.buffer = torch.full((self.rows * ld + self.offset + 8,), SENTINEL, dtype=dtype, device="cuda")
        return self.buffer[self.offset:].as_strided((self.rows, self.vocab), (ld, 1))

    def outside_is_untouched(self):
        written = torch.zeros_like(self.buffer, dtype=torch.bool)
        written[self.offset:].as_strided((self.rows, self.vocab), (self.vocab + self.pad, 1)).fill_(True)
        return (self.buffer[~written] == SENTINEL).all()

    def reference(self, inv_t, threads):
        """Loss, its bound, stats and gradient of the sampled rows.  The bounds of distill_ref are for 256 threads or more, which add up vocab / 256
        numbers one by one; fewer threads add up vocab / threads."""
        s = self.sample
        more = max(0.0, (self.vocab / threads - self.vocab / 256) * U)
        dloss = self.dloss[s].cpu().numpy()
        loss, tol, stats, s_err, dz, dz_tol = distill_ref(self.Z[s].cpu(), [self.lists[i] for i in s], inv_t, dloss)
        with np.errstate(invalid="ignore"):
            dz_tol = dz_tol + more * (np.abs(dz) + dz_tol + abs(inv_t) * dloss[:, None])
        return loss, tol + more, stats, s_err + more, dz, dz_tol


def assert_gradient(p, got, dz, tol):
    got = got[p.sample]
    assert_within(got, dz, tol + u(got.dtype) * (np.abs(dz) + tol) + tiny(got.dtype), "gradient")


@pytest.mark.parametrize("rows,vocab,threads", [(1030, 2999, 512), (1024, 40001, 512), (2047, 4097, 512), (2048, 1000, 64), (2050, 4096, 64),
                                                (4099, 37, 64), (2048, 4097, 256), (2100, 20001, 256)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_loss_then_gradient(rows, vocab, threads, kind):
    p = Problem(rows, vocab, kind, rows + vocab, pad=vocab % 2 * 5, offset=vocab % 8)
    inv_t = [1.0, 0.5, 1.7][vocab % 3]
    ref, tol, ref_stats, s_err, dz, dz_tol = p.reference(inv_t, threads)
    loss, stats = torch.full((rows,), SENTINEL, device="cuda"), torch.full((rows, 2), SENTINEL, device="cuda")
    sp.scorch_distill_loss(p.Z, p.rowptr, p.colidx, p.vals, inv_t, loss, stats)
    assert_within(loss[p.sample], ref, tol, "loss")
    assert loss[p.numbers].isfinite().all()
    top = ref_stats[:, 0]
    with np.errstate(invalid="ignore"):
        fine = np.isfinite(ref_stats).all(axis=1)
        assert_within(stats[p.sample][fine, 0], top[fine], 0, "largest logit")
        assert_within(stats[p.sample][fine, 1], ref_stats[fine, 1], s_err * ref_stats[fine, 1], "sum of exponentials")
    Z = p.Z
    dZ = p.matrix(Z.dtype)
    sp.scorch_distill_gradient(Z, p.rowptr, p.colidx, p.vals, inv_t, stats, p.dloss, dZ)
    assert_gradient(p, dZ, dz, dz_tol)
    assert dZ[p.numbers].isfinite().all() and p.outside_is_untouched()
    sp.scorch_distill_gradient(Z, p.rowptr, p.colidx, p.vals, inv_t, stats, p.dloss, Z)  # in place
    assert torch.equal(Z.isnan(), dZ.isnan()) and torch.equal(Z.nan_to_num(), dZ.nan_to_num())


# Columns on both sides of what the threads' registers hold, in 16-bit types (half as many in 32 bits): 64 x 4, 256 x 4, 256 x 16, 512 x 16, 512 x 20
# vectors, and rows that are longer than these.
@pytest.mark.parametrize("columns,threads", [(2000, 64), (2048, 64), (2050, 256), (5000, 256), (8194, 256), (30000, 256), (32768, 256), (32770, 512), (60000, 512),
                                             (65538, 512), (81920, 512), (100006, 512)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shift,in_place", [(0, False), (1, True)])
def test_both_at_once(columns, threads, kind, shift, in_place):
    rows, vocab = 259 + columns % 3, (columns // 2 if kind == "f32" else columns) + shift
    p = Problem(rows, vocab, kind, vocab, pad=shift * 3, offset=shift * 5)
    inv_t = [1.0, 0.5, 1.7][vocab % 3]
    ref, tol, _, _, dz, dz_tol = p.reference(inv_t, threads)
    Z = p.Z
    dZ = Z if in_place else p.matrix(Z.dtype)
    loss = torch.full((rows,), SENTINEL, device="cuda")
    sp.scorch_distill_loss_gradient(Z, p.rowptr, p.colidx, p.vals, inv_t, p.dloss, loss, dZ)
    assert_within(loss[p.sample], ref, tol, "loss")
    assert_gradient(p, dZ, dz, dz_tol)
    assert loss[p.numbers].isfinite().all() and dZ[p.numbers].isfinite().all() and p.outside_is_untouched()


@pytest.mark.parametrize("rows,vocab", [(1, 131072), (3, 100003), (12, 524288), (40, 50257)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_gradient_of_few_rows_in_place(rows, vocab, kind):
    """Rows cut over workgroups, each of which may have stored its part before another reads its own."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    Z = torch.randn((rows, vocab), device="cuda", generator=g).mul_(3).to(TYPES[kind])
    k = 300
    rowptr = torch.arange(rows + 1, dtype=torch.int32, device="cuda") * k
    colidx = torch.randint(0, vocab, (rows * k,), dtype=torch.int32, device="cuda", generator=g)
    colidx[:k] %= 50  # columns that repeat
    vals = torch.randn(rows * k, device="cuda", generator=g)
    loss, stats = torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")
    sp.scorch_distill_loss(Z, rowptr, colidx, vals, 0.5, loss, stats)
    want = torch.empty_like(Z)
    sp.scorch_distill_gradient(Z, rowptr, colidx, vals, 0.5, stats, None, want)
    sp.scorch_distill_gradient(Z, rowptr, colidx, vals, 0.5, stats, None, Z)
    assert torch.equal(Z, want)
