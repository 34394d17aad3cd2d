"""Attention over paged caches with shared prefixes against the 64-bit oracle on the sequences' logical caches.

How far a value may be off.  A probability is rounded to bf16 (half a step, 2^-8), so an output is off by at most 2^-8 A with A = sum_j p_j |v_j|,
and rounded to bf16 itself.  Scores are sums of D products in 32 bits: at most (D + 4) 2^-24 times the sum of the products' sizes, below 2^-11 for the
inputs here (products of at most 64 together), twice that in a ratio of two sums: 2^-10 A.  The sums of the probabilities are smaller terms."""
import numpy as np
import pytest

import oracle
import workloads as wl
from oracle.kv_int8 import dequantize_rows, quantize_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hip():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2404_15778_amd import harness
    return harness


class Batch:
    """Sequences with common prefixes: logical rows, tables over pages in random order, and the references."""

    def __init__(self, seed, Hq, Hkv, D, P, ctx, nq, kmax, of=None, plen=None, dtype="bf16", scale=None):
        rng = np.random.default_rng(seed)
        self.B, self.kmax, self.Hq, self.Hkv, self.D, self.P, self.dtype = len(ctx), kmax, Hq, Hkv, D, P, dtype
        self.ctx, self.nq = np.array(ctx, np.int32), np.array(nq, np.int32)
        self.of = None if of is None else np.array(of, np.int32)
        self.plen = None if plen is None else np.array(plen, np.int32)
        self.scale = 1.0 / np.sqrt(D) if scale is None else scale
        T = max(1, int((self.ctx + self.nq).max()))
        draw = lambda *s: wl.to_bf16_bits(rng.standard_normal(s, dtype=np.float32))  # noqa: E731
        self.Q = draw(self.B, kmax, Hq, D)
        self.K, self.V = draw(self.B, T, Hkv, D), draw(self.B, T, Hkv, D)
        need = [-(-int(n) // P) for n in self.ctx + self.nq]
        self.most = max(max(need), 1) + 1
        self.n_pages = sum(need) + 3
        ids = iter(rng.permutation(self.n_pages).tolist())
        self.tables = np.full((self.B, self.most), -1, np.int32)
        first = {}
        for b in range(self.B):
            x = -1 if of is None else of[b]
            if x >= 0 and x in first:
                src, n = first[x], int(plen[x])
                n = min(n, int(self.ctx[b]), int(self.ctx[src])) // P * P  # whole pages
                self.tables[b, :n // P] = self.tables[src, :n // P]
                self.K[b, :n], self.V[b, :n] = self.K[src, :n], self.V[src, :n]
            elif x >= 0:
                first[x] = b
            for j in range(need[b]):
                if self.tables[b, j] < 0:
                    self.tables[b, j] = next(ids)

    def pages(self, hip, layers_poison=True):
        pg = hip.DevicePages(self.B, self.kmax, self.Hq, self.Hkv, self.D, self.P, self.n_pages, self.most, self.dtype, self.scale, poison=layers_poison)
        for b in range(self.B):
            n = int(self.ctx[b] + self.nq[b])
            if n:
                t = np.arange(n)
                slots = self.tables[b, t // self.P] * self.P + t % self.P
                pg.append(hip.to_device(self.K[b:b + 1, :n]), hip.to_device(self.V[b:b + 1, :n]), hip.i32(slots[None]))
        return pg

    def run(self, hip, pg=None, share=True, want_lse=True):
        pg = pg or self.pages(hip)
        of, plen = (hip.i32(self.of), hip.i32(self.plen)) if share and self.of is not None else (None, None)
        O, lse = pg.verify(hip.to_device(self.Q), hip.i32(self.tables), hip.i32(self.ctx), hip.i32(self.nq), of, plen, want_lse)
        return wl.bf16_bits_to_f32(hip.to_host(O)), hip.to_host(lse), int(pg.status.item())

    def reference(self):
        """(O, lse, A) in 64 bits."""
        x = [wl.bf16_bits_to_f32(y) for y in (self.Q, self.K, self.V)]
        if self.dtype == "int8kv":
            x = [dequantize_rows(*quantize_rows(y)) for y in x]
        O, lse = oracle.verify_attention(*x, self.ctx, self.nq, self.scale)
        A, _ = oracle.verify_attention(x[0], x[1], np.abs(x[2]), self.ctx, self.nq, self.scale)
        return O, lse, A

    def check(self, hip, **kw):
        O, lse, status = self.run(hip, **kw)
        Or, lser, A = self.reference()
        assert status == 0
        assert np.isfinite(O).all() and np.isfinite(lse).all()
        assert (np.abs(O - Or) <= (2 ** -8 * (1 + 2 ** -8) + 2 ** -10) * A + 2 ** -8 * np.abs(Or) + 1e-30).all()
        assert (np.abs(lse - lser) <= 2 ** -11 + 2 ** -20 * np.abs(lser)).all()
        for b in range(self.B):
            assert (O[b, self.nq[b]:] == 0).all() and (lse[b, self.nq[b]:] == 0).all()
        return O, lse


HEADS = [(4, 4, 64), (8, 2, 128), (28, 4, 128), (6, 2, 64), (8, 1, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("P", [32, 96])
def test_sequences_of_all_lengths(hip, dtype, Hq, Hkv, D, P):
    """Nothing shared: no context, one token, block and page borders, unused places, short and longer lists."""
    kmax = min(7, 64 * Hkv // Hq)
    ctx = [0, 0, 1, 31, 32, 33, 95, 96, 97, 500, 5]
    nq = [1, kmax, 0, 1, kmax, 2, 1, kmax, 3, kmax, 0]
    Batch(Hq * 100 + P, Hq, Hkv, D, P, ctx, [min(n, kmax) for n in nq], kmax, dtype=dtype).check(hip)


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("P,n", [(32, 10), (64, 23), (96, 5)])
def test_shared_prefixes(hip, dtype, Hq, Hkv, D, P, n):
    """Two prefixes, sequences without one, a prefix of one sequence, unused places; members in any order."""
    rng = np.random.default_rng([Hq, D, P, n])
    kmax = min(6, 64 * Hkv // Hq)
    of = rng.integers(-1, 2, size=n)
    of[0], of[1], of[2] = 2, 0, 0
    plen = np.array([7 * P, 4 * P, 3 * P])
    ctx = np.where(of >= 0, plen[of], 0) + rng.integers(0, 300, size=n)
    nq = rng.integers(0, kmax + 1, size=n)
    nq[1], nq[2] = kmax, 1
    Batch(n * 7 + P, Hq, Hkv, D, P, ctx, nq, kmax, of, plen, dtype).check(hip)


@pytest.mark.parametrize("n", [2, 9, 33, 70])
def test_many_rows_of_one_prefix(hip, n):
    """From two sequences to several tiles of query rows."""
    rng = np.random.default_rng(n)
    ctx = 640 + rng.integers(0, 70, size=n)
    Batch(n, 8, 2, 128, 64, ctx, rng.integers(0, 9, size=n), 8, np.zeros(n, int), [640]).check(hip)


def test_sharing_is_optional(hip):
    """The same batch with and without its prefixes named, and with a prefix that claims too much."""
    rng = np.random.default_rng(0)
    ctx = 512 + rng.integers(0, 90, size=8)
    batch = Batch(4, 8, 2, 128, 64, ctx, [3] * 8, 4, np.zeros(8, int), [512])
    a, la = batch.check(hip)
    b, lb = batch.check(hip, share=False)
    assert np.abs(a - b).max() <= 2 ** -6 and np.abs(la - lb).max() <= 1e-4


def test_prefix_longer_than_some_sequences(hip):
    """What is common ends with the shortest sequence; whole blocks only; the rest goes by itself."""
    batch = Batch(11, 4, 2, 64, 32, [200, 300, 170, 290], [2, 2, 2, 2], 2, [0, 0, 0, 0], [256])
    batch.check(hip)


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(hip, scale):
    """Products of at most 64 together: |scale| sum |q k| < 3 * 3 * 3 ... is not bounded so for scale 3, so inputs are an eighth."""
    batch = Batch(5, 4, 2, 64, 32, [100, 160, 130], [3, 2, 1], 3, [0, 0, 0], [96], scale=scale)
    batch.Q = wl.to_bf16_bits(wl.bf16_bits_to_f32(batch.Q) / 16)
    batch.check(hip)


def test_no_lse_wanted(hip):
    batch = Batch(6, 4, 2, 64, 32, [100, 160, 130], [3, 2, 1], 3, [0, 0, 0], [96])
    O, lse, status = batch.run(hip, want_lse=False)
    O2, _, _ = batch.run(hip)
    assert status == 0 and np.isnan(lse).all() and np.array_equal(O, O2)


def test_nothing_to_do(hip):
    batch = Batch(7, 4, 2, 64, 32, [100, 0, 130], [0, 0, 0], 3, [0, 0, 0], [96])
    O, lse, status = batch.run(hip)
    assert status == 0 and (O == 0).all() and (lse == 0).all()


def test_exact_counts(hip):
    """All keys zero and small whole values: every visible token counts alike, so lse = log n counts them and O is their mean."""
    rng = np.random.default_rng(8)
    n = 12
    ctx = 1024 + rng.integers(0, 2000, size=n)
    batch = Batch(9, 8, 2, 128, 64, ctx, rng.integers(1, 5, size=n), 4, np.zeros(n, int), [1024])
    batch.K[:] = 0
    batch.V = wl.to_bf16_bits(rng.integers(-8, 9, size=batch.V.shape).astype(np.float32))
    for b in range(1, n):
        batch.V[b, :1024] = batch.V[0, :1024]
    O, lse = batch.check(hip)
    for b in range(n):
        for i in range(batch.nq[b]):
            assert np.abs(lse[b, i] - np.log(ctx[b] + i + 1)).max() <= 2e-6


def test_pages_out_of_range(hip):
    """An entry that is no page: page 0 is read in its place, and the call says so."""
    batch = Batch(10, 4, 2, 64, 32, [100, 160], [2, 2], 2)
    batch.tables[1, 2] = batch.n_pages + 7
    good = Batch(10, 4, 2, 64, 32, [100, 160], [2, 2], 2)
    pg = good.pages(hip, layers_poison=False)
    O, lse, status = batch.run(hip, pg)
    assert status == 16 and np.isfinite(O).all()
    ref, _, A = good.reference()
    assert (np.abs(O[0] - ref[0]) <= 2 ** -6 * A[0]).all()


def test_a_plan_of_another_shape_computes_nothing(hip):
    import torch
    import paper_2404_15778_amd as bass
    batch = Batch(12, 4, 2, 64, 32, [100, 160], [2, 2], 2)
    pg = batch.pages(hip)
    args = (hip.to_device(batch.Q), pg.K, pg.V, hip.i32(batch.tables))
    for plan in (torch.full_like(pg.plan, 0xA5), torch.zeros_like(pg.plan)):
        pg.status.zero_()
        bass.bass_paged_verify_attention(pg.desc, *args, plan, pg.O, pg.lse, pg.ws, pg.status)
        assert int(pg.status.item()) == 8 and torch.isnan(pg.O.float()).all()
    other = pg.desc.replace(max_pages=batch.most + 1)
    plan = bass.alloc_paged_plan(other)
    bass.bass_paged_attention_plan(other, hip.i32(batch.ctx), hip.i32(batch.nq), None, None, plan)
    pg.status.zero_()
    bass.bass_paged_verify_attention(pg.desc, *args, plan, pg.O, pg.lse, pg.ws, pg.status)
    assert int(pg.status.item()) == 8 and torch.isnan(pg.O.float()).all()


def test_lengths_are_clamped_and_prefix_numbers_checked(hip):
    import torch
    batch = Batch(13, 4, 2, 64, 32, [100, 160, 64], [2, 2, 2], 2, [0, 0, 0], [64])
    pg = batch.pages(hip)
    pg.verify(hip.to_device(batch.Q), hip.i32(batch.tables), hip.i32([100, 160, 64]), hip.i32([2, 2, 9]), hip.i32([0, 0, 5]), hip.i32([64]))
    assert int(pg.status.item()) == 1
    O = wl.bf16_bits_to_f32(hip.to_host(pg.O))
    ref, _, A = batch.reference()
    assert (np.abs(O - ref) <= 2 ** -6 * A + 1e-30).all()
    torch.cuda.synchronize()
