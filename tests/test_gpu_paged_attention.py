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


def quantize_queries(x):
    """Codes and scales of query rows over INT8 pools: as of cached rows, with 127 * (1 / amax) in two rounded steps."""
    amax = np.abs(x).max(axis=-1).astype(np.float32)
    with np.errstate(divide="ignore"):
        inv = np.where(amax > 0, (np.float32(1) / amax).astype(np.float32) * np.float32(127), np.float32(0)).astype(np.float32)
    return np.rint(x * inv[..., None]).astype(np.int8), (amax / np.float32(127)).astype(np.float32)


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

    def shared_runs(self, pg):
        """Prefixes that the plan computes for all of their sequences: its second word counts the runs, one per live sequence more or less."""
        return int(pg.plan[:8].cpu().numpy().view(np.int32)[1]) - int((self.nq > 0).sum())

    def reference(self):
        """(O, lse, A) in 64 bits."""
        x = [wl.bf16_bits_to_f32(y) for y in (self.Q, self.K, self.V)]
        if self.dtype == "int8kv":
            x = [dequantize_rows(*f(y)) for f, y in zip((quantize_queries, quantize_rows, quantize_rows), x)]
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


@pytest.mark.parametrize("n", [3, 20])
def test_prefix_that_ends_inside_a_page(hip, n):
    """Whole pages are shared; the rest of the prefix lies in pages of each sequence's own, which hold the same rows."""
    P, common = 96, 20 * 96 + 71
    batch = Batch(13, 32, 8, 128, P, common + np.arange(n) * 7, [3] * n, 4, np.zeros(n, int), [common])
    batch.K[:, :common], batch.V[:, :common] = batch.K[0, :common], batch.V[0, :common]
    pg = batch.pages(hip)
    batch.check(hip, pg=pg)
    assert batch.shared_runs(pg) == (1 if n == 20 else 0)


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


# Query rows per kv head and prefix sizes that take each of the ways: rows of at most 32 (a wavefront has all of them), half a tile of 128 rows and a
# full one, part of a tile of 256 rows, two and three tiles; odd and even numbers of blocks, more than a window of 64.
# members, query tokens, heads, kv heads, prefix tokens
KINDS = [(4, 7, 16, 16, 992), (4, 10, 32, 32, 3712), (4, 16, 32, 32, 3680), (8, 8, 32, 16, 2272), (13, 4, 32, 8, 2688), (19, 4, 32, 8, 2080), (40, 4, 32, 8, 1088)]


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("int8kv", 128), ("int8kv", 64)])
@pytest.mark.parametrize("n,q,Hq,Hkv,P", KINDS)
def test_every_way_of_sharing(hip, dtype, D, n, q, Hq, Hkv, P):
    rng = np.random.default_rng([n, q, P])
    ctx = P + rng.integers(0, 40, size=n)
    nq = rng.integers(max(1, q - 1), q + 1, size=n)
    nq[0] = q
    batch = Batch(n + P, Hq, Hkv, D, 32, ctx, nq, q, np.zeros(n, int), [P], dtype)
    pg = batch.pages(hip)
    batch.check(hip, pg=pg)
    assert batch.shared_runs(pg) == 1


def heads_per_unit(pg):
    """kv heads of a unit where each workgroup of the plan starts (64 bytes of header; 32 bytes and the run of 64 bytes per workgroup)."""
    shares = pg.plan[64:64 + 256 * 96].cpu().numpy().view(np.int32).reshape(256, 24)
    return shares[shares[:, 4] > 0][:, 8 + 13]


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("B,kmax,Hq,Hkv,D,most", [(64, 4, 10, 5, 64, 252), (64, 4, 10, 5, 128, 252), (64, 8, 40, 5, 128, 500), (64, 8, 40, 5, 64, 500),
                                                  (200, 3, 6, 2, 128, 200), (300, 1, 4, 4, 64, 511)])
@pytest.mark.parametrize("shared", [False, True])
def test_many_short_sequences(hip, dtype, B, kmax, Hq, Hkv, D, most, shared):
    """A wavefront per kv head: heads that do not fill the workgroup's four, up to 32 query rows and more, whole units and cut ones, sequences
    alone and the rests of a prefix's."""
    rng = np.random.default_rng([B, Hq, D])
    ctx, nq = rng.integers(0, most - kmax, size=B), rng.integers(0, kmax + 1, size=B)
    nq[:3] = kmax
    of = np.where(np.arange(B) % 3 == 0, 0, -1) if shared else None
    if shared:
        ctx = ctx + 1024 * (of == 0)
    batch = Batch(B + D, Hq, Hkv, D, 32, ctx, nq, kmax, of, [1024] if shared else None, dtype)
    pg = batch.pages(hip)
    batch.check(hip, pg=pg)
    assert (heads_per_unit(pg) == 4).any()


def test_the_same_call_gives_the_same_bits(hip):
    """Nothing depends on the order in which workgroups arrive.  (Equal sequences agree up to rounding only: the list is cut at other blocks of each.)"""
    n = 24
    batch = Batch(3, 32, 8, 128, 64, [2048 + 37] * n, [4] * n, 4, np.zeros(n, int), [2048])
    pg = batch.pages(hip)
    O, lse = batch.check(hip, pg=pg)
    assert batch.shared_runs(pg) == 1
    for _ in range(3):
        pg.ws.fill_(0xFF)
        O2, lse2, _ = batch.run(hip, pg)
        assert np.array_equal(O, O2) and np.array_equal(lse, lse2)


def test_large_batches_and_many_prefixes(hip):
    """More sequences and prefixes than the small planning kernel takes; half of them not in use."""
    rng = np.random.default_rng(4)
    n, G = 300, 40
    of = rng.integers(-1, G, size=n)
    plen = rng.integers(1, 5, size=G) * 32
    ctx = np.where(of >= 0, plen[of], 0) + rng.integers(0, 60, size=n)
    Batch(21, 8, 4, 64, 32, ctx, rng.integers(0, 3, size=n), 2, of, plen).check(hip)


@pytest.mark.parametrize("n,P", [(2, 64), (16, 2048)])
def test_scores_of_any_finite_size(hip, n, P):
    """Products that are exact in 32 bits, up to 2^31: one key wins, the output is its value row.  Apart and together."""
    rng = np.random.default_rng(n)
    batch = Batch(n, 32, 8, 64, 32, [P + 20] * n, [4] * n, 4, np.zeros(n, int), [P], scale=1.0)
    f = np.zeros(batch.Q.shape, np.float32)
    f[..., 0] = 2.0 ** 24
    batch.Q = wl.to_bf16_bits(f)
    k = np.zeros(batch.K.shape, np.float32)
    k[..., 0] = rng.integers(-60, 60, size=k.shape[:-1])
    winner = rng.integers(0, P + 20, size=n)
    k[:, :P] = k[0, :P]
    for b in range(n):
        k[b, winner[b] if winner[b] >= P else winner[0] % P, :, 0] = 100 + (b if winner[b] >= P else 0) % 20
    k[:, :P] = k[0, :P]
    k[:, winner[0] % P, :, 0] = 90
    batch.K = wl.to_bf16_bits(k)
    pg = batch.pages(hip)
    O, lse, status = batch.run(hip, pg)
    assert status == 0 and batch.shared_runs(pg) == (1 if n > 2 else 0)
    v = wl.bf16_bits_to_f32(batch.V)
    for b in range(n):
        for h in range(8):
            for i in range(4):
                row = k[b, :P + 21 + i, h, 0]
                best = np.flatnonzero(row == row.max())
                want = v[b, best, h].astype(np.float64).mean(0)
                assert np.abs(O[b, i, 4 * h:4 * h + 4] - want).max() <= 2 ** -7 * np.abs(v[b, best, h]).max()


@pytest.mark.parametrize("n,P", [(3, 96), (16, 2048)])
def test_an_infinite_value_stays_infinite(hip, n, P):
    batch = Batch(n + 50, 32, 8, 128, 32, [P + 20] * n, [4] * n, 4, np.zeros(n, int), [P])
    v = wl.bf16_bits_to_f32(batch.V)
    v[:, 5, 3, 77] = np.inf
    v[1, P + 2, 1, 11] = -np.inf
    batch.V = wl.to_bf16_bits(v)
    pg = batch.pages(hip)
    O, lse, _ = batch.run(hip, pg)
    assert batch.shared_runs(pg) == (1 if n > 3 else 0)
    want = np.zeros(O.shape, np.float32)
    want[:, :, 12:16, 77] = np.inf
    want[1, :, 4:8, 11] = -np.inf
    assert np.array_equal(np.where(np.isinf(O), O, 0), want) and not np.isnan(O).any()


def test_a_context_of_two_million_tokens(hip):
    """More blocks per workgroup than a window of page numbers: keys are zero, so every token counts alike; a block's values are one number."""
    import torch
    n = 2_200_000 + 5
    P = 4096
    pages = n // P + 2
    pg = hip.DevicePages(1, 2, 2, 1, 64, P, pages, pages, "bf16", 1.0)
    blocks = pages * P // 32
    value = torch.randint(-8, 9, (blocks,), device="cuda").float()
    pg.V.view(torch.bfloat16).view(blocks, 32 * 64).copy_(value[:, None].expand(-1, 32 * 64))
    tables = torch.randperm(pages, device="cuda").to(torch.int32)[None].contiguous()
    order = (tables[0].long()[:, None] * (P // 32) + torch.arange(P // 32, device="cuda")).view(-1)
    per_token = value[order].double().repeat_interleave(32)
    Q = torch.randn((1, 2, 2, 64), device="cuda").to(torch.bfloat16)
    O, lse = pg.verify(Q, tables, hip.i32([n - 2]), hip.i32([2]))
    for i in range(2):
        mean = per_token[:n - 1 + i].mean().item()
        assert abs(lse[0, i].cpu().numpy() - np.log(n - 1 + i)).max() <= 2e-6
        assert (O[0, i].float() - mean).abs().max().item() <= 2 ** -8 * abs(mean) + 1e-6 * 8
    assert int(pg.status.item()) == 0


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("int8kv", 128), ("int8kv", 64)])
@pytest.mark.parametrize("n", [10, 40])
@pytest.mark.parametrize("blocks", [2100, 4301])
def test_long_stretches_of_a_shared_prefix(hip, dtype, D, n, blocks):
    """65 and 134 blocks per workgroup and what lies around them, in tiles of 60 and of 240 query rows.  Keys are zero, so that lse counts the tokens; a
    page's values are one whole number (O: probabilities, over INT8 pages times the scale, and O itself are rounded to bf16: 2^-8 each)."""
    rng = np.random.default_rng([blocks, n])
    Hq, Hkv, P, q, unique = 16, 8, 32, 3, 150
    pages = unique + 2 * n
    pg = hip.DevicePages(n, q, Hq, Hkv, D, P, pages, blocks + 2, dtype, 0.125)
    value = rng.integers(-8, 9, size=pages)
    V = np.repeat(value, P).astype(np.float32)[None, :, None, None] * np.ones((1, 1, Hkv, D), np.float32)
    pg.append(hip.to_device(np.zeros(V.shape, np.uint16)), hip.to_device(wl.to_bf16_bits(V)), hip.i32(np.arange(pages * P)[None]))
    prefix = rng.integers(0, unique, size=blocks)
    own = unique + rng.permutation(2 * n).reshape(n, 2)
    tables = np.concatenate([np.repeat(prefix[None], n, 0), own], 1)
    extra = rng.integers(0, 40, size=n)
    Q = wl.to_bf16_bits(rng.standard_normal((n, q, Hq, D), dtype=np.float32))
    O, lse = pg.verify(hip.to_device(Q), hip.i32(tables), hip.i32(blocks * P + extra), hip.i32([q] * n), hip.i32([0] * n), hip.i32([blocks * P]))
    assert int(pg.plan[:8].cpu().numpy().view(np.int32)[1]) == n + 1 and int(pg.status.item()) == 0
    O, lse = wl.bf16_bits_to_f32(hip.to_host(O)), hip.to_host(lse)
    for b in range(n):
        for i in range(q):
            tail = np.repeat(value[own[b]], P)[:extra[b] + i + 1]
            count = blocks * P + len(tail)
            mean, size = (P * value[prefix].sum() + tail.sum()) / count, (P * np.abs(value[prefix]).sum() + np.abs(tail).sum()) / count
            assert np.abs(lse[b, i] - np.log(count)).max() <= 2e-6
            assert np.abs(O[b, i] - mean).max() <= 2 ** -8 * abs(mean) + (2 ** -8 * size if dtype == "int8kv" else 1e-5)


def test_replayed_graph(hip):
    """Plan and two layers captured; every replay, with other lengths and eager work between, equals the eager call bit for bit."""
    import torch
    import paper_2404_15778_amd as bass
    rng = np.random.default_rng(9)
    n = 16
    batch = Batch(31, 32, 8, 128, 64, [2048 + 300] * n, [4] * n, 4, np.zeros(n, int), [2048])
    pg = batch.pages(hip)
    ctx, nq, of, plen, tables = (hip.i32(x) for x in (batch.ctx, batch.nq, batch.of, batch.plen, batch.tables))
    Q = hip.to_device(batch.Q)

    def step(plan, ws, O, lse):
        bass.bass_paged_attention_plan(pg.desc, ctx, nq, of, plen, plan, pg.status)
        for l in range(2):
            bass.bass_paged_verify_attention(pg.desc, Q, pg.K, pg.V, tables, plan, O[l], lse[l], ws, pg.status)

    new = lambda: ([torch.empty_like(pg.O) for _ in range(2)], [torch.empty_like(pg.lse) for _ in range(2)])  # noqa: E731
    (O1, l1), (O2, l2) = new(), new()
    ws2, plan2 = bass.alloc_paged_workspace(pg.desc), bass.alloc_paged_plan(pg.desc)
    step(pg.plan, pg.ws, O1, l1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pg.plan, pg.ws, O1, l1)
    for _ in range(4):
        ctx.copy_(torch.tensor(2048 + rng.integers(0, 290, size=n), dtype=torch.int32))
        nq.copy_(torch.tensor(rng.integers(0, 5, size=n), dtype=torch.int32))
        for x in O1 + l1:
            x.fill_(float("nan"))
        graph.replay()
        step(plan2, ws2, O2, l2)
        torch.cuda.synchronize()
        for a, b in zip(O1 + l1, O2 + l2):
            assert torch.equal(a, b)
    assert int(pg.status.item()) == 0


def test_two_streams_at_once(hip):
    """Two batches on streams of their own, with workspaces of their own and one plan."""
    import torch
    import paper_2404_15778_amd as bass
    n = 16
    batch = Batch(41, 32, 8, 128, 64, [2048 + 100] * n, [4] * n, 4, np.zeros(n, int), [2048])
    pg = batch.pages(hip)
    Q = [hip.to_device(batch.Q), hip.to_device(batch.Q[::-1])]
    tables = [hip.i32(batch.tables), hip.i32(batch.tables[::-1].copy())]
    want = [pg.verify(Q[k], tables[k], hip.i32(batch.ctx), hip.i32(batch.nq), hip.i32(batch.of), hip.i32(batch.plen))[0].clone() for k in range(2)]
    O = pg.O
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(O) for _ in range(5)] for _ in range(2)]
    ws = [bass.alloc_paged_workspace(pg.desc) for _ in range(2)]
    torch.cuda.synchronize()
    for r in range(5):
        for k in range(2):
            bass.bass_paged_verify_attention(pg.desc, Q[k], pg.K, pg.V, tables[k], pg.plan, outs[k][r], None, ws[k], pg.status, streams[k])
    torch.cuda.synchronize()
    for k in range(2):
        for r in range(5):
            assert torch.equal(outs[k][r], want[k])


def test_tensors_of_the_wrong_kind_are_refused(hip):
    import torch
    import paper_2404_15778_amd as bass
    batch = Batch(51, 4, 2, 64, 32, [40, 50], [1, 2], 2)
    pg = batch.pages(hip)
    Q, t = hip.to_device(batch.Q), hip.i32(batch.tables)
    good = dict(Q=Q, Kpool=pg.K, Vpool=pg.V, tables=t, plan=pg.plan, O=pg.O, lse=pg.lse, workspace=pg.ws)
    bad = dict(Q=Q.float(), Kpool=pg.K[:-16], Vpool=pg.V.cpu(), tables=t.long(), plan=pg.plan[:64], O=pg.O.float(), lse=pg.lse[:1], workspace=None)
    for name, x in bad.items():
        with pytest.raises(ValueError):
            bass.bass_paged_verify_attention(pg.desc, **{**good, name: x})
    with pytest.raises(ValueError):
        bass.bass_paged_verify_attention(pg.desc, **{**good, "Q": Q.transpose(0, 1).contiguous().transpose(0, 1)})
    with pytest.raises(bass.BassError):
        bass.bass_paged_verify_attention(pg.desc, **{**good, "workspace": pg.ws[:64]})
    assert torch.isnan(pg.O.float()).all()


def test_steps_of_a_server(hip):
    """The operators together: requests that begin with a held prompt, tables, slots, rows appended, attention; drafts that are taken back, requests
    that end and places that are taken again, over a pool that is just large enough."""
    import torch
    import paper_2404_15778_amd as bass
    rng = np.random.default_rng(12)
    B, kmax, Hq, Hkv, D, P, most, n_pages = 6, 5, 8, 4, 64, 32, 12, 44
    prompt = 5 * P + 7
    pg = hip.DevicePages(B, kmax, Hq, Hkv, D, P, n_pages, most, "bf16", 0.125, poison=True)
    dt = hip.DeviceTables(B + 1, most, P, n_pages)   # the last row holds the prompt
    tables = dt.tables[:B]
    draw = lambda *s: wl.to_bf16_bits(rng.standard_normal(s, dtype=np.float32))  # noqa: E731
    pk, pv = draw(1, prompt, Hkv, D), draw(1, prompt, Hkv, D)
    none = [0] * B
    slots = dt.update(none + [prompt], ctx_len=none + [0], n_new=none + [prompt], kmax=prompt)
    pg.append(hip.to_device(pk), hip.to_device(pv), slots[B:].contiguous())
    whole = prompt // P * P                          # what can be shared
    K, V = np.zeros((B, most * P, Hkv, D), np.uint16), np.zeros((B, most * P, Hkv, D), np.uint16)
    ctx = np.zeros(B, int)                           # 0: the place is empty
    for step in range(12):
        begin = [b for b in range(B) if ctx[b] == 0 and (step == 0 or rng.random() < 0.6)]
        new = np.zeros(B, int)
        for b in range(B):
            if b in begin:
                K[b, :whole], V[b, :whole] = pk[0, :whole], pv[0, :whole]
                ctx[b] = whole
            if ctx[b]:
                new[b] = rng.integers(1, kmax + 1)
        share = [B if b in begin else -1 for b in range(B)] + [-1]
        slots = dt.update((ctx + new).tolist() + [prompt], share, [prompt] * (B + 1), ctx.tolist() + [0], new.tolist() + [0], kmax)
        rows = [draw(B, kmax, Hkv, D) for _ in range(2)]
        pg.append(hip.to_device(rows[0]), hip.to_device(rows[1]), slots[:B].contiguous())
        for b in range(B):
            K[b, ctx[b]:ctx[b] + new[b]], V[b, ctx[b]:ctx[b] + new[b]] = rows[0][b, :new[b]], rows[1][b, :new[b]]
        Q = draw(B, kmax, Hq, D)
        O, lse = pg.verify(hip.to_device(Q), tables, hip.i32(ctx), hip.i32(new), hip.i32(np.where(ctx > 0, 0, -1)), hip.i32([whole]))
        f = [wl.bf16_bits_to_f32(x) for x in (Q, K, V)]
        Or, lser = oracle.verify_attention(*f, ctx, new, 0.125)
        A, _ = oracle.verify_attention(f[0], f[1], np.abs(f[2]), ctx, new, 0.125)
        got = wl.bf16_bits_to_f32(hip.to_host(O))
        assert (np.abs(got - Or) <= (2 ** -8 * (1 + 2 ** -8) + 2 ** -10) * A + 2 ** -8 * np.abs(Or) + 1e-30).all(), step
        for b in range(B):
            if ctx[b]:
                ctx[b] += rng.integers(0, new[b] + 1)  # the others are taken back: written over by the next step
                if rng.random() < 0.2 or ctx[b] + kmax > most * P:
                    ctx[b] = 0
    assert int(pg.status.item()) == 0 and int(dt.status.item()) == 0
    dt.update([0] * (B + 1))
    assert not dt.refs.any() and not dt.held.any() and (dt.tables == -1).all()
    assert bass.STATUS_NO_PAGES == 32 and torch.cuda.is_available()
