"""Attention over paged caches where the plan does compute prefixes for all of their sequences together, which each test asserts: several prefixes at once in
every form that a shared run has (rows of at most 32, tiles of up to 128 and of 256 rows, several tiles), their members in any order among sequences without one
and places that are not in use, in both planning kernels; and windows of page numbers that follow one another.

Bounds of errors as derived in test_gpu_paged_attention."""
import numpy as np
import pytest

import oracle
import workloads as wl
from oracle.kv_int8 import dequantize_rows, quantize_rows
from test_gpu_paged_attention import Batch, quantize_queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hip():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2404_15778_amd import harness
    return harness


def shared_runs(pg):
    """Of every shared run: (query rows of a tile, tiles, common blocks), smallest tiles first."""
    words = pg.plan.cpu().numpy().view(np.int32)
    runs = words[16 + 24 * 256:][:16 * words[1]].reshape(-1, 16)
    g = pg.desc.Hq // pg.desc.Hkv
    return sorted((int(r[3] * g), int(r[4]), int(r[6])) for r in runs if r[7] < 0)


def form(rows, tiles):
    """How a shared run of such tiles is computed: 0 rows of at most 32, 1 and 2 tiles of up to 128 and 256 rows, 3 several tiles."""
    return 3 if tiles > 1 else 0 if rows <= 32 else 1 if rows <= 128 else 2


def batch_of(seed, Hq, Hkv, D, P, q, prefixes, alone, dtype, scale=None, longest=90):
    """prefixes: (members, tokens) of each.  One more member of each has no query tokens, and one at the end no tokens either: neither counts."""
    rng = np.random.default_rng(seed)
    of = np.concatenate([np.repeat(np.arange(len(prefixes)), [m + 1 for m, _ in prefixes]), np.full(alone, -1)])
    plen = np.array([n for _, n in prefixes])
    nq = rng.integers(q - 1, q + 1, size=len(of))
    idle = np.cumsum([m + 1 for m, _ in prefixes]) - 1
    nq[idle] = 0
    ctx = np.where(of >= 0, plen[of], 0) + rng.integers(0, longest, size=len(of))
    order = rng.permutation(len(of))
    of, nq, ctx = (np.append(x[order], extra) for x, extra in ((of, np.arange(len(prefixes))), (nq, [0] * len(prefixes)), (ctx, [0] * len(prefixes))))
    return Batch(seed, Hq, Hkv, D, P, ctx, nq, q, of, plen, dtype, scale)


# heads, kv heads, head size, tokens of a page, query tokens, (members, tokens) of every prefix, sequences without one, forms of the shared runs
SEVERAL = [(32, 16, 64, 32, 2, [(4, 544), (4, 704), (4, 900)], 3, [0, 0, 0]),
           (32, 8, 128, 64, 4, [(6, 1600), (6, 1920)], 4, [1, 1]),
           (32, 8, 64, 32, 4, [(12, 900), (12, 1300)], 3, [2, 2]),
           (32, 8, 128, 32, 4, [(40, 330), (38, 480)], 2, [3, 3]),
           (32, 8, 128, 96, 4, [(2, 3264), (6, 1248), (14, 768)], 5, [0, 1, 2]),
           (8, 4, 64, 32, 2, [(8, 960), (30, 300), (60, 200), (150, 130)], 11, [0, 1, 2, 3])]  # more than the small planning kernel takes


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("Hq,Hkv,D,P,q,prefixes,alone,forms", SEVERAL)
def test_several_prefixes_at_once(hip, dtype, Hq, Hkv, D, P, q, prefixes, alone, forms):
    batch = batch_of(len(prefixes) * 100 + D + P, Hq, Hkv, D, P, q, prefixes, alone, dtype)
    assert (batch.B + len(prefixes) > 256) == (len(prefixes) == 4)
    pg = batch.pages(hip)
    batch.check(hip, pg=pg)
    assert sorted(form(rows, tiles) for rows, tiles, _ in shared_runs(pg)) == forms
    assert sorted(n for _, _, n in shared_runs(pg)) == sorted(n // 32 for _, n in prefixes)


# heads, kv heads, query tokens, members, tokens of the prefix: one for each form
ONE = [(32, 16, 2, 6, 640), (32, 8, 4, 7, 3200), (32, 8, 4, 14, 1600), (32, 8, 4, 40, 640)]


def one(i, dtype, scale=None, D=128, seed=0):
    Hq, Hkv, q, n, P = ONE[i]
    rng = np.random.default_rng([i, seed])
    return Batch(i + 10 * seed, Hq, Hkv, D, 32, P + rng.integers(0, 60, size=n), np.full(n, q), q, np.zeros(n, int), [P], dtype, scale)


def assert_form(pg, i):
    assert [form(rows, tiles) for rows, tiles, _ in shared_runs(pg)] == [i]


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("i", range(4))
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(hip, dtype, i, scale):
    """Inputs an eighth as large, so that the products stay below 64 together."""
    batch = one(i, dtype, scale)
    batch.Q = wl.to_bf16_bits(wl.bf16_bits_to_f32(batch.Q) / 16)
    pg = batch.pages(hip)
    batch.check(hip, pg=pg)
    assert_form(pg, i)


@pytest.mark.parametrize("i", range(4))
def test_together_and_apart(hip, i):
    """The same batch with its prefix named and not: both within their bounds, so no further apart than twice those; and lse is left alone where it is not asked for."""
    batch = one(i, "bf16")
    pg = batch.pages(hip)
    a, la = batch.check(hip, pg=pg)
    assert_form(pg, i)
    pg.lse.fill_(float("nan"))
    again, _, status = batch.run(hip, pg, want_lse=False)
    assert status == 0 and np.array_equal(a, again) and bool(pg.lse.isnan().all())
    b, lb = batch.check(hip, pg=pg, share=False)
    assert shared_runs(pg) == []
    _, _, A = batch.reference()
    assert (np.abs(a - b) <= 2 * (2 ** -8 * (1 + 2 ** -8) + 2 ** -10) * A + 2 ** -7 * np.maximum(np.abs(a), np.abs(b)) + 1e-30).all()
    assert np.abs(la - lb).max() <= 2 ** -10 + 2 ** -19 * np.abs(la).max()


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("i", range(4))
def test_what_is_common_ends_with_the_shortest_sequence(hip, dtype, i):
    """A prefix that reaches beyond some sequences, whose tokens are not whole blocks: the rest goes by itself."""
    Hq, Hkv, q, n, P = ONE[i]
    rng = np.random.default_rng(i)
    ctx = P + 45 + rng.integers(0, 200, size=n)
    ctx[n // 2] = P + 43
    batch = Batch(70 + i, Hq, Hkv, 64, 32, ctx, np.full(n, q), q, np.zeros(n, int), [P + 150], dtype)
    pg = batch.pages(hip)
    batch.check(hip, pg=pg)
    assert_form(pg, i)
    assert shared_runs(pg)[0][2] == P // 32 + 1


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("i", range(4))
def test_every_token_counts_once(hip, dtype, i):
    """Keys of zero: lse is the logarithm of the number of visible tokens."""
    batch = one(i, dtype, seed=3)
    batch.K[:] = 0
    pg = batch.pages(hip)
    O, lse = batch.check(hip, pg=pg)
    assert_form(pg, i)
    seen = batch.ctx[:, None] + np.arange(batch.kmax) + 1
    assert np.abs(lse - np.log(seen)[:, :, None]).max() <= 2e-6


# Sequences of one prefix and heads that make tiles of 96 and of 240 query rows, and of 24 (no tile)
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("int8kv", 128), ("int8kv", 64)])
@pytest.mark.parametrize("n,Hq,Hkv,rows", [(16, 32, 16, 96), (40, 16, 8, 240), (4, 16, 8, 24)])
def test_windows_of_page_numbers(hip, dtype, D, n, Hq, Hkv, rows):
    """More than two windows of 64 page numbers per workgroup (a window of a wavefront: four times as many blocks), with keys and values of every block
    its own.  The prefix is made of few pages in random order, so that the reference is a sum over those pages with the numbers of their uses.  (Here products are at most 25 together, and a lane adds up 2400 terms: 2^-12.3 + 2^-12.8 in lse.)"""
    rng = np.random.default_rng([n, D])
    P, q, unique = 32, 3, 90
    shares = 256 // Hkv
    blocks = shares * (150 if rows > 32 else 4 * 150) + 11
    pages = unique + n
    pg = hip.DevicePages(n, q, Hq, Hkv, D, P, pages, blocks + 1, dtype, 1.0 / np.sqrt(D), poison=True)
    K, V = (wl.to_bf16_bits(rng.standard_normal((pages * P, Hkv, D), dtype=np.float32) * rng.uniform(0.5, 1.5, size=(pages * P, Hkv, 1)).astype(np.float32)) for _ in range(2))
    pg.append(hip.to_device(K[None]), hip.to_device(V[None]), hip.i32(np.arange(pages * P)[None]))
    # the first half uses the first pages twice as often as the others, the second half the last ones
    odds = np.repeat([2.0, 1.0], unique // 2)
    prefix = np.concatenate([rng.choice(unique, size=blocks // 2, p=odds / odds.sum()), rng.choice(unique, size=blocks - blocks // 2, p=odds[::-1] / odds.sum())])
    tables = np.concatenate([np.repeat(prefix[None], n, 0), unique + rng.permutation(n)[:, None]], 1)
    extra = rng.integers(0, P - q, size=n)
    Q = wl.to_bf16_bits(2 * rng.standard_normal((n, q, Hq, D), dtype=np.float32))
    ctx = blocks * P + extra
    O, lse = pg.verify(hip.to_device(Q), hip.i32(tables), hip.i32(ctx), hip.i32([q] * n), hip.i32([0] * n), hip.i32([blocks * P]))
    assert int(pg.status.item()) == 0 and shared_runs(pg) == [(rows, 1, blocks)]
    O, lse = wl.bf16_bits_to_f32(hip.to_host(O)).astype(np.float64), hip.to_host(lse)
    f = [wl.bf16_bits_to_f32(x) for x in (Q, K, V)]
    if dtype == "int8kv":
        f = [dequantize_rows(*quantizer(x)) for quantizer, x in zip((quantize_queries, quantize_rows, quantize_rows), f)]
    Qf, Kf, Vf = (x.astype(np.float64) for x in f)

    def reference(uses, b, i, h):
        """lse, O and A of row (b, i, h) where the prefix's pages are used so often."""
        count = np.append(np.repeat(uses, P), np.repeat(np.arange(n) == tables[b, -1] - unique, P) * (np.arange(n * P) % P < extra[b] + i + 1))
        s = Kf[:, h // (Hq // Hkv)] @ Qf[b, i, h] / np.sqrt(D)
        m = s[count > 0].max()
        w = count * np.exp(s - m)
        v = Vf[:, h // (Hq // Hkv)]
        return m + np.log(w.sum()), w @ v / w.sum(), w @ np.abs(v) / w.sum()

    uses = np.bincount(prefix, minlength=unique)
    twice = np.bincount(prefix[:blocks // 2], minlength=unique) * 2  # the first half read again in place of the second
    told = 0
    for b in rng.choice(n, size=4, replace=False):
        for i in range(q):
            for h in range(Hq):
                want_lse, want, A = reference(uses, b, i, h)
                assert abs(lse[b, i, h] - want_lse) <= 2 ** -11 + 2 ** -20 * abs(want_lse)
                assert (np.abs(O[b, i, h] - want) <= (2 ** -8 * (1 + 2 ** -8) + 2 ** -10) * A + 2 ** -8 * np.abs(want)).all()
                told += abs(reference(twice, b, i, h)[0] - want_lse) > 2 ** -10 + 2 ** -19 * abs(want_lse)
    assert told > 2 * q * Hq  # that mistake would show in most rows


@pytest.mark.parametrize("i", [None, 0, 1, 2, 3])
@pytest.mark.parametrize("D", [64, 128])
def test_int8_pages_and_caches_of_their_own(hip, i, D):
    """The same rows in INT8 pages and in INT8 caches per sequence.  Queries are whole multiples of 2^-5 of up to 127, so that both quantizers give the multiples
    themselves; scores are then products of the same whole numbers and of scales that are rounded four times each way: 8 2^-24 of 24 at most.  A sum is at most 1664
    additions one after the other (a whole context by one lane), half of that many half steps on average.  Both sides: 2 (192 + 832) 2^-24 = 2^-13, where one other
    code of a query moves lse by about 2^-9.  O: probabilities to bf16 on both sides, the paged result too."""
    Hq, Hkv, q, n, P = ONE[i or 0]
    rng = np.random.default_rng([i or 0, D])
    ctx = (P if i is not None else 40) + rng.integers(0, 70, size=n)
    batch = Batch(5, Hq, Hkv, D, 32, ctx, np.full(n, q), q, np.zeros(n, int), [P], "int8kv")
    codes = np.clip(np.rint(rng.standard_normal((n, q, Hq, D)) * 32), -127, 127)
    codes[..., 3] = rng.choice([-127, 127], size=codes.shape[:3])
    batch.Q = wl.to_bf16_bits((codes / 32).astype(np.float32))
    for quantizer in (quantize_queries, quantize_rows):
        assert np.array_equal(quantizer(wl.bf16_bits_to_f32(batch.Q))[0], codes)
    pg = batch.pages(hip)
    O, lse = batch.check(hip, pg=pg)
    assert [form(rows, tiles) for rows, tiles, _ in shared_runs(pg)] == ([] if i is None else [i])
    T = int((ctx + q).max())
    da = hip.DeviceAttention(n, q, Hq, Hkv, D, T, "int8kv", batch.scale)
    da.append(hip.to_device(batch.K[:, :T]), hip.to_device(batch.V[:, :T]), hip.i32([0] * n), hip.i32(ctx + q))
    Oc, lsec = (hip.to_host(x) for x in da.verify(hip.to_device(batch.Q), hip.i32(ctx), hip.i32(batch.nq)))
    _, want_lse, A = batch.reference()
    assert np.abs(want_lse).max() < 24 and int(da.status.item()) == 0
    assert np.abs(lse - lsec).max() <= 2 ** -13
    assert (np.abs(O - Oc) <= (2 * 2 ** -8 + 2 ** -14) * A + 2 ** -8 * np.abs(Oc)).all()


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("i", [None, 0, 1, 2])
def test_pools_beyond_four_gigabytes(hip, dtype, i):
    """All pages behind the first 2^32 bytes of a pool, in every form, apart and together."""
    batch = one(i or 0, dtype, seed=5)
    page = 32 * batch.Hkv * (batch.D + 4 if dtype == "int8kv" else 2 * batch.D)
    front = 2 ** 32 // page + 1
    batch.tables[batch.tables >= 0] += front
    batch.n_pages += front
    pg = batch.pages(hip)
    assert pg.K.numel() > 2 ** 32 + 100 * page
    batch.check(hip, pg=pg, share=i is not None)
    assert [form(rows, tiles) for rows, tiles, _ in shared_runs(pg)] == ([] if i is None else [i])
