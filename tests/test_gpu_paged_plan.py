"""The plan of the attention over paged caches by itself, as the device made it: its runs, its list and the division of the list, in whole numbers of
any size.  What the launches that read it rely on: the list is the units laid end to end, the shares are the list, every share between the first and the last one of
a unit has a block of that unit (the merge reads a partial result of each), and every sequence's blocks are there once."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
WAVES, SHARES = 4, 256


@pytest.fixture(scope="module")
def hip():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2404_15778_amd import harness
    return harness


def make_plan(hip, desc, ctx, nq, of=None, plen=None):
    """(bytes of the plan, status)"""
    import torch
    import paper_2404_15778_amd as bass
    plan, status = bass.alloc_paged_plan(desc).fill_(0xA5), torch.zeros(1, dtype=torch.int32, device="cuda")
    up = lambda x: None if x is None else hip.i32(x)  # noqa: E731
    bass.bass_paged_attention_plan(desc, up(ctx), up(nq), up(of), up(plen), plan, status)
    return plan.cpu().numpy(), int(status.item())


def check_plan(plan, desc, ctx, nq, of=None, plen=None):
    """Returns the numbers of shared runs and of shares in use."""
    words = plan.view(np.int32)
    n_runs, total, per, rem, used = (int(x) for x in words[1:6])
    shares = words[16:16 + 24 * SHARES].reshape(SHARES, 24).astype(np.int64)
    at = 16 + 24 * SHARES
    runs = words[at:at + 16 * n_runs].reshape(n_runs, 16).astype(np.int64)
    row, tok, n_tok, tile_tok, n_tiles, first, n_blk, L, start, row_base, whole, cost, pad, heads = runs.T[:14]
    g, live = desc.Hq // desc.Hkv, np.flatnonzero(nq > 0)
    entries, units = n_blk * cost + pad, (desc.Hkv + heads - 1) // heads * n_tiles
    # the list
    ends = np.cumsum(units * entries)
    assert (n_runs, total) == (n_runs, int(ends[-1]) if n_runs else 0) and total < 2 ** 31
    assert np.array_equal(start, ends - units * entries)
    assert np.array_equal(row_base, np.cumsum(n_tok * desc.Hq) - n_tok * desc.Hq)
    assert (n_tiles == (n_tok + tile_tok - 1) // tile_tok).all() and (n_blk > 0).all() and (tile_tok * g <= 256).all()
    # its division
    assert (per, rem) == (total // used, total % used) and 1 <= used <= SHARES
    cut = np.minimum(np.arange(SHARES + 1) * per + np.minimum(np.arange(SHARES + 1), rem), total)
    assert np.array_equal(shares[:, 4], np.diff(cut))
    for w in range(used if total else 0):
        a, b = cut[w], cut[w + 1]
        r = int(np.searchsorted(start, a, side="right")) - 1
        assert (shares[w, 1], shares[w, 2], shares[w, 3]) == (r, (a - start[r]) // entries[r], (a - start[r]) % entries[r])
        assert np.array_equal(shares[w, 8:22], runs[r, :14])
        if shares[w, 3] + b - a <= n_blk[r] * cost[r]:  # nothing but blocks of one unit
            assert -(-shares[w, 3] // cost[r]) < -(-(shares[w, 3] + b - a) // cost[r])
    # the sequences' blocks: those of a shared run, and the rest
    shared = np.flatnonzero(L < 0)
    assert np.array_equal(shared, np.arange(len(shared)))
    own = runs[len(shared):]
    assert np.array_equal(own[:, 0], live) and np.array_equal(own[:, 7], ctx[live]) and np.array_equal(own[:, 2], nq[live])
    assert np.array_equal(own[:, 5] + own[:, 6], (ctx[live] + nq[live] + 31) // 32)
    common = {}
    for i in shared:
        prefix = of[row[i]]
        members = live[of[live] == prefix]
        assert row[i] == members[0] and n_tok[i] == nq[members].sum() and len(members) >= 2
        assert n_blk[i] == min(plen[prefix], ctx[members].min()) // 32
        common[prefix] = n_blk[i]
    assert np.array_equal(own[:, 5], [common.get(-1 if of is None else of[b], 0) for b in live])
    assert np.array_equal(own[:, 10], own[:, 5] == 0)
    return len(shared), used


def lengths(rng, B, kmax, prefixes, most, longest):
    """Random sequences, a third without a prefix."""
    of = rng.integers(-(prefixes + 1) // 2, prefixes, size=B) if prefixes else None
    plen = rng.integers(0, most, size=prefixes) if prefixes else None
    ctx = rng.integers(0, longest + 1, size=B)
    if prefixes:
        of = np.maximum(of, -1)
        ctx = ctx + np.where(of >= 0, plen[of], 0)
    return ctx, rng.integers(0, kmax + 1, size=B), of, plen


# sequences, slots, heads, kv heads, prefixes, tokens of a prefix and of a sequence's own: short lists, whose shares are as small as they get, and longer ones;
# both planning kernels
SHAPES = [(1, 1, 1, 1, 0, 0, 40), (2, 1, 4, 4, 0, 0, 90), (3, 4, 8, 2, 1, 90000, 64), (8, 7, 32, 32, 1, 3000, 300), (12, 5, 64, 8, 2, 25000, 40),
          (24, 8, 64, 8, 3, 9000, 100), (40, 4, 32, 8, 2, 6000, 64), (64, 4, 10, 5, 1, 6000, 250), (200, 3, 6, 2, 20, 3000, 200), (300, 2, 64, 4, 9, 5000, 60)]


@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("B,kmax,Hq,Hkv,prefixes,most,longest", SHAPES)
def test_random_batches(hip, dtype, B, kmax, Hq, Hkv, prefixes, most, longest):
    import paper_2404_15778_amd as bass
    rng = np.random.default_rng([B, kmax, Hkv])
    desc = bass.make_paged_desc(B, kmax, Hq, Hkv, 128, 32, 1000, 3000, dtype, 0.1)
    seen = []
    for _ in range(25):
        top = max(1, int(most * rng.random() ** 2))
        ctx, nq, of, plen = lengths(rng, B, kmax, prefixes, top + 1, int(longest * rng.random()))
        plan, status = make_plan(hip, desc, ctx, nq, of, plen)
        assert status == 0
        seen.append(check_plan(plan, desc, ctx, nq, of, plen))
    assert max(n for n, _ in seen) >= min(prefixes, 2)  # some of them share prefixes, two at once where there are several
    assert B > 12 or min(used for _, used in seen) < SHARES  # short lists


# sequences, slots, heads, kv heads, tokens of a page, entries of a table: the largest lists that shapes are accepted for
@pytest.mark.parametrize("dtype", ["bf16", "int8kv"])
@pytest.mark.parametrize("shared", [0, 1, 5])
@pytest.mark.parametrize("B,kmax,Hq,Hkv,P,most", [(1000, 1, 32, 32, 32, 2048), (4096, 1, 8, 8, 32, 8159), (4032, 8, 256, 32, 32, 2047), (2, 16, 8, 2, 64, 33554399), (250, 7, 27, 3, 256, 44699)])
def test_the_largest_lists(hip, dtype, shared, B, kmax, Hq, Hkv, P, most):
    """Full tables with as many query tokens as there may be; nothing shared, one prefix of nearly everything, and five of different lengths."""
    import paper_2404_15778_amd as bass
    desc = bass.make_paged_desc(B, kmax, Hq, Hkv, 64, P, 100, most, dtype, 0.1)
    assert bass.bass_paged_attention_plan_bytes(desc) > 0
    rng = np.random.default_rng(B)
    nq = np.full(B, kmax)
    ctx = most * P - kmax - rng.integers(0, 200, size=B)
    of = np.arange(B) % shared if shared else None
    plen = most * P // np.arange(1, shared + 1) - 1000 if shared else None
    plan, status = make_plan(hip, desc, ctx, nq, of, plen)
    assert status == 0
    runs, used = check_plan(plan, desc, ctx, nq, of, plen)
    assert runs == (shared if B > 5 or shared == 1 else 0) and used == SHARES
