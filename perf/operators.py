"""Paged KV caches with shared prefixes: what a program that serves batched speculative sampling asks of them, as cases to be timed.

Several answers to one prompt, or many users behind one system prompt, hold the same first tokens.  Their keys and values
are kept once, in pages that the sequences' tables share, and a step's attention reads them once for all.  A case's `op` says
which operator one pass goes through:

  tables  pages taken, shared and given back for the lengths of a step, and the slots of the step's new tokens (bass_page_tables)
  write   keys and values of new tokens written into the pages by slot (bass_paged_append)
  read    keys and values of sequences read back through their tables (bass_paged_gather)
  attend  verification attention of a step over the pages, shared prefixes computed once for all sequences that begin with
          them: one plan (bass_paged_attention_plan) and one call (bass_paged_verify_attention) per layer

A pool holds pages of `page` tokens, [page][kv head][page / 32] blocks of 32 tokens; how a block is laid out is written at _K_BLOCK below.
Where `own` is false a pass computes the same in elementary torch operations, in 32 bits, rounded once at the end.
Lengths belong to the case (they follow from its `lens` number, so that work() knows them); tensors are drawn from the seed.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

DEV = "cuda:0"
BLOCK = 32  # tokens of a block


def _attend(name, **kw):
    c = {"name": name, "op": "attend", "kv": "bf16", "B": 8, "kmax": 6, "q_lo": 1, "Hq": 32, "Hkv": 32, "D": 128, "page": 64, "prefixes": 1,
         "with_prefix": 8, "prefix_lo": 1024, "prefix_hi": 1024, "own_lo": 16, "own_hi": 512, "layers": 4, "lens": 1}
    c.update(kw)
    return c


def _rows(name, op, **kw):
    c = {"name": name, "op": op, "B": 8, "kmax": 6, "Hkv": 32, "D": 128, "page": 64, "ctx_lo": 512, "ctx_hi": 2048, "layers": 4, "lens": 1}
    c.update(kw)
    return c


def _tables(name, **kw):
    c = {"name": name, "op": "tables", "rows": 16, "prefixes": 1, "page": 64, "pages": 1024, "max_pages": 64, "kmax": 6, "lens": 1}
    c.update(kw)
    return c


def listed():
    return [
        # A step of a small server: 16 requests, one system prompt, a few pages change hands.  Latency and launches.
        _tables("tables_16"),
        # A large server: a thousand requests with up to 65536 tokens each, some ending, some beginning, a quarter of a million pages.
        _tables("tables_1000", rows=1000, prefixes=7, page=32, pages=250007, max_pages=2048, kmax=8),
        # The new rows of a step: 8 sequences, up to 6 tokens each.
        _rows("write_step_b8", "write"),
        # Prompts of up to 2000 tokens written page by page.
        _rows("write_prompts_b8", "write", kmax=2000, ctx_lo=0, ctx_hi=0),
        # The last 64 tokens of 24 sequences read back (a window for a draft model), odd page size.
        _rows("read_window_b24", "read", B=24, kmax=64, Hkv=8, page=96, layers=1),
        # Whole sequences read back to be moved to another place.
        _rows("read_prompts_b8", "read", kmax=2000, ctx_lo=0, ctx_hi=0),
        # The smallest call: two short sequences, one token each, 4 heads of 64, nothing shared.  Latency.
        _attend("attend_decode_b2", B=2, kmax=1, Hq=4, Hkv=4, D=64, page=32, prefixes=0, with_prefix=0, own_lo=1, own_hi=90, layers=1),
        # The paper's use: 8 answers to one prompt at a time, each with its own drafts.  32 heads, nothing grouped.
        _attend("attend_answers_b8", kmax=7, prefix_lo=1500, prefix_hi=1500),
        # Many users behind three system prompts, some without one; grouped-query heads.
        _attend("attend_prompts_gqa_b32", B=32, kmax=5, Hq=64, Hkv=8, prefixes=3, with_prefix=26, prefix_lo=1000, prefix_hi=8000, own_lo=32,
                own_hi=2048),
        # A long document and 64 questions about it: 2048 query rows per kv head see the same 16384 tokens.  Bound by arithmetic.
        _attend("attend_document_b64", B=64, kmax=8, q_lo=8, Hq=32, Hkv=8, page=128, with_prefix=64, prefix_lo=16384, prefix_hi=16384, own_lo=100,
                own_hi=400, layers=2),
        # Nothing shared: ragged lengths over small pages, as left behind by sequences that came and went.
        _attend("attend_ragged_b16", B=16, kmax=4, Hq=32, Hkv=8, page=32, prefixes=0, with_prefix=0, own_lo=128, own_hi=8192),
        # INT8 pages, one token each (no drafts), a system prompt of 4096 tokens.
        _attend("attend_prompt_int8_b24", kv="int8kv", B=24, kmax=1, Hq=64, Hkv=8, with_prefix=24, prefix_lo=4096, prefix_hi=4096, own_lo=64,
                own_hi=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(("attend", "tables", "write", "read"), (12, 3, 3, 3))[0]
    lens = rng.randrange(1 << 20)
    if op == "tables":
        rows, page = _log_int(rng, 1, 1024), rng.choice((32, 64, 96, 256))
        max_pages = _log_int(rng, 16, 2048)
        c = _tables("", rows=rows, prefixes=rng.randint(0, min(8, rows - 1)), page=page, max_pages=max_pages,
                    pages=max(_log_int(rng, 256, 262144), 2 * rows), kmax=rng.randint(1, 16), lens=lens)
    elif op in ("write", "read"):
        Hkv, D = rng.choice(((32, 128), (8, 128), (4, 128), (16, 64), (8, 64)))
        c = _rows("", op, B=_log_int(rng, 1, 48), kmax=_log_int(rng, 1, 2048), Hkv=Hkv, D=D, page=rng.choice((32, 64, 96, 128, 256)), lens=lens)
        c["ctx_hi"] = 0 if rng.random() < 0.4 else _log_int(rng, 1, 4096)
        c["ctx_lo"] = c["ctx_hi"] // rng.randint(1, 8)
        c["layers"] = max(1, min(4, int(5e8 / work(c)["bytes"])))
        while c["B"] > 1 and work(c)["bytes"] > 8e8:
            c["B"] //= 2
    else:
        Hq, Hkv, D = rng.choice(((32, 32, 128), (64, 8, 128), (32, 8, 128), (28, 4, 128), (24, 8, 128), (16, 16, 64), (32, 8, 64), (15, 5, 64)))
        B = _log_int(rng, 1, 64)
        c = _attend("", kv=rng.choice(("bf16", "bf16", "int8kv")), B=B, kmax=_log_int(rng, 1, min(16, 64 * Hkv // Hq)), Hq=Hq, Hkv=Hkv, D=D,
                    page=rng.choice((32, 32, 64, 96, 128, 256)), lens=lens)
        c["q_lo"] = rng.randint(1, c["kmax"])
        c["with_prefix"] = rng.choice((0, rng.randint(0, B), B, B))
        c["prefixes"] = 0 if c["with_prefix"] == 0 else rng.choice((1, 1, rng.randint(1, min(4, c["with_prefix"]))))
        c["prefix_hi"] = _log_int(rng, 64, 16384)
        c["prefix_lo"] = max(1, c["prefix_hi"] // rng.randint(1, 4))
        c["own_hi"] = _log_int(rng, 1, 4096)
        c["own_lo"] = max(1, c["own_hi"] // rng.randint(1, 32))
        c["layers"] = 1
        # the plain form widens every sequence's whole context, and scores every row against it
        span = (c["prefix_hi"] if c["prefixes"] else 0) + c["own_hi"] + c["kmax"] + c["page"]
        while c["B"] > 1 and c["B"] * span * max(c["Hkv"] * c["D"], c["Hq"] * c["kmax"]) > 64 * 17000 * 1024:
            c["B"] //= 2
            c["with_prefix"] = min(c["with_prefix"], c["B"])
            c["prefixes"] = min(c["prefixes"], c["with_prefix"])
        c["layers"] = max(1, min(4, int(3e8 / work(c)["bytes"])))
    del c["name"]
    return c


# ---- lengths and tables ---------------------------------------------------------------------------

def _lengths(c):
    """attend: (prefix number of every sequence or -1, tokens of every prefix, cached tokens, query tokens)."""
    rng = np.random.default_rng([c["lens"], c["B"], c["own_hi"], c["kmax"]])
    B, G, P = c["B"], c["prefixes"], c["page"]
    plen = rng.integers(c["prefix_lo"], c["prefix_hi"] + 1, size=max(G, 1))[:G] // P * P  # whole pages are shared
    of = np.full(B, -1, np.int32)
    if G:
        members = rng.permutation(B)[: c["with_prefix"]]
        of[members] = np.concatenate([np.arange(G), rng.integers(0, G, size=len(members))])[: len(members)]
    mine = np.rint(np.exp(rng.uniform(math.log(c["own_lo"]), math.log(c["own_hi"]), size=B))).astype(np.int64)
    nq = rng.integers(min(c["q_lo"], c["kmax"]), c["kmax"] + 1, size=B).astype(np.int32)
    if B >= 8:
        nq[rng.integers(0, B)] = 0  # a place in the batch that is not in use
    ctx = mine + np.where(of >= 0, plen[of] if G else 0, 0)
    return of, plen.astype(np.int32), ctx.astype(np.int32), nq


def _page_rows(c, rng, lengths, prefix_of, prefix_len):
    """Tables for these lengths over pages in no order, as after sequences came and went: (tables, pages in the pool)."""
    P = c["page"]
    need = [-(-int(n) // P) for n in lengths]
    common = [int(n) // P for n in prefix_len]
    total = sum(common) + sum(n - (common[int(g)] if g >= 0 else 0) for n, g in zip(need, prefix_of))
    n_pages = total + total // 16 + 3
    ids = iter(rng.permutation(n_pages).tolist())
    first = [[next(ids) for _ in range(n)] for n in common]
    tables = np.full((len(need), max(need) + 1), -1, np.int32)
    for b, (n, g) in enumerate(zip(need, prefix_of)):
        head = first[int(g)] if g >= 0 else []
        tables[b, :n] = head + [next(ids) for _ in range(n - len(head))]
    return tables, n_pages


def _row_lengths(c):
    """write, read: (first token, number of tokens) of every sequence."""
    rng = np.random.default_rng([c["lens"], c["B"], c["kmax"], c["ctx_hi"]])
    n = rng.integers((c["kmax"] + 1) // 2, c["kmax"] + 1, size=c["B"])
    return rng.integers(c["ctx_lo"], c["ctx_hi"] + 1, size=c["B"]).astype(np.int32), n.astype(np.int32)


# ---- the layout of a block ------------------------------------------------------------------------
# bf16, 32 D elements.  K: [token / 16][d / 32][d / 8 % 4][token % 16][d % 8], V: [d / 16][token / 4 % 4][d % 16][token / 16][token % 4].
# INT8, 32 D codes and 32 scales (fp32).  K: [token / 16][d / 64][d / 16 % 4][token % 16][d % 16],
# V: [d / 32][token / 4 % 4][d % 16][d / 16 % 2][token / 16][token % 4].

def _K_BLOCK(D, int8):
    """Shape of a K block and the order of its axes that gives [token][d]."""
    return ((2, D // 64, 4, 16, 16), (0, 3, 1, 2, 4)) if int8 else ((2, D // 32, 4, 16, 8), (0, 3, 1, 2, 4))


def _V_BLOCK(D, int8):
    return ((D // 32, 4, 16, 2, 2, 4), (4, 1, 5, 0, 3, 2)) if int8 else ((D // 16, 4, 16, 2, 4), (3, 1, 4, 0, 2))


def _block_bytes(D, int8):
    return BLOCK * (D + 4) if int8 else BLOCK * D * 2


# ---- inputs ---------------------------------------------------------------------------------------

def _i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32, device=DEV)


def _randn(gen, shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _pool(c, gen, n_pages, int8):
    """One layer's K or V pages: values ~ N(0, 1), or what such values are quantized to."""
    shape, D = (n_pages, c["Hkv"], c["page"] // BLOCK), c["D"]
    if not int8:
        return _randn(gen, shape + (BLOCK * D,))
    raw = torch.empty(shape + (BLOCK * (D + 4),), dtype=torch.int8, device=DEV)
    amax = torch.rand(shape + (BLOCK,), generator=gen, device=DEV) * 1.5 + 2.0  # the largest of D values
    raw[..., : BLOCK * D] = torch.randn(shape + (BLOCK * D,), generator=gen, device=DEV).mul_(127.0 / 2.75).round_().clamp_(-127, 127).to(torch.int8)
    raw[..., BLOCK * D:] = (amax / 127.0).view(torch.int8)
    return raw


def _prepare_tables(c, seed):
    rng = np.random.default_rng(seed)
    R, G, P, N, M = c["rows"], c["prefixes"], c["page"], c["pages"], c["max_pages"]
    # rows 0 .. G - 1 hold the prefixes; the others are requests: most go on, some end, some begin in empty places
    top = max(1, min(M, N // R))
    have = np.rint(np.exp(rng.uniform(0.0, math.log(top), size=R))).astype(np.int64)
    have[G:][rng.random(R - G) < 0.1] = 0
    common = np.minimum(have[:G] // 2 + 1, have[:G])
    of = rng.integers(0, G, size=R) if G else np.full(R, -1)
    ids = rng.permutation(N)
    tables, refs, at = np.full((R, M), -1, np.int32), np.zeros(N, np.int32), 0
    for r in range(R):
        head = tables[of[r], : min(common[of[r]], have[r])] if G and r >= G else ids[:0]
        tables[r, : len(head)] = head
        tables[r, len(head): have[r]] = ids[at: at + have[r] - len(head)]
        at += have[r] - len(head)
    np.add.at(refs, tables[tables >= 0], 1)
    ctx = np.maximum(have * P - rng.integers(0, P, size=R), 0)
    ctx[have == 0] = 0
    n_new = rng.integers(1, c["kmax"] + 1, size=R)
    n_new[:G] = 0
    length, begin = ctx + n_new, np.full(R, -1, np.int32)
    fate = rng.random(R)
    fate[:G] = 1.0
    ends, starts = (have > 0) & (fate < 0.05), (have == 0) & (fate < 0.8)
    length[ends] = n_new[ends] = 0
    length[(have == 0) & ~starts] = n_new[(have == 0) & ~starts] = 0
    if G:
        begin[starts] = of[starts]
    share = np.where(begin >= 0, (common[of] if G else 0) * P + rng.integers(0, P, size=R), 0)
    ctx = np.where(starts, np.where(begin >= 0, share // P * P, 0), ctx)
    length = np.minimum(np.where(starts, ctx + n_new, length), M * P)
    s = SimpleNamespace(case=c, held=None, tables=None, refs=None)
    s.length, s.share_from, s.share_len, s.ctx, s.n_new = (_i32(x) for x in (length, begin, share, ctx, n_new))
    parts, at = [have, refs, tables.reshape(-1)], np.cumsum([0, R + -R % 64, N + -N % 64])
    s.before = _i32(np.concatenate([np.pad(x, (0, -len(x) % 64)) for x in parts]))
    s.now = torch.empty_like(s.before)
    s.held, s.refs, s.tables = (s.now[a: a + len(x)] for a, x in zip(at, parts))
    s.tables = s.tables.view(R, M)
    s.slots = torch.empty((R, c["kmax"]), dtype=torch.int32, device=DEV)
    s.scratch = torch.empty(4 * (R + N) + 65536, dtype=torch.uint8, device=DEV)
    s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def _prepare_rows(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    first, n = _row_lengths(c)
    tables, n_pages = _page_rows(c, np.random.default_rng(seed), first + n, np.full(c["B"], -1), [])
    s = SimpleNamespace(case=c, tables=_i32(tables), n_pages=n_pages, first=_i32(first), n=_i32(n), status=torch.zeros(1, dtype=torch.int32, device=DEV))
    tok = first[:, None] + np.arange(c["kmax"])
    used = np.arange(c["kmax"]) < n[:, None]
    page = np.take_along_axis(tables, np.where(used, tok // c["page"], 0), 1)
    s.slots = _i32(np.where(used, page * c["page"] + tok % c["page"], -1))
    s.K, s.V = ([_pool(c, gen, n_pages, False) for _ in range(c["layers"])] for _ in range(2))
    rows = (c["B"], c["kmax"], c["Hkv"], c["D"])
    s.Kr, s.Vr = ([_randn(gen, rows) if c["op"] == "write" else torch.zeros(rows, dtype=torch.bfloat16, device=DEV) for _ in range(c["layers"])]
                  for _ in range(2))
    s.desc = None
    return s


def _prepare_attend(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    of, plen, ctx, nq = _lengths(c)
    tables, n_pages = _page_rows(c, np.random.default_rng(seed), ctx + nq, of, plen)
    int8 = c["kv"] == "int8kv"
    s = SimpleNamespace(case=c, tables=_i32(tables), n_pages=n_pages, ctx=_i32(ctx), nq=_i32(nq), status=torch.zeros(1, dtype=torch.int32, device=DEV))
    s.prefix_of, s.prefix_len = (_i32(of), _i32(plen)) if c["prefixes"] else (None, None)
    s.K, s.V = ([_pool(c, gen, n_pages, int8) for _ in range(c["layers"])] for _ in range(2))
    q = (c["B"], c["kmax"], c["Hq"], c["D"])
    s.Q = [_randn(gen, q) for _ in range(c["layers"])]
    s.O = [torch.zeros(q, dtype=torch.bfloat16, device=DEV) for _ in range(c["layers"])]
    s.lse = [torch.zeros(q[:3], dtype=torch.float32, device=DEV) for _ in range(c["layers"])]
    s.desc = s.plan = s.ws = None
    return s


def prepare(case, seed):
    return {"tables": _prepare_tables, "write": _prepare_rows, "read": _prepare_rows, "attend": _prepare_attend}[case["op"]](case, seed)


# ---- one pass, in plain operations ------------------------------------------------------------------

def _plain_tables(s):
    c = s.case
    P, M, N = c["page"], c["max_pages"], c["pages"]
    held0, tables = s.held.long(), s.tables.long()
    R = held0.numel()
    need = (s.length.long() + P - 1) // P
    src = s.share_from.long()
    takes = (held0 == 0) & (src >= 0) & (need > 0)
    shared = torch.where(takes, torch.minimum(torch.minimum(s.share_len.long() // P, held0[src.clamp(min=0)]), need), 0)
    col = torch.arange(M, device=DEV)
    in_shared = col < shared[:, None]
    tables = torch.where(in_shared, tables[src.clamp(min=0)], tables)
    held = torch.where(takes, shared, held0)
    gone = (col >= need[:, None]) & (col < held[:, None])
    moved = in_shared | gone
    refs = s.refs.long().index_add(0, tables[moved], (in_shared.long() - gone.long())[moved])
    tables = torch.where(gone, -1, tables)
    held = torch.minimum(held, need)
    # free pages in the order of their numbers go to the rows in their order; rows behind the first that finds too few get none
    free = refs == 0
    rank = torch.cumsum(free, 0) - 1
    by_rank = torch.full((N + 1,), -1, device=DEV, dtype=torch.long).scatter_(0, torch.where(free, rank, N), torch.arange(N, device=DEV))
    wants = need - held
    last = torch.cumsum(wants, 0)
    gets = torch.where(last <= free.sum(), wants, 0)
    fill = (col >= held[:, None]) & (col < (held + gets)[:, None])
    at = (last - wants)[:, None] + col - held[:, None]
    fresh = by_rank[at.clamp(0, N - 1)]
    tables = torch.where(fill, fresh, tables)
    refs[fresh[fill]] = 1
    held = held + gets
    i = torch.arange(c["kmax"], device=DEV)
    tok = s.ctx.long()[:, None] + i
    ok = (i < s.n_new[:, None]) & (tok < held[:, None] * P)
    page = torch.gather(tables, 1, (tok // P).clamp(max=M - 1))
    slots = torch.where(ok, page * P + tok % P, -1)
    return {"held": held.int(), "tables": tables.int(), "refs": refs.int(), "slots": slots.int()}


def _token_index(c, slots):
    """(page, block, token of the block) of slots."""
    tok = slots % c["page"]
    return slots // c["page"], tok // BLOCK, tok % BLOCK


def _plain_write(s, layer):
    c = s.case
    D, H = c["D"], c["Hkv"]
    used = s.slots.view(-1) >= 0
    page, blk, tok = (x[used] for x in _token_index(c, s.slots.view(-1).long()))
    out = []
    for pool, rows, (shape, order) in ((s.K[layer], s.Kr[layer], _K_BLOCK(D, False)), (s.V[layer], s.Vr[layer], _V_BLOCK(D, False))):
        place = torch.arange(BLOCK * D, device=DEV).view(shape).permute(order).reshape(BLOCK, D)  # where [token][d] lies in a block
        base = ((page[:, None] * H + torch.arange(H, device=DEV)) * (c["page"] // BLOCK) + blk[:, None]) * (BLOCK * D)
        at = base[:, :, None] + place[tok][:, None, :]
        pool.view(-1)[at.view(-1)] = rows.view(-1, H * D)[used].view(-1)
        out.append(pool.view(torch.int16))
    return out


def _decoded(pool, shape, order, D, int8):
    """[..., block bytes or elements] -> [..., token, d] in 32 bits."""
    lead = pool.dim() - 1
    x = pool[..., : BLOCK * D].unflatten(-1, shape).permute(*range(lead), *(lead + o for o in order)).reshape(*pool.shape[:-1], BLOCK, D).float()
    return x * pool[..., BLOCK * D:].contiguous().view(torch.float32).unsqueeze(-1) if int8 else x


def _plain_read(s, layer):
    c = s.case
    D, H = c["D"], c["Hkv"]
    i = torch.arange(c["kmax"], device=DEV)
    used = i < s.n[:, None]
    tok = s.first.long()[:, None] + i
    page = torch.gather(s.tables.long(), 1, (tok // c["page"]).clamp(max=s.tables.shape[1] - 1)).clamp(min=0)
    _, blk, t = _token_index(c, tok)
    out = []
    for pool, rows, (shape, order) in ((s.K[layer], s.Kr[layer], _K_BLOCK(D, False)), (s.V[layer], s.Vr[layer], _V_BLOCK(D, False))):
        place = torch.arange(BLOCK * D, device=DEV).view(shape).permute(order).reshape(BLOCK, D)
        base = ((page[:, :, None] * H + torch.arange(H, device=DEV)) * (c["page"] // BLOCK) + blk[:, :, None]) * (BLOCK * D)
        x = pool.view(-1)[base[..., None] + place[t][:, :, None, :]]
        rows.copy_(torch.where(used[:, :, None, None], x, rows))
        out.append(rows.view(torch.int16))
    return out


def _plain_attend(s, layer):
    c = s.case
    B, kmax, Hq, H, D, int8 = c["B"], c["kmax"], c["Hq"], c["Hkv"], c["D"], c["kv"] == "int8kv"
    g = Hq // H
    at = s.tables.long().clamp(min=0)
    T = at.shape[1] * c["page"]
    K = _decoded(s.K[layer][at], *_K_BLOCK(D, int8), D, int8).permute(0, 2, 5, 1, 3, 4).reshape(B, H, D, T)
    q = s.Q[layer].float()
    if int8:  # queries are quantized like cached rows
        amax = q.abs().amax(-1, keepdim=True)
        q = torch.round(q * torch.where(amax > 0, 127.0 / amax, 0.0)) * (amax / 127.0)
    q = q.view(B, kmax, H, g, D).permute(0, 2, 1, 3, 4).reshape(B, H, kmax * g, D)
    S = torch.matmul(q, K).mul_(1.0 / math.sqrt(D)).view(B, H, kmax, g, T)
    del K
    i = torch.arange(kmax, device=DEV)
    hidden = torch.arange(T, device=DEV) > (s.ctx.long()[:, None] + i)[:, :, None]
    S.masked_fill_(hidden[:, None, :, None, :], float("-inf"))
    m = S.amax(-1, keepdim=True)
    S.sub_(m).exp_()
    l = S.sum(-1, keepdim=True)
    V = _decoded(s.V[layer][at], *_V_BLOCK(D, int8), D, int8).permute(0, 2, 1, 3, 4, 5).reshape(B, H, T, D)
    O = torch.matmul(S.view(B, H, kmax * g, T), V).view(B, H, kmax, g, D) / l
    live = (i < s.nq[:, None])[:, None, :, None, None]
    O = torch.where(live, O, 0.0).permute(0, 2, 1, 3, 4).reshape(B, kmax, Hq, D)
    lse = torch.where(live, m + l.log(), 0.0).permute(0, 2, 1, 3, 4).reshape(B, kmax, Hq)
    return O.to(torch.bfloat16), lse


# ---- one pass ---------------------------------------------------------------------------------------

def _scale(c):
    return 1.0 / math.sqrt(c["D"])


def _own_rows(s):
    import paper_2404_15778_amd as bass
    c = s.case
    if s.desc is None:
        s.desc = bass.make_paged_desc(c["B"], c["kmax"], c["Hkv"], c["Hkv"], c["D"], c["page"], s.n_pages, s.tables.shape[1], "bf16", _scale(c))
    for l in range(c["layers"]):
        if c["op"] == "write":
            bass.bass_paged_append(s.desc, s.K[l], s.V[l], s.Kr[l], s.Vr[l], s.slots, s.status)
        else:
            bass.bass_paged_gather(s.desc, s.K[l], s.V[l], s.Kr[l], s.Vr[l], s.tables, s.first, s.n, s.status)
    a, b = (s.K, s.V) if c["op"] == "write" else (s.Kr, s.Vr)
    return {"K": [x.view(torch.int16) for x in a], "V": [x.view(torch.int16) for x in b]}


def _own_tables(s):
    import paper_2404_15778_amd as bass
    c = s.case
    bass.bass_page_tables(s.length, s.held, s.tables, s.refs, c["page"], s.scratch, s.share_from, s.share_len, s.ctx, s.n_new, s.slots, s.status)
    return {"held": s.held, "tables": s.tables, "refs": s.refs, "slots": s.slots}


def _own_attend(s):
    import paper_2404_15778_amd as bass
    c = s.case
    if s.desc is None:
        s.desc = bass.make_paged_desc(c["B"], c["kmax"], c["Hq"], c["Hkv"], c["D"], c["page"], s.n_pages, s.tables.shape[1], c["kv"], _scale(c))
        s.plan, s.ws = bass.alloc_paged_plan(s.desc, DEV), bass.alloc_paged_workspace(s.desc, DEV)
    bass.bass_paged_attention_plan(s.desc, s.ctx, s.nq, s.prefix_of, s.prefix_len, s.plan, s.status)
    for l in range(c["layers"]):
        bass.bass_paged_verify_attention(s.desc, s.Q[l], s.K[l], s.V[l], s.tables, s.plan, s.O[l], s.lse[l], s.ws, s.status)
    return {"O": s.O, "lse": s.lse}


def run(state):
    s, c = state, state.case
    if c["op"] == "tables":
        s.now.copy_(s.before)  # the call changes its tables; every pass begins with the same
        return _own_tables(s) if own else _plain_tables(s)
    if c["op"] == "attend":
        if own:
            return _own_attend(s)
        both = [_plain_attend(s, l) for l in range(c["layers"])]
        return {"O": [x[0] for x in both], "lse": [x[1] for x in both]}
    if own:
        return _own_rows(s)
    both = [(_plain_write if c["op"] == "write" else _plain_read)(s, l) for l in range(c["layers"])]
    return {"K": [x[0] for x in both], "V": [x[1] for x in both]}


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "tables":
        # the references of every page are looked at, and each row's lengths, counts and slots; the tables only where they change
        return {"bytes": 4 * c["pages"] + 4 * c["rows"] * (7 + c["kmax"]), "flops": c["pages"]}
    if c["op"] in ("write", "read"):
        _, n = _row_lengths(c)
        return {"bytes": c["layers"] * 2 * 2 * int(n.sum()) * c["Hkv"] * c["D"] * 2, "flops": 0}
    of, plen, ctx, nq = (x.astype(np.int64) for x in _lengths(c))
    row = c["Hkv"] * (c["D"] + 4) if c["kv"] == "int8kv" else c["Hkv"] * c["D"] * 2  # one cached token of K or V
    live = nq > 0
    mine = ctx + nq - np.where(of >= 0, plen[of] if len(plen) else 0, 0)
    used = [int(n) for g, n in enumerate(plen) if np.any(live & (of == g))]
    tokens = int(mine[live].sum()) + sum(used)
    outs = c["B"] * c["kmax"] * c["Hq"]
    q = int(nq.sum()) * c["Hq"] * c["D"] * 2
    seen = int((nq * ctx + nq * (nq + 1) // 2).sum())
    return {"bytes": c["layers"] * (2 * tokens * row + q + outs * (2 * c["D"] + 4)), "flops": c["layers"] * 4 * seen * c["Hq"] * c["D"]}


# ---- what a pass returns, in 64 bits ----------------------------------------------------------------

def _value(pool, kind, D, int8, page, head, token):
    """K or V of tokens [n] of pages [n] (one kv head) as [n, D] in 64 bits, each element from its own place."""
    d = torch.arange(D, device=DEV)
    t = (token % BLOCK)[:, None]
    if kind == "K":
        width = 16 if int8 else 8
        at = ((((t // 16) * (D // (4 * width)) + d // (4 * width)) * 4 + d // width % 4) * 16 + t % 16) * width + d % width
    elif int8:
        at = ((((d // 32) * 4 + t // 4 % 4) * 16 + d % 16) * 2 + d // 16 % 2) * 8 + t // 16 * 4 + t % 4
    else:
        at = (((d // 16) * 4 + t // 4 % 4) * 16 + d % 16) * 8 + t // 16 * 4 + t % 4
    blk = token // BLOCK
    x = pool[page[:, None], head, blk[:, None], at].double()
    if int8:
        x = x * pool.view(torch.float32)[page, head, blk, BLOCK * D // 4 + token % BLOCK].double()[:, None]
    return x


def exact(case, seed):
    c = case
    if c["op"] != "attend":
        return None  # whole numbers and copies
    s = prepare(c, seed)
    _, _, ctx, nq = _lengths(c)
    Hq, H, D, P, int8 = c["Hq"], c["Hkv"], c["D"], c["page"], c["kv"] == "int8kv"
    g = Hq // H
    outs = {"O": [], "lse": []}
    for l in range(c["layers"]):
        O = torch.zeros((c["B"], c["kmax"], Hq, D), dtype=torch.float64, device=DEV)
        lse = torch.zeros((c["B"], c["kmax"], Hq), dtype=torch.float64, device=DEV)
        for b in range(c["B"]):
            n, L = int(nq[b]), int(ctx[b])
            if n == 0:
                continue
            tok = torch.arange(L + n, device=DEV)
            page = s.tables[b].long()[tok // P]
            Q = s.Q[l][b, :n].double()
            if int8:
                x = s.Q[l][b, :n].float()  # the quantizer's steps are single operations in 32 bits
                amax = x.abs().amax(-1, keepdim=True)
                Q = torch.round(x * torch.where(amax > 0, 127.0 / amax, torch.zeros_like(amax))).double() * (amax / 127.0).double()
            hidden = (tok > L + torch.arange(n, device=DEV)[:, None])[:, None, :]
            for h in range(H):
                K = _value(s.K[l], "K", D, int8, page, h, tok % P)
                V = _value(s.V[l], "V", D, int8, page, h, tok % P)
                q = Q[:, h * g:(h + 1) * g].reshape(n * g, D)
                S = (torch.matmul(q, K.t().contiguous()) / math.sqrt(D)).view(n, g, L + n).masked_fill(hidden, float("-inf"))
                lse[b, :n, h * g:(h + 1) * g] = torch.logsumexp(S, -1)
                O[b, :n, h * g:(h + 1) * g] = torch.matmul(torch.softmax(S, -1).view(n * g, L + n), V).view(n, g, D)
        outs["O"].append(O)
        outs["lse"].append(lse)
    return outs
