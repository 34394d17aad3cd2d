"""Oracle for page tables: one row after the other, with sets.  TEST INFRASTRUCTURE ONLY.

A row holds the pages of its table; a page is free when no row holds it.  Rows without pages begin with the first pages of another row
as it was; rows give their last pages back, or take the lowest free numbers, until they hold ceil(length / page_tokens).
"""
from __future__ import annotations

LEN_CLAMPED, PAGE_CLAMPED, NO_PAGES = 1, 16, 32


def page_tables(length, held, tables, refs, page_tokens, share_from=None, share_len=None, ctx_len=None, n_new=None, kmax=0):
    """Lists in, new lists out: (held, tables, refs, slots or None, status)."""
    rows, most, status = len(length), len(tables[0]), 0
    before = [list(t) for t in tables]
    held0 = [min(max(h, 0), most) for h in held]
    held, tables, refs = list(held0), [list(t) for t in tables], list(refs)
    need = []
    for n in length:
        if not 0 <= n <= most * page_tokens:
            n, status = min(max(n, 0), most * page_tokens), status | LEN_CLAMPED
        need.append(-(-n // page_tokens))
    for r in range(rows):
        if share_from is None or held0[r] or not need[r]:
            continue
        src = share_from[r]
        if src >= rows or src == r:
            status |= LEN_CLAMPED
        elif src >= 0:
            held[r] = min(max(share_len[r], 0) // page_tokens, held0[src], need[r])
            for j in range(held[r]):
                page = before[src][j]
                if not 0 <= page < len(refs):
                    page, status = -1, status | PAGE_CLAMPED
                else:
                    refs[page] += 1
                tables[r][j] = page
    for r in range(rows):
        for j in range(need[r], held[r]):
            page = tables[r][j]
            if 0 <= page < len(refs):
                refs[page] -= 1
            else:
                status |= PAGE_CLAMPED
            tables[r][j] = -1
        held[r] = min(held[r], need[r])
    free = [p for p, n in enumerate(refs) if n == 0]
    enough = True
    for r in range(rows):
        want = need[r] - held[r]
        if want == 0:
            continue
        enough = enough and want <= len(free)
        if not enough:
            status |= NO_PAGES
            continue
        for page in free[:want]:
            tables[r][held[r]] = page
            refs[page] = 1
            held[r] += 1
        free = free[want:]
    slots = None
    if ctx_len is not None:
        slots = [[-1] * kmax for _ in range(rows)]
        for r in range(rows):
            if not 0 <= n_new[r] <= kmax:
                status |= LEN_CLAMPED
            for i in range(min(max(n_new[r], 0), kmax)):
                t = ctx_len[r] + i
                if t < 0:
                    status |= LEN_CLAMPED
                elif t // page_tokens < held[r]:
                    page = tables[r][t // page_tokens]
                    if 0 <= page < len(refs):
                        slots[r][i] = page * page_tokens + t % page_tokens
                    else:
                        status |= PAGE_CLAMPED
    return held, tables, refs, slots, status
