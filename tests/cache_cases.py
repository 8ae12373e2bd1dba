"""Paged caches for tests, and their bookkeeping in plain Python."""
import math

import torch

from attention_cases import offsets


def plan(length, added, pages, ring, turn, page_rows, n_rows):
    """What surel_cache_plan writes: (off, slots, length, turn, pages, ring) as lists; one page and one row at a time."""
    length, added, ring = length.tolist(), added.tolist(), ring.tolist()
    old = pages.tolist()
    table = [r[:] for r in old]
    width, n = pages.shape[1], len(ring)
    (taken, given), free = turn.tolist(), ring[:]
    end = given
    off, slots, after = [0], [-1] * n_rows, []
    for s, (have, add) in enumerate(zip(length, added)):
        if add < 0:
            for j in range(-(-have // page_rows)):
                ring[given % n] = old[s][j]
                given += 1
            off.append(off[-1])
            after.append(0)
            continue
        add = min(add, n_rows - off[-1])
        off.append(off[-1] + add)
        want = min(have + add, width * page_rows)
        held = -(-have // page_rows)
        for j in range(held, -(-want // page_rows)):
            table[s][j] = -1
            if taken < end:
                table[s][j] = free[taken % n]
                taken, held = taken + 1, held + 1
        kept = min(want, held * page_rows)
        for i in range(have, kept):
            slots[off[s] + i - have] = table[s][i // page_rows] * page_rows + i % page_rows
        after.append(kept)
    return off, slots, after, [taken, given], table, ring


def bookkeeping(lengths, added, page_rows, width, spare=0, round_=3, seed=0, device="cuda"):
    """(length, added, pages, ring, turn): sequences that hold pages in any order, the rest of them and `spare` more (as
    many as all need at least, where it is not negative) in a ring that has been round before and whose free ones pass its
    end."""
    g = torch.Generator().manual_seed(seed)
    held = [-(-x // page_rows) for x in lengths]
    fresh = [0 if a < 0 else -(-min(x + a, width * page_rows) // page_rows) - h for x, a, h in zip(lengths, added, held)]
    n = max(1, sum(held) + sum(fresh) + spare)
    order = torch.randperm(n, generator=g).tolist()
    pages = torch.full((len(lengths), width), -7, dtype=torch.int32)
    for s, h in enumerate(held):
        for j in range(h):
            pages[s, j] = order.pop()
    taken = round_ * n - min(2, n - 1)
    ring = torch.full((n,), -9, dtype=torch.int32)
    for i, page in enumerate(order):
        ring[(taken + i) % n] = page
    as_int = lambda x: torch.tensor(x, dtype=torch.int32).view(-1).to(device)  # noqa: E731
    return (as_int(lengths), as_int(added), pages.to(device), ring.to(device),
            torch.tensor([taken, taken + len(order)], device=device))


def cache(lengths, heads, kv_heads, dim, page_rows, dtype, seed=0, heads_first=False, device="cuda"):
    """(q, k, v, k_off, k_pages, v_pages, pages, length): one row a sequence, its keys packed and the same in pages, all
    other places of which hold NaN; the table's entries behind a sequence's pages are no pages."""
    g = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g).to(dtype)  # noqa: E731
    total = sum(lengths)
    q, k, v = normal(len(lengths), heads, dim), normal(total, kv_heads, dim), normal(total, kv_heads, dim)
    held = [-(-x // page_rows) for x in lengths]
    n = sum(held) + 3
    order = torch.randperm(n, generator=g).tolist()
    shape = (n, kv_heads, page_rows, dim) if heads_first else (n, page_rows, kv_heads, dim)
    stores = [torch.full(shape, math.nan, dtype=dtype) for _ in range(2)]
    views = [x.transpose(1, 2) if heads_first else x for x in stores]
    pages = torch.full((len(lengths), max(held, default=0) + 1), 2 ** 31 - 1, dtype=torch.int32)
    at = 0
    for s, x in enumerate(lengths):
        for j in range(held[s]):
            page = pages[s, j] = order.pop()
            rows = min(page_rows, x - j * page_rows)
            views[0][page, :rows], views[1][page, :rows] = k[at:at + rows], v[at:at + rows]
            at += rows
    stores = [x.to(device) for x in stores]
    views = [x.transpose(1, 2) if heads_first else x for x in stores]
    return (q.to(device), k.to(device), v.to(device), offsets(lengths, device), *views, pages.to(device),
            torch.tensor(lengths, dtype=torch.int32, device=device).view(-1))
