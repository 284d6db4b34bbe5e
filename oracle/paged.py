"""Plain CPU definition of the serving calls over a paged cache of latents (test infrastructure:
only tests and the smoke check use it; the HIP path never imports it).

  * ``plan`` / ``release``: pages, slots and positions of a step's tokens, and the pages of
    requests that ended, one token and one page at a time, in plain Python integers;
  * ``append``: a token's cache row, the producers' normalisation and rotation
    (``oracle.producers``) written at its slot;
  * ``attend``: the explicit form of ``oracle.laga`` at single rows: K_nope and V of every head
    rebuilt from the cached latents of the row's request, softmax over positions 0 .. p, in fp64.
    (The kernels compute the absorbed form, which ``oracle.absorbed`` pins to the explicit one.)

Parity status: pinned by tests/test_paged_oracle.py (hand-written steps, conservation of pages,
the rows of ``oracle.laga.attn_fwd`` and of the absorbed form, the producers' rows).
"""
from __future__ import annotations

import numpy as np

from . import producers

__all__ = ["PLAN_ROWS", "PLAN_TABLE", "PLAN_PAGES", "PLAN_INVALID", "plan", "release", "append", "gather", "attend"]

PLAN_ROWS, PLAN_TABLE, PLAN_PAGES, PLAN_INVALID = 1, 2, 4, 8


def _pages(n, page):
    return -(-n // page)


def plan(lengths, fresh, table, free_pages, free_count, rows, page):
    """One step that adds fresh[r] tokens to request r. Returns a dict of the call's outputs
    (table included); the inputs are not written."""
    lengths, fresh = [int(x) for x in lengths], [int(x) for x in fresh]
    table, free, n_pages, width = np.array(table), [int(x) for x in free_pages], len(free_pages), table.shape[1]
    status, R = 0, len(lengths)
    need = 0
    for n, f in zip(lengths, fresh):
        if n < 0 or f < 0:
            status |= PLAN_INVALID
        elif n + f > width * page:
            status |= PLAN_TABLE
        else:
            need += _pages(n + f, page) - _pages(n, page)
    good = [(n, f) for n, f in zip(lengths, fresh) if n >= 0 and f >= 0 and n + f <= width * page]
    if not 0 <= free_count <= n_pages:
        status |= PLAN_INVALID
    elif need > free_count:
        status |= PLAN_PAGES
    if sum(f for _, f in good) > rows:
        status |= PLAN_ROWS
    out = {"block_table": table, "row_request": [-1] * rows, "position": [-1] * rows, "slot": [-1] * rows,
           "row_begin": [0] * (R + 1), "lengths_out": list(lengths), "free_count_out": free_count, "status": status}
    if status:
        return out
    t = 0
    for r in range(R):
        out["row_begin"][r] = t
        for p in range(lengths[r], lengths[r] + fresh[r]):
            if p % page == 0:
                free_count -= 1
                table[r, p // page] = free[free_count]
            pid = int(table[r, p // page])
            out["row_request"][t], out["position"][t] = r, p
            out["slot"][t] = pid * page + p % page if 0 <= pid < n_pages else -1
            t += 1
        out["lengths_out"][r] = lengths[r] + fresh[r]
    out["row_begin"][R] = t
    out["free_count_out"] = free_count
    return out


def release(lengths, drop, table, free_pages, free_count, page):
    """The pages of the requests with drop[r] != 0 go back on the stack."""
    lengths, free, n_pages = [int(x) for x in lengths], [int(x) for x in free_pages], len(free_pages)
    status, back = 0, []
    for r, n in enumerate(lengths):
        if n < 0:
            status |= PLAN_INVALID
        elif n > table.shape[1] * page:
            status |= PLAN_TABLE
        elif drop[r]:
            back += [int(table[r, j]) for j in range(_pages(n, page))]
    if not 0 <= free_count <= n_pages:
        status |= PLAN_INVALID
    elif free_count + len(back) > n_pages:
        status |= PLAN_PAGES
    if status:
        return {"free_pages": free, "lengths_out": lengths, "free_count_out": free_count, "status": status}
    for pid in back:
        free[free_count] = pid
        free_count += 1
    return {"free_pages": free, "lengths_out": [0 if d else n for n, d in zip(lengths, drop)],
            "free_count_out": free_count, "status": 0}


def append(latent_raw, kpe_raw, position, slot, cache, gamma=None, eps=1e-6, base=10000.0, offset=0):
    """cache [n_pages, page, d_c + d_rope] (fp64 copy) with the tokens' rows in their slots."""
    out = np.array(cache, dtype=np.float64)
    n_pages, page = out.shape[:2]
    y, _ = producers.rms_norm(latent_raw, gamma, eps)
    for t, s in enumerate(slot):
        if 0 <= s < n_pages * page:
            k = producers.rope(np.asarray(kpe_raw, np.float64)[None, t:t + 1], np.array([offset + int(position[t])]), base)
            out[s // page, s % page] = np.concatenate([y[t], k[0, 0]])
    return out


def gather(cache, table_row, n):
    """The first n cached rows of a request, [n, d_c + d_rope]."""
    page = cache.shape[1]
    return np.stack([np.asarray(cache[table_row[j // page], j % page], np.float64) for j in range(n)])


def attend(q, w_kv_b, cache, table, position, request, *, d_c, d_nope, d_v, scale, base=None, offset=0):
    """out [T, H, d_v] and lse [T, H] of rows at position[t] of request[t]; with ``base`` q's rope
    band is rotated first. A row at a negative position is 0 and -inf; one outside the table, or
    that sees a page outside the pool, NaN."""
    q, w = np.array(q, np.float64), np.asarray(w_kv_b, np.float64)
    T, H, _ = q.shape
    n_pages, page = cache.shape[:2]
    out, lse = np.zeros((T, H, d_v)), np.full((T, H), -np.inf)
    for t in range(T):
        p, r = int(position[t]), int(request[t])
        if p < 0:
            continue
        ids = table[r, :p // page + 1] if 0 <= r < table.shape[0] and p < table.shape[1] * page else [-1]
        if any(not 0 <= int(i) < n_pages for i in ids):
            out[t], lse[t] = np.nan, np.nan
            continue
        rows = gather(cache, table[r], p + 1)
        if base is not None:
            q[t, :, d_nope:] = producers.rope(q[None, t:t + 1, :, d_nope:], np.array([offset + p]), base)[0, 0]
        for h in range(H):
            kv = rows[:, :d_c] @ w[:, h * (d_nope + d_v):(h + 1) * (d_nope + d_v)]
            z = scale * (kv[:, :d_nope] @ q[t, h, :d_nope] + rows[:, d_c:] @ q[t, h, d_nope:])
            m = z.max()
            e = np.exp(z - m)
            lse[t, h] = m + np.log(e.sum())
            out[t, h] = (e / e.sum()) @ kv[:, d_nope:]
    return out, lse
