"""Plain definitions of the operators of horizonserve_beams.h, on the CPU: lists and numpy, scores in 64 bits."""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def pages(n: int) -> int:
    return -(-n // PAGE)


# -------------------------------------------------------------------------------------------------------------- selection
def log_sum(row, scale):
    """log sum_v exp(scale x_v) of a row of fp64 logits; None where it has NaN or +infinity."""
    if np.isnan(row).any() or (row == math.inf).any():
        return None
    top = row.max()
    return -math.inf if top == -math.inf else scale * top + math.log(np.exp(scale * (row - top)).sum())


def select(x, scores, done, weight, n_out, end_token, scale):
    """x [requests * beams, vocab] fp64.  Returns a list per request of (ranked score, beam, token, score, over), best first, and the rows' lse."""
    n, b = scores.shape
    chosen, lse = [], []
    for r in range(n):
        found = []
        for i in range(b):
            w, s = float(weight[r, i]) if weight is not None else 1.0, float(scores[r, i])
            if done is not None and done[r, i]:
                lse.append(0.0)
                if w * s > -math.inf:
                    found.append((w * s, i, end_token, s, 1))
                continue
            row = x[r * b + i]
            big = log_sum(row, scale)
            lse.append(math.nan if big is None else big)
            if big is None or big == -math.inf:
                continue
            top = row.max()                              # (scores relative to it: a row far from zero keeps its differences)
            rest = math.log(np.exp(scale * (row - top)).sum())
            for v in np.argsort(-row, kind="stable")[:n_out]:
                c = s + (scale * (row[v] - top) - rest)
                if w * c > -math.inf:
                    found.append((w * c, i, int(v), c, int(v == end_token)))
        found.sort(key=lambda f: (-f[0], f[1], f[2]))
        chosen.append(found[:n_out])
    return chosen, lse


# ------------------------------------------------------------------------------------------------------------ shared pages
def fork(parent, ctx, tables, shares, free_list, free_count, num_pages):
    """Returns (status name or None, dict of what the call leaves)."""
    n = len(parent)
    same = {"ctx_len": list(ctx), "block_tables": tables.copy(), "shares": list(shares), "free_list": list(free_list), "free_count": free_count,
            "copy_src": [-1] * n, "copy_dst": [-1] * n, "copy_len": [0] * n}
    if any(not -1 <= p < n for p in parent) or any(not 0 <= c <= tables.shape[1] * PAGE for c in ctx) or not 0 <= free_count <= num_pages:
        return "INVALID_ARG", same
    first = {}
    for i, p in enumerate(parent):
        if p >= 0:
            first.setdefault(p, i)
    copies = [i for i, p in enumerate(parent) if p >= 0 and ctx[p] % PAGE and first[p] != i]
    if len(copies) > free_count:
        return "OUT_OF_PAGES", same
    out, status, inside = dict(same, ctx_len=[0] * n), None, lambda page: 0 <= page < num_pages
    holders = [s + 1 for s in shares]
    lost, new = set(), out["block_tables"]
    for i in range(n):
        for c in range(pages(ctx[i])):
            new[i, c] = -1
    top = free_count
    for i, p in enumerate(parent):
        if p < 0:
            continue
        out["ctx_len"][i] = ctx[p]
        for c in range(pages(ctx[p])):
            page = int(tables[p, c])
            if i in copies and c == ctx[p] // PAGE:
                top -= 1
                fresh = int(free_list[top])
                if inside(page) and inside(fresh):
                    out["copy_src"][i], out["copy_dst"][i], out["copy_len"][i] = page, fresh, ctx[p] % PAGE
                else:
                    status = "BAD_BLOCK_TABLE"
                page = fresh
            new[i, c] = page
    for i in range(n):                                   # holders: minus the old rows', plus the new rows' but their copies
        for c in range(pages(ctx[i])):
            page = int(tables[i, c])
            if not inside(page):
                status = "BAD_BLOCK_TABLE"
                continue
            kept = sum(1 for j, p in enumerate(parent) if p == i and not (j in copies and c == ctx[i] // PAGE))
            holders[page] += kept - 1
            lost.add(page)
    for page in sorted(lost):
        if holders[page] == 0:
            holders[page] = 1
            out["free_list"][top] = page
            top += 1
    out["shares"], out["free_count"] = [h - 1 for h in holders], top
    return status, out


def compact(keep, ctx, tables, shares, free_list, free_count, num_pages, max_copies):
    same = {"block_tables": tables.copy(), "shares": list(shares), "free_list": list(free_list), "copy_src": [-1] * max_copies, "copy_dst": [-1] * max_copies}
    if any(not 0 <= c <= tables.shape[1] * PAGE for c in ctx) or not 0 <= free_count <= num_pages:
        return "INVALID_ARG", same
    free = [int(p) for p in free_list[:free_count]]
    if len(set(free)) != len(free) or any(not 0 <= p < num_pages for p in free):
        return "INVALID_ARG", same
    free = set(free)
    low, used = sorted(p for p in free if p < keep), [p for p in range(keep, num_pages) if p not in free]
    if len(used) > max_copies:
        return "INVALID_ARG", same
    if len(used) > len(low):
        return "OUT_OF_PAGES", same
    to, status, out = dict(zip(used, low)), None, same
    for i, c in enumerate(ctx):
        for j in range(pages(c)):
            page = int(tables[i, j])
            if page in to:
                out["block_tables"][i, j] = to[page]
            elif page >= keep or page < 0:
                status = "BAD_BLOCK_TABLE"
    for k, (a, b) in enumerate(to.items()):
        out["shares"][b], out["shares"][a] = out["shares"][a], 0
        out["copy_src"][k], out["copy_dst"][k] = a, b
    rest = low[len(used):] + list(range(keep, num_pages))
    out["free_list"][:len(rest)] = rest[::-1]
    return status, out


# ------------------------------------------------------------------------------------------------------------------ inputs
def shared_rows(rng, n_requests, beams, lens, spare):
    """Block tables of requests whose beams (all of a request's of one length) share ever fewer of their later pages, with counts and free pages."""
    rows, width = n_requests * beams, max(pages(x) for x in lens) + 2
    tables, used, ctx = np.full((rows, width), -1, dtype=np.int64), 0, []
    for r in range(n_requests):
        full = lens[r] // PAGE
        for c in range(pages(lens[r])):
            together = int(rng.choice([d for d in (1, 2, beams) if d <= beams])) if c < full else 1
            for b in range(0, beams, together):
                tables[r * beams + b:r * beams + min(b + together, beams), c] = used
                used += 1
        ctx += [lens[r]] * beams
    num_pages = used + spare
    name = rng.permutation(num_pages)
    shares = np.zeros(num_pages, dtype=np.int64)
    np.add.at(shares, name[tables[tables >= 0]], 1)
    return ctx, np.where(tables >= 0, name[tables.clip(0)], -1).astype(np.int32), (shares - 1).clip(0).tolist(), name[used:].tolist(), num_pages


def grouped_tables(rng, groups, width, num_pages=None):
    """groups: (shared keys, [own keys of each sequence]).  Block tables of the sequences, the first shared // 16 pages of a group's the same, -1 behind."""
    need = sum(s // PAGE + sum(pages(s + n) - s // PAGE for n in own) for s, own in groups)
    num_pages = num_pages or need + 2
    name, used, rows = rng.permutation(num_pages), 0, []
    for shared, own in groups:
        whole = shared // PAGE
        common, used = name[used:used + whole], used + whole
        for n in own:
            mine = pages(shared + n) - whole
            rows.append(np.concatenate([common, name[used:used + mine], np.full(width - whole - mine, -1)]))
            used += mine
    return np.stack(rows).astype(np.int32), num_pages
