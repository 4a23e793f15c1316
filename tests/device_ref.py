"""Plain 64-bit definitions of the operators of horizonserve_device.h, on the CPU, and inputs that their tests share."""
from __future__ import annotations

import math

import numpy as np
import torch

PAGE = 16


def pages(n: int) -> int:
    return -(-n // PAGE)


# ------------------------------------------------------------------------------------------------------------ page tables
def step_tables(ctx, q, free_list, free_count, tables, num_pages, max_tokens):
    """Returns (status name or None, dict of arrays).  Lists of int; tables a 2-D int array (copied)."""
    n, width = len(ctx), tables.shape[1]
    tables = tables.copy()
    empty = {"kv_len": list(ctx), "tok_begin": [0] * (n + 1), "tok_seq": [-1] * max_tokens, "tok_pos": [-1] * max_tokens, "tok_slot": [-1] * max_tokens,
             "block_tables": tables, "free_count": free_count}
    if any(c < 0 or m < 0 or c + m > width * PAGE for c, m in zip(ctx, q)) or sum(q) > max_tokens or not 0 <= free_count <= num_pages:
        return "INVALID_ARG", empty
    if sum(pages(c + m) - pages(c) for c, m in zip(ctx, q)) > free_count:
        return "OUT_OF_PAGES", empty
    status, left = None, free_count
    seq, pos, slot, begin = [], [], [], [0]
    for s in range(n):
        for p in range(pages(ctx[s]), pages(ctx[s] + q[s])):
            left -= 1
            tables[s, p] = free_list[left]
        for p in range(ctx[s], ctx[s] + q[s]):
            page = int(tables[s, p // PAGE])
            seq.append(s)
            pos.append(p)
            if 0 <= page < num_pages:
                slot.append(page * PAGE + p % PAGE)
            else:
                slot.append(-1)
                status = "BAD_BLOCK_TABLE"
        begin.append(begin[-1] + q[s])
    pad = [-1] * (max_tokens - len(seq))
    return status, {"kv_len": [c + m for c, m in zip(ctx, q)], "tok_begin": begin, "tok_seq": seq + pad, "tok_pos": pos + pad, "tok_slot": slot + pad,
                    "block_tables": tables, "free_count": left}


def release_pages(done, ctx, tables, free_list, free_count):
    tables, ctx, free_list = tables.copy(), list(ctx), list(free_list)
    for s, d in enumerate(done):
        if not d:
            continue
        for p in reversed(range(pages(ctx[s]))):
            free_list[free_count] = int(tables[s, p])
            tables[s, p] = -1
            free_count += 1
        ctx[s] = 0
    return ctx, tables, free_list, free_count


# ------------------------------------------------------------------------------------------------------------------- rope
def frequencies(rot, base, scaling="plain", factor=1.0, trained=0, slow=1.0, fast=32.0):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2.0))
    w = base ** (-2.0 * i / rot)
    if scaling == "linear":
        w = w / factor
    if scaling == "by_parts":
        keep = np.clip((trained * w / (2 * math.pi) - slow) / (fast - slow), 0.0, 1.0)
        w = w * keep + w / factor * (1 - keep)
    return w


def rotate(x, table, pos, interleaved):
    """x [tokens, heads, dim] fp64; table [positions, pairs, 2]; returns the rotated copy."""
    x, pairs = x.clone(), table.shape[1]
    for t, p in enumerate(pos):
        for i in range(pairs):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
            c, s = float(table[p, i, 0]), float(table[p, i, 1])
            u, v = x[t, :, a].clone(), x[t, :, b].clone()
            x[t, :, a], x[t, :, b] = u * c - v * s, u * s + v * c
    return x


# -------------------------------------------------------------------------------------------------------------- attention
def attention(q, pool_layer, tables, kv_len, q_len, prefix=None, slopes=None, scale=1.0, cap=0.0, window=0):
    """q [tokens, hq, dim], pool_layer [2, pages, hkv, 16, dim], both fp64.  Returns (o, lse) of all rows."""
    t, hq, dim = q.shape
    hkv = pool_layer.shape[2]
    o, lse = torch.zeros(t, hq, dim, dtype=torch.float64), torch.full((t, hq), -math.inf, dtype=torch.float64)
    row = 0
    for s, (kv, n) in enumerate(zip(kv_len, q_len)):
        for r in range(n):
            p = kv - n + r
            pre = 0 if prefix is None else min(max(prefix[s], 0), kv)
            keys = [j for j in range(kv) if (j <= p and (window == 0 or p - j < window)) or j < pre]
            if keys:
                page = torch.tensor([int(tables[s][j // PAGE]) for j in keys])
                off = torch.tensor([j % PAGE for j in keys])
                k, v = pool_layer[0][page, :, off], pool_layer[1][page, :, off]          # [keys, hkv, dim]
                x = torch.einsum("hgd,khd->hgk", q[row].view(hkv, hq // hkv, dim), k) * scale
                if cap:
                    x = cap * torch.tanh(x / cap)
                if slopes is not None:
                    x = x - slopes.view(hkv, -1, 1) * (p - torch.tensor(keys, dtype=torch.float64)).abs()
                lse[row] = torch.logsumexp(x, -1).view(hq)
                o[row] = torch.einsum("hgk,khd->hgd", torch.softmax(x, -1), v).reshape(hq, dim)
            row += 1
    return o, lse


# ---------------------------------------------------------------------------------------------------------- log probabilities
def logprobs(x, targets, n_top, scale):
    """x [rows, vocab] fp64 without NaN and +infinity."""
    out = {"logprob": [], "entropy": [], "rank": [], "top_ids": [], "top_logprobs": []}
    for row, t in zip(x, targets):
        l = row * scale
        big = float(l.max())
        if big == -math.inf:
            lp, entropy = l, 0.0
        else:
            lp = l - (big + math.log(float(torch.exp(l - big).sum())))
            p = torch.exp(lp)
            entropy = -float((p * torch.where(p > 0, lp, torch.zeros_like(lp))).sum())
        real = 0 <= t < len(row)
        out["logprob"].append(float(lp[t]) if real else 0.0)
        out["entropy"].append(entropy)
        out["rank"].append(int((row > row[t]).sum()) if real else -1)
        order = sorted(range(len(row)), key=lambda v: (-float(row[v]), v))[:n_top] if len(row) <= 4096 else \
            torch.sort(-row, stable=True).indices[:n_top].tolist()
        out["top_ids"].append(order)
        out["top_logprobs"].append([float(lp[v]) for v in order])
    return out


# ------------------------------------------------------------------------------------------------------------------ inputs
def random_tables(rng, lens, width, num_pages):
    """Block tables [n, width] with distinct random pages for `lens` tokens, -1 behind them, and the free pages."""
    order = rng.permutation(num_pages).astype(np.int32)
    tables, at = np.full((len(lens), width), -1, dtype=np.int32), 0
    for s, n in enumerate(lens):
        tables[s, :pages(n)] = order[at:at + pages(n)]
        at += pages(n)
    return tables, order[at:]
