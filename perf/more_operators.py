"""Cases of the operators of beam search and shared prompts on the device, with their plain forms.

Requests that continue one prompt in several ways share its pages.  Five operators keep such a loop on the device:

  select      the best continuations over the beams and the vocabulary of every request, from logits and accumulated scores
  fork        rows of block tables continue other rows: pages shared and counted, partly filled ones listed to be copied, dropped ones freed
  copy        the keys and values of listed pages, in every layer
  compact     pages moved below a bound, so that the upper end of the pool is free
  attention   one new token per sequence over the paged cache, where the sequences of a group share their first keys

The plain forms are elementary torch operations in 32 bits, rounded once at the end; `select` ranks in 64, as candidates of different beams lie
as near to one another as they please.  The layout of the cache is the library's: [layer][K or V][page][kv head][16][head_dim].
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
WORKSPACE_BYTES = 32 << 20
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # one request of an interactive user, four beams, fp32 logits as the head leaves them: latency
        {"name": "select_1x4", "op": "select", "requests": 1, "beams": 4, "vocab": 152064, "type": "f32", "out": 8, "ended": False, "mix": 1},
        # a full batch, eight beams each, some of them ended and ranked by their length: the logits' bytes
        {"name": "select_64x8", "op": "select", "requests": 64, "beams": 8, "vocab": 152064, "type": "bf16", "out": 8, "ended": True, "mix": 2},
        # two requests with eight beams of a short context
        {"name": "fork_2x8", "op": "fork", "requests": 2, "beams": 8, "ctx_lo": 100, "ctx_hi": 1000, "spare": 500, "mix": 3},
        # a full batch of long contexts in a pool of a whole card
        {"name": "fork_64x8", "op": "fork", "requests": 64, "beams": 8, "ctx_lo": 512, "ctx_hi": 4096, "spare": 100000, "mix": 4},
        # partly filled pages of forked rows at the talker's dimensions
        {"name": "copy_tails_24", "op": "copy", "pages": 24, "layers": 12, "hkv": 4, "dh": 64, "type": "f16", "part": True, "mix": 5},
        # whole pages of a pool that is made smaller, at the 7B dimensions
        {"name": "copy_whole_300", "op": "copy", "pages": 300, "layers": 28, "hkv": 4, "dh": 128, "type": "bf16", "part": False, "mix": 6},
        # a small pool gives a quarter of its pages away
        {"name": "compact_1000", "op": "compact", "pages": 1000, "keep": 750, "rows": 16, "fill": 0.5, "mix": 7},
        # the pool of a whole card
        {"name": "compact_200000", "op": "compact", "pages": 200000, "keep": 150001, "rows": 512, "fill": 0.6, "mix": 8},
        # four beams of one prompt at the 7B dimensions: latency
        {"name": "attention_1x4", "op": "attention", "groups": 1, "m_lo": 4, "m_hi": 4, "hq": 28, "hkv": 4, "dh": 128, "type": "bf16", "shared_lo": 500,
         "shared_hi": 500, "own_lo": 1, "own_hi": 60, "cap": 0.0, "bias": False, "mix": 9},
        # groups of different sizes at the talker's dimensions with capped scores and a distance bias
        {"name": "attention_talker_9", "op": "attention", "groups": 9, "m_lo": 1, "m_hi": 16, "hq": 16, "hkv": 4, "dh": 64, "type": "f16", "shared_lo": 64,
         "shared_hi": 1024, "own_lo": 1, "own_hi": 200, "cap": 30.0, "bias": True, "mix": 10},
        # a full batch of beam searches: every prompt is read once for its eight beams
        {"name": "attention_64x8", "op": "attention", "groups": 64, "m_lo": 8, "m_hi": 8, "hq": 28, "hkv": 4, "dh": 128, "type": "bf16", "shared_lo": 512,
         "shared_hi": 2048, "own_lo": 16, "own_hi": 200, "cap": 50.0, "bias": False, "mix": 11},
        # 256 requests behind one long system prompt
        {"name": "attention_system_256", "op": "attention", "groups": 1, "m_lo": 256, "m_hi": 256, "hq": 28, "hkv": 4, "dh": 128, "type": "bf16",
         "shared_lo": 8191, "shared_hi": 8191, "own_lo": 64, "own_hi": 1024, "cap": 0.0, "bias": False, "mix": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("select", "select", "fork", "copy", "compact", "attention", "attention", "attention"))
    mix = rng.randrange(1 << 30)
    if op == "select":
        beams, vocab, dt = rng.choice((1, 2, 4, 5, 8, 16, 32)), rng.choice((152064, _log(rng, 1000, 152064))), rng.choice(("f32", "bf16", "f16"))
        most = max(1, min(64, 512 * 152064 // (beams * vocab) // (2 if dt == "f32" else 1)))
        return {"op": "select", "requests": _log(rng, 1, most), "beams": beams, "vocab": vocab, "type": dt, "out": rng.choice((beams, min(2 * beams, 32), 8)),
                "ended": rng.random() < 0.5, "mix": mix}
    if op == "fork":
        hi = _log(rng, 16, 4096)
        return {"op": "fork", "requests": _log(rng, 1, 64), "beams": rng.choice((1, 2, 3, 4, 8)), "ctx_lo": hi // rng.choice((1, 4, 16)), "ctx_hi": hi,
                "spare": _log(rng, 100, 100000), "mix": mix}
    if op == "copy":
        layers, hkv, dh = rng.choice(((28, 4, 128), (12, 4, 64), (2, 1, 128), (4, 8, 64), (5, 3, 128)))
        return {"op": "copy", "pages": _log(rng, 1, 300), "layers": layers, "hkv": hkv, "dh": dh, "type": rng.choice(("bf16", "f16")), "part": rng.random() < 0.5,
                "mix": mix}
    if op == "compact":
        pages = _log(rng, 64, 200000)
        fill = rng.uniform(0.1, 0.7)
        return {"op": "compact", "pages": pages, "keep": int(pages * rng.uniform(min(fill + 0.15, 0.9), 0.95)), "rows": _log(rng, 1, max(1, min(512, pages // 16))),
                "fill": fill, "mix": mix}
    hq, hkv = rng.choice(((28, 4), (16, 2), (16, 4), (16, 16), (12, 1), (5, 5)))
    case = {"op": "attention", "hq": hq, "hkv": hkv, "dh": rng.choice((64, 128)), "type": rng.choice(("bf16", "f16")), "cap": rng.choice((0.0, 0.0, 30.0, 50.0)),
            "bias": rng.random() < 0.3, "mix": mix}
    shared, m, most_own = _log(rng, 16, 8192), _log(rng, 1, 64), _log(rng, 4, 1024)
    most = max(1, min(64, 16000 // (m * most_own // 8 + shared) // max(1, hkv // 4), 512 // m))
    return dict(case, groups=_log(rng, 1, most), m_lo=max(1, m // rng.choice((1, 4))), m_hi=m, shared_lo=max(1, shared // rng.choice((1, 4))), shared_hi=shared,
                own_lo=max(1, most_own // rng.choice((1, 8))), own_hi=most_own)


# ------------------------------------------------------------------------------------------- sizes of a case
def _pages(n):
    return -(-n // PAGE)


def _fork_lengths(case):
    """Tokens of every row: the beams of a request have the same number."""
    r = random.Random(case["mix"])
    return [n for n in (r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["requests"])) for _ in range(case["beams"])]


def _copy_lengths(case):
    r = random.Random(case["mix"])
    return [r.randint(1, PAGE - 1) if case["part"] else PAGE for _ in range(case["pages"])]


def _compact_lengths(case):
    """Pages of every row."""
    r, left = random.Random(case["mix"]), int(case["pages"] * case["fill"])
    parts = [r.uniform(0.2, 1.8) for _ in range(case["rows"])]
    return [int(left * part / sum(parts)) for part in parts]


def _attention_lengths(case):
    """(sequences, shared keys) of each group, and the keys of each sequence behind the shared ones."""
    r = random.Random(case["mix"])
    groups = [(r.randint(case["m_lo"], case["m_hi"]), r.randint(case["shared_lo"], case["shared_hi"])) for _ in range(case["groups"])]
    return groups, [[r.randint(case["own_lo"], case["own_hi"]) for _ in range(m)] for m, _ in groups]


# ------------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 29)
    return g


def _i32(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device="cuda")


def prepare(case, seed):
    state = {"select": _prepare_select, "fork": _prepare_fork, "copy": _prepare_copy, "compact": _prepare_compact, "attention": _prepare_attention}[case["op"]](case, seed)
    state["op"] = case["op"]
    state["workspace"] = torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    state["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return state


def _prepare_select(case, seed):
    g, n, b, v, k = _gen(seed), case["requests"], case["beams"], case["vocab"], case["out"]
    x = torch.empty(n * b, v, dtype=TYPES[case["type"]], device="cuda")
    for i in range(0, n * b, 256):                   # a trained head's logits: a broad body and a few strong candidates per row
        part = 2.0 * torch.randn(min(256, n * b - i), v, generator=g, device="cuda")
        part += 12.0 * (torch.rand(part.shape, generator=g, device="cuda") < 8.0 / v)
        x[i:i + 256] = part.to(x.dtype)
    scores = -20.0 - 3.0 * torch.rand(n, b, generator=g, device="cuda")
    done = weight = None
    if case["ended"]:                                # beams that ended at different lengths are ranked by their mean log probability
        done = (torch.rand(n, b, generator=g, device="cuda") < 0.125).int()
        length = torch.where(done > 0, torch.randint(20, 40, (n, b), generator=g, device="cuda"), torch.full((n, b), 40, device="cuda"))
        weight = length.float() ** -0.7
    f = lambda: torch.empty(n, k, dtype=torch.float32, device="cuda")  # noqa: E731
    i = lambda: torch.empty(n, k, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"logits": x, "scores": scores, "done": done, "weight": weight, "end_token": v // 3, "scale": 1.25, "out_score": f(), "out_parent": i(), "out_token": i(),
            "out_done": i(), "lse": torch.empty(n * b, dtype=torch.float32, device="cuda")}


def _prepare_fork(case, seed):
    rng, lens, beams = np.random.default_rng(seed), _fork_lengths(case), case["beams"]
    rows, width = len(lens), max(_pages(n) for n in lens) + 4
    tables, used = np.full((rows, width), -1, dtype=np.int64), 0
    for r in range(0, rows, beams):                  # the prompt's pages are all beams', those behind it ever fewer beams', the last one each its own
        full, all_pages = lens[r] // PAGE, _pages(lens[r])
        for c in range(all_pages):
            together = beams if c < full * 3 // 4 else max(1, beams >> min(c - full * 3 // 4 + 1, 5)) if c < full else 1
            for b in range(0, beams, together):
                tables[r + b:r + min(b + together, beams), c] = used
                used += 1
    num_pages = used + rows + case["spare"]
    name = rng.permutation(num_pages)
    shares = np.zeros(num_pages, dtype=np.int64)
    np.add.at(shares, name[tables[tables >= 0]], 1)
    parent = np.concatenate([r + rng.integers(0, beams, beams) for r in range(0, rows, beams)])
    parent[(rng.random(rows // beams) < 1 / 16).repeat(beams)] = -1       # requests that have ended
    free = name[used:]
    i = lambda: torch.empty(rows, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"parent": _i32(parent), "ctx_len": _i32(lens), "block_tables": _i32(np.where(tables >= 0, name[tables.clip(0)], -1)), "shares": _i32((shares - 1).clip(0)),
            "free_list": _i32(np.concatenate([free, np.zeros(num_pages - len(free), dtype=np.int64)])), "free_count": _i32([len(free)]), "copy_src": i(),
            "copy_dst": i(), "copy_len": i()}


def _prepare_copy(case, seed):
    g, n = _gen(seed), case["pages"]
    pool = torch.empty(case["layers"], 2, 2 * n + 3, case["hkv"], PAGE, case["dh"], dtype=TYPES[case["type"]], device="cuda")
    for layer in pool:
        layer.copy_(torch.randn(layer.shape, generator=g, device="cuda"))
    order = torch.randperm(2 * n + 3, generator=g, device="cuda").int()
    return {"kv_pool": pool, "src": order[:n].contiguous(), "dst": order[n:2 * n].contiguous(), "len": _i32(_copy_lengths(case)) if case["part"] else None}


def _prepare_compact(case, seed):
    rng, owned = np.random.default_rng(seed), _compact_lengths(case)
    name = rng.permutation(case["pages"])
    width, used = max(owned) + 2, sum(owned)
    begin = np.cumsum(owned) - owned
    col = np.arange(width)
    tables = np.where(col < np.asarray(owned)[:, None], name[(begin[:, None] + col).clip(0, case["pages"] - 1)], -1)
    if len(owned) > 1 and owned[0] and owned[1]:     # one page that two rows share
        tables[1, 0] = tables[0, 0]
        name[begin[1]], name[used - 1], used = name[used - 1], name[begin[1]], used - 1
        tables[tables == name[begin[1]]] = name[begin[1]]
    shares = np.zeros(case["pages"], dtype=np.int64)
    np.add.at(shares, tables[tables >= 0], 1)
    free = np.setdiff1d(np.arange(case["pages"]), tables[tables >= 0])
    rng.shuffle(free)
    capacity = case["pages"] - case["keep"]
    i = lambda: torch.empty(capacity, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"keep": case["keep"], "ctx_len": _i32([max(0, PAGE * n - 3) for n in owned]), "block_tables": _i32(tables), "shares": _i32((shares - 1).clip(0)),
            "free_list": _i32(np.concatenate([free, np.zeros(case["pages"] - len(free), dtype=np.int64)])), "free_count": _i32([len(free)]), "copy_src": i(),
            "copy_dst": i()}


def _prepare_attention(case, seed):
    g, (groups, own_keys) = _gen(seed), _attention_lengths(case)
    hq, hkv, dh, dt = case["hq"], case["hkv"], case["dh"], TYPES[case["type"]]
    tables, kv_len, begin, used = [], [], [0], 0     # tables: (shared pages, own pages) of every sequence
    for (m, shared), keys in zip(groups, own_keys):
        whole = shared // PAGE                       # pages that the group's sequences share: the prompt's whole ones
        for n in keys:
            mine = _pages(shared + n) - whole
            tables.append((whole, mine))
            kv_len.append(shared + n)
        begin.append(begin[-1] + m)
    width = max(a + b for a, b in tables) + 1
    rows, s = np.full((len(tables), width), -1, dtype=np.int64), 0
    for (m, shared), _ in zip(groups, own_keys):
        whole = shared // PAGE
        first, used = used, used + whole
        for _ in range(m):
            mine = tables[s][1]
            rows[s, :whole] = np.arange(first, first + whole)
            rows[s, whole:whole + mine] = np.arange(used, used + mine)
            used, s = used + mine, s + 1
    num_pages = used + 5
    name = torch.randperm(num_pages, generator=g, device="cuda").int()
    at = torch.tensor(rows, device="cuda")
    n = len(kv_len)
    slopes = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda", dtype=torch.float32) / hq) if case["bias"] else None
    return {"q": (3.0 * torch.randn(n, hq, dh, generator=g, device="cuda")).to(dt), "layer": 0,
            "kv_pool": torch.randn(1, 2, num_pages, hkv, PAGE, dh, generator=g, device="cuda").to(dt),
            "block_tables": torch.where(at >= 0, name[at.clamp(min=0)], torch.full_like(name[:1], -1)).contiguous(), "kv_len": _i32(kv_len), "group_begin": _i32(begin),
            "shared_len": _i32([shared for _, shared in groups]), "most": max(m for m, _ in groups), "most_shared": max(shared // PAGE for _, shared in groups),
            "most_own": max(b for _, b in tables), "slopes": slopes, "scale": dh ** -0.5, "cap": case["cap"], "o": torch.empty(n, hq, dh, dtype=dt, device="cuda"),
            "lse": torch.empty(n, hq, dtype=torch.float32, device="cuda")}


# --------------------------------------------------------------------------------------------------------- run
def run(state):
    if own:
        from paper_2608_01785_b200 import device_ops as ops
        return _own(ops, state)
    return {"select": _plain_select, "fork": _plain_fork, "copy": _plain_copy, "compact": _plain_compact, "attention": _plain_attention}[state["op"]](state)


def _own(ops, s):
    if s["op"] == "select":
        ops.beam_select(s["logits"], s["scores"], s["out_score"], s["out_parent"], s["out_token"], s["workspace"], s["status"], done=s["done"], weight=s["weight"],
                        out_done=s["out_done"], lse=s["lse"], end_token=s["end_token"], scale=s["scale"])
        return {k: s[k] for k in ("out_score", "out_parent", "out_token", "out_done", "lse")}
    if s["op"] == "fork":
        ops.fork_pages(s["parent"], s["ctx_len"], s["block_tables"], s["shares"], s["free_list"], s["free_count"], s["copy_src"], s["copy_dst"], s["copy_len"],
                       s["workspace"], s["status"])
        return {k: s[k] for k in ("ctx_len", "block_tables", "shares", "free_list", "free_count", "copy_src", "copy_dst", "copy_len")}
    if s["op"] == "copy":
        ops.copy_pages(s["kv_pool"], s["src"], s["dst"], s["status"], length=s["len"])
        return s["kv_pool"]
    if s["op"] == "compact":
        ops.compact_pages(s["keep"], s["ctx_len"], s["block_tables"], s["shares"], s["free_list"], s["free_count"], s["copy_src"], s["copy_dst"], s["workspace"],
                          s["status"])
        return {k: s[k] for k in ("block_tables", "shares", "free_list", "free_count", "copy_src", "copy_dst")}
    ops.shared_attention(s["q"], s["kv_pool"], s["layer"], s["block_tables"], s["kv_len"], s["group_begin"], s["shared_len"], s["o"], s["workspace"], s["status"],
                         lse=s["lse"], slopes=s["slopes"], scale=s["scale"], cap=s["cap"])
    return {"o": s["o"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------------- plain forms
def _plain_select(s):
    (n, b), v, k = s["scores"].shape, s["logits"].shape[1], s["out_score"].shape[1]
    x = s["logits"].double() * s["scale"]
    top = x.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(1, keepdim=True))
    s["lse"].copy_(lse[:, 0] if s["done"] is None else torch.where(s["done"].flatten() > 0, 0.0, lse[:, 0]))
    x = x - lse
    x = (x.view(n, b, v) + s["scores"].double()[..., None])
    if s["done"] is not None:                        # an ended beam has one continuation, itself
        itself = torch.where(torch.arange(v, device="cuda") == s["end_token"], s["scores"].double()[..., None], torch.full_like(x[:1, :1, :1], -math.inf))
        x = torch.where(s["done"][..., None] > 0, itself, x)
    rank = x if s["weight"] is None else x * s["weight"].double()[..., None]
    best = torch.sort(rank.view(n, -1), dim=1, descending=True, stable=True).indices[:, :k]
    beam, token = best // v, best % v
    score = x.view(n, -1).gather(1, best)
    some = score > -math.inf                         # fewer continuations than are asked for, where beams have ended
    over = token == s["end_token"]
    s["out_score"].copy_(score)
    s["out_parent"].copy_(torch.where(some, torch.arange(n, device="cuda")[:, None] * b + beam, -1))
    s["out_token"].copy_(torch.where(some, token, -1))
    s["out_done"].copy_(some & (over if s["done"] is None else over | (s["done"].gather(1, beam) > 0)))
    return {k: s[k] for k in ("out_score", "out_parent", "out_token", "out_done", "lse")}


def _plain_fork(s):
    parent, ctx, tables, free_list = s["parent"].long(), s["ctx_len"].long(), s["block_tables"].long(), s["free_list"]
    n, width = tables.shape
    row, col = torch.arange(n, device="cuda"), torch.arange(width, device="cuda")
    on, of = parent >= 0, parent.clamp(min=0)
    owned = (ctx + PAGE - 1) // PAGE
    first = torch.full((n,), n, device="cuda").scatter_reduce(0, of, torch.where(on, row, n), "amin")      # a row's first successor keeps its last page
    children = torch.zeros(n, dtype=torch.long, device="cuda").index_add_(0, of, on.long())
    full = col[None] < (ctx // PAGE)[:, None]
    tail = (col[None] == (ctx // PAGE)[:, None]) & (ctx % PAGE > 0)[:, None]
    delta = torch.where(full, children[:, None] - 1, 0) + torch.where(tail & (children == 0)[:, None], -1, 0)
    s["shares"].index_add_(0, tables.clamp(min=0).flatten(), delta.flatten().int())
    # rows and the pages of their copies
    length = torch.where(on, ctx[of], 0)
    copied = on & (length % PAGE > 0) & (first[of] != row)
    pop = s["free_count"].long() - torch.cumsum(copied, 0)
    fresh = torch.where(copied, free_list[pop.clamp(0, free_list.numel() - 1)].long(), -1)
    held = torch.where(on[:, None], tables[of], -1)
    at_tail = col[None] == (length // PAGE)[:, None]
    s["copy_src"].copy_(torch.where(copied, held.gather(1, (length // PAGE).clamp(max=width - 1)[:, None])[:, 0], -1))
    s["copy_dst"].copy_(fresh)
    s["copy_len"].copy_(torch.where(copied, length % PAGE, 0))
    mine = (length + PAGE - 1) // PAGE
    new = torch.where(copied[:, None] & at_tail, fresh[:, None], held)
    s["block_tables"].copy_(torch.where(col[None] < mine[:, None], new, torch.where(col[None] < owned[:, None], -1, tables)))
    s["ctx_len"].copy_(length)
    # pages that nobody holds any more, in rising order
    left = s["free_count"].long() - copied.sum()
    gone = s["shares"] < 0
    place = torch.where(gone, left + torch.cumsum(gone, 0) - 1, free_list.numel())
    longer = torch.cat([free_list, free_list[:1]])
    longer.scatter_(0, place, torch.where(gone, torch.arange(gone.numel(), device="cuda"), 0).int())
    free_list.copy_(longer[:-1])
    s["shares"].clamp_(min=0)
    s["free_count"].copy_(left + gone.sum())
    return {k: s[k] for k in ("ctx_len", "block_tables", "shares", "free_list", "free_count", "copy_src", "copy_dst", "copy_len")}


def _plain_copy(s):
    pool, src, dst = s["kv_pool"], s["src"].long(), s["dst"].long()
    if s["len"] is None:
        pool[:, :, dst] = pool[:, :, src]
    else:
        keep = (torch.arange(PAGE, device="cuda")[None] < s["len"][:, None]).view(1, 1, -1, 1, PAGE, 1)
        pool[:, :, dst] = torch.where(keep, pool[:, :, src], pool[:, :, dst])
    return pool


def _plain_compact(s):
    keep, n, free_list = s["keep"], s["free_list"].numel(), s["free_list"]
    page = torch.arange(n, device="cuda")
    free = torch.zeros(n + 1, dtype=torch.bool, device="cuda")
    free[torch.where(page < s["free_count"], free_list, n).long()] = True
    free = free[:n]
    low, moved = free & (page < keep), ~free & (page >= keep)
    moves = moved.sum()
    rank = lambda mask: torch.cumsum(mask, 0) - 1  # noqa: E731
    target = torch.full((n + 1,), -1, dtype=torch.long, device="cuda").scatter_(0, torch.where(low, rank(low), n), page)[:n]         # k-th free page below the bound
    source = torch.full((n + 1,), -1, dtype=torch.long, device="cuda").scatter_(0, torch.where(moved, rank(moved), n), page)[:n]
    to = torch.where(moved, target[rank(moved).clamp(min=0)], page)
    k = torch.arange(s["copy_src"].numel(), device="cuda")
    s["copy_src"].copy_(torch.where(k < moves, source[:k.numel()], -1))
    s["copy_dst"].copy_(torch.where(k < moves, target[:k.numel()], -1))
    col = torch.arange(s["block_tables"].shape[1], device="cuda")
    mine = col[None] < ((s["ctx_len"] + PAGE - 1) // PAGE)[:, None]
    s["block_tables"].copy_(torch.where(mine, to[s["block_tables"].long().clamp(min=0)], s["block_tables"].long()))
    shares = torch.zeros_like(s["shares"]).index_add_(0, to, s["shares"])
    s["shares"].copy_(shares)
    free = (low & (rank(low) >= moves)) | (page >= keep)                         # all of the upper end, and the lowest on top
    longer = torch.cat([free_list, free_list[:1]]).scatter_(0, torch.where(free, s["free_count"] - 1 - rank(free), n), page.int())
    free_list.copy_(longer[:-1])
    return {k: s[k] for k in ("block_tables", "shares", "free_list", "free_count", "copy_src", "copy_dst")}


def _plain_attention(s):
    n, hq, dh = s["q"].shape
    hkv = s["kv_pool"].shape[3]
    r = hq // hkv
    begin, kv = s["group_begin"].long(), s["kv_len"].long()
    groups = begin.numel() - 1
    seq = torch.arange(n, device="cuda")
    group = torch.searchsorted(begin[1:], seq, right=True)
    whole = (s["shared_len"].long() // PAGE)[group]                              # pages that a sequence shares
    tables = s["block_tables"].long()
    slopes = None if s["slopes"] is None else s["slopes"].view(1, hkv, r, 1)

    def scores(x, far, seen):                                                    # [n, hkv, r, keys], [n, keys], [n, keys]
        x = x * s["scale"]
        if s["cap"]:
            x = s["cap"] * torch.tanh(x / s["cap"])
        if slopes is not None:
            x = x - slopes * far[:, None, None].float()
        return x.masked_fill(~seen[:, None, None], -math.inf)

    def pages(which, at):                                                        # [rows, pages] -> [rows, hkv, keys, dh]
        return s["kv_pool"][s["layer"], which][at.clamp(min=0)].transpose(1, 2).flatten(2, 3).float()

    q = s["q"].float().view(n, hkv, r, dh)
    slot = seq - begin[group]                                                    # of a sequence in its group
    padded = torch.zeros(groups, s["most"], hkv, r, dh, device="cuda")
    padded[group, slot] = q
    common = tables[begin[:-1], :max(s["most_shared"], 1)]                       # the shared keys once per group, for all its rows
    x = torch.matmul(padded.permute(0, 2, 1, 3, 4).flatten(2, 3), pages(0, common).transpose(2, 3)).unflatten(2, (s["most"], r))
    x = x.permute(0, 2, 1, 3, 4)[group, slot]
    key = torch.arange(x.shape[-1], device="cuda")[None]
    x = scores(x, kv[:, None] - 1 - key, key < whole[:, None] * PAGE)
    col = whole[:, None] + torch.arange(s["most_own"], device="cuda")[None]      # the others of each sequence
    mine = tables.gather(1, col.clamp(max=tables.shape[1] - 1))
    key = whole[:, None] * PAGE + torch.arange(s["most_own"] * PAGE, device="cuda")[None]
    y = scores(torch.matmul(q, pages(0, mine).transpose(2, 3)), kv[:, None] - 1 - key, key < kv[:, None])
    top = torch.maximum(x.amax(-1, keepdim=True), y.amax(-1, keepdim=True))
    x, y = torch.exp(x - top), torch.exp(y - top)
    total = x.sum(-1, keepdim=True) + y.sum(-1, keepdim=True)
    padded = torch.zeros(groups, s["most"], hkv, r, x.shape[-1], device="cuda")
    padded[group, slot] = x
    o = torch.matmul(padded.permute(0, 2, 1, 3, 4).flatten(2, 3), pages(1, common)).unflatten(2, (s["most"], r)).permute(0, 2, 1, 3, 4)[group, slot]
    o = (o + torch.matmul(y, pages(1, mine))) / total
    s["o"].copy_(o.reshape(n, hq, dh))
    s["lse"].copy_((top + torch.log(total)).view(n, hq))
    return {"o": s["o"], "lse": s["lse"]}


# -------------------------------------------------------------------------------------------------------- work
def work(case):
    if case["op"] == "select":
        rows = case["requests"] * case["beams"]
        read = rows * (0.875 if case["ended"] else 1) * case["vocab"]             # (an ended beam's logits are not looked at)
        return {"bytes": int(read * TYPES[case["type"]].itemsize) + rows * (16 if case["ended"] else 8) + 16 * case["requests"] * case["out"], "flops": int(4 * read)}
    if case["op"] == "fork":
        lens = _fork_lengths(case)
        return {"bytes": 4 * (2 * sum(_pages(n) for n in lens) + 6 * len(lens)), "flops": 0}
    if case["op"] == "copy":
        return {"bytes": case["layers"] * 2 * sum(_copy_lengths(case)) * case["hkv"] * case["dh"] * 2 * 2 + 12 * case["pages"], "flops": 0}
    if case["op"] == "compact":
        used = sum(_compact_lengths(case))
        moves = int((case["pages"] - case["keep"]) * used / case["pages"])
        return {"bytes": 4 * (2 * used + 2 * (case["pages"] - used) + 6 * moves), "flops": 0}
    groups, own_keys = _attention_lengths(case)
    keys = pairs = n = 0
    for (m, shared), mine in zip(groups, own_keys):
        whole = shared // PAGE * PAGE
        behind = sum(shared - whole + k for k in mine)
        keys += whole + behind
        pairs += m * whole + behind
        n += m
    return {"bytes": keys * case["hkv"] * case["dh"] * 4 + n * case["hq"] * (4 * case["dh"] + 4), "flops": 4 * pairs * case["hq"] * case["dh"]}


# ------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"select": _exact_select, "fork": _exact_fork, "copy": _exact_copy, "compact": _exact_compact, "attention": _exact_attention}[case["op"]](case, s)


def _exact_select(case, s):
    n, b, v, k = case["requests"], case["beams"], case["vocab"], case["out"]
    out = {key: np.full((n, k), of, dtype=np.float64 if key == "out_score" else np.int32)
           for key, of in (("out_score", -np.inf), ("out_parent", -1), ("out_token", -1), ("out_done", 0))}
    scores = s["scores"].double().cpu().numpy()
    done = s["done"].cpu().numpy() if case["ended"] else np.zeros((n, b), dtype=int)
    weight = s["weight"].double().cpu().numpy() if case["ended"] else np.ones((n, b))
    out["lse"] = np.zeros(n * b)
    for r in range(n):
        found = []
        out["lse"][r * b:(r + 1) * b] = np.where(done[r] > 0, 0.0, torch.logsumexp(s["logits"][r * b:(r + 1) * b].double() * s["scale"], 1).cpu().numpy())
        lp = torch.log_softmax(s["logits"][r * b:(r + 1) * b].double() * s["scale"], 1)
        order = torch.argsort(-s["logits"][r * b:(r + 1) * b].double(), dim=1, stable=True)[:, :k]
        lp, order = lp.gather(1, order).cpu().numpy(), order.cpu().numpy()
        for i in range(b):
            if done[r, i]:
                found.append((-scores[r, i] * weight[r, i], i, s["end_token"], scores[r, i]))
            else:
                found += [(-(scores[r, i] + p) * weight[r, i], i, int(t), scores[r, i] + p) for p, t in zip(lp[i], order[i])]
        for j, (_, i, t, score) in enumerate(sorted(found)[:k]):
            out["out_score"][r, j], out["out_parent"][r, j], out["out_token"][r, j] = score, r * b + i, t
            out["out_done"][r, j] = bool(done[r, i]) or t == s["end_token"]
    return out


def _exact_fork(case, s):
    parent, ctx, old = s["parent"].tolist(), s["ctx_len"].tolist(), s["block_tables"].cpu().numpy()
    n, new, free = len(parent), old.copy(), s["free_list"].tolist()
    top, holders = int(s["free_count"].item()), s["shares"].cpu().numpy() + 1
    listed_free = set(free[:top])
    src, dst, length, kept = [-1] * n, [-1] * n, [0] * n, set()
    for i in range(n):
        own_pages = [int(p) for p in old[i, :_pages(ctx[i])]]
        for p in own_pages:
            holders[p] -= 1
        new[i, :len(own_pages)] = -1
    for i, p in enumerate(parent):
        if p < 0:
            continue
        pages = [int(x) for x in old[p, :_pages(ctx[p])]]
        if ctx[p] % PAGE and p in kept:
            top -= 1
            src[i], dst[i], length[i] = pages[-1], free[top], ctx[p] % PAGE
            pages[-1] = free[top]
            listed_free.discard(free[top])
        kept.add(p)
        new[i, :len(pages)] = pages
        if dst[i] < 0:
            holders[pages] += 1
        else:
            holders[pages[:-1]] += 1                # (a free page counts as held once, and is held once now)
    for page in range(len(holders)):
        if holders[page] == 0 and page not in listed_free:
            free[top] = page
            top += 1
            holders[page] = 1
    a = lambda x: np.asarray(x, dtype=np.int32)  # noqa: E731
    return {"ctx_len": a([ctx[p] if p >= 0 else 0 for p in parent]), "block_tables": a(new), "shares": a(holders - 1), "free_list": a(free), "free_count": a([top]),
            "copy_src": a(src), "copy_dst": a(dst), "copy_len": a(length)}


def _exact_copy(case, s):
    pool = s["kv_pool"].clone()
    for a, b, n in zip(s["src"].tolist(), s["dst"].tolist(), _copy_lengths(case)):
        pool[:, :, b, :, :n] = s["kv_pool"][:, :, a, :, :n]
    return pool.double() if pool.numel() < 1 << 28 else pool


def _exact_compact(case, s):
    keep, free, top = case["keep"], s["free_list"].cpu().numpy(), int(s["free_count"].item())
    is_free = set(free[:top].tolist())
    low = sorted(p for p in is_free if p < keep)
    source = [p for p in range(keep, case["pages"]) if p not in is_free]
    to = dict(zip(source, low))
    tables, shares = s["block_tables"].cpu().numpy().copy(), s["shares"].cpu().numpy().copy()
    flat = tables.reshape(-1)
    flat[:] = [to.get(int(p), int(p)) for p in flat]
    for a, b in to.items():
        shares[b], shares[a] = shares[a], 0
    free[:top] = sorted(low[len(source):] + list(range(keep, case["pages"])), reverse=True)
    pad = [-1] * (case["pages"] - keep - len(source))
    a = lambda x: np.asarray(x, dtype=np.int32)  # noqa: E731
    return {"block_tables": a(tables), "shares": a(shares), "free_list": a(free), "free_count": a([top]), "copy_src": a(source + pad),
            "copy_dst": a(low[:len(source)] + pad)}


def _exact_attention(case, s):
    hq, hkv = case["hq"], case["hkv"]
    o, lse = [], []
    for i, kv in enumerate(s["kv_len"].tolist()):
        at = s["block_tables"][i, :_pages(kv)].long()
        k, v = (s["kv_pool"][0, w][at].double().permute(1, 0, 2, 3).reshape(hkv, -1, case["dh"])[:, :kv].repeat_interleave(hq // hkv, 0) for w in (0, 1))
        x = torch.einsum("hd,hkd->hk", s["q"][i].double(), k) / math.sqrt(case["dh"])
        if case["cap"]:
            x = torch.tanh(x / case["cap"]) * case["cap"]
        if case["bias"]:
            x = x - (2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda", dtype=torch.float64) / hq))[:, None] * (kv - 1 - torch.arange(kv, device="cuda"))
        lse.append(torch.logsumexp(x, 1))
        o.append(torch.einsum("hk,hkd->hd", torch.softmax(x, 1), v))
    return {"o": torch.stack(o), "lse": torch.stack(lse)}
