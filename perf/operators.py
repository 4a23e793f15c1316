"""Cases of the operators whose lengths, positions and page tables stay on the device, with their plain forms.

Four operators that a decoding loop calls one after the other without a word from the host:

  tables      page allocation, token -> (sequence, position, cache slot) from the requests' lengths
  rope        rotary positions on q and k, and the scatter of k and v into the paged cache
  attention   attention over the paged cache with capped scores, a distance bias, a window and a prefix; one new token per
              sequence ("decode") or chunks of new tokens ("chunk")
  logprobs    log probability and rank of given tokens, entropy and the top alternatives of logit rows

The plain forms are elementary torch operations in 32 bits, rounded once at the end.  The layout of the cache is the
library's: [layer][K or V][page][kv head][16][head_dim].
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
WORKSPACE_BYTES = 32 << 20     # what the operators' header asks for, whatever the sizes
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # a decode tick: every one of 64 requests grows by one token, a sixteenth of them into a new page
        {"name": "tables_decode_64", "op": "tables", "seqs": 64, "ctx_lo": 512, "ctx_hi": 4096, "chunks": 0, "chunk_hi": 1, "mix": 1},
        # a busy mixed tick: 1000 requests, 24 of them with prompt chunks of up to 1024 tokens
        {"name": "tables_mixed_1000", "op": "tables", "seqs": 1000, "ctx_lo": 0, "ctx_hi": 4096, "chunks": 24, "chunk_hi": 1024, "mix": 2},
        # the projections of 64 decode rows at the 7B dimensions, fp32 accumulators as the GEMM leaves them
        {"name": "rope_decode_64", "op": "rope", "tokens": 64, "hq": 28, "hkv": 4, "dh": 128, "rot": 128, "interleaved": False,
         "scaling": "none", "src": "f32", "dst": "bf16", "chunk": 1, "mix": 3},
        # a tick of the talker's dimensions with interleaved pairs on half of each head, an odd number of rows
        {"name": "rope_talker_1111", "op": "rope", "tokens": 1111, "hq": 16, "hkv": 4, "dh": 64, "rot": 32, "interleaved": True,
         "scaling": "linear", "src": "f16", "dst": "f16", "chunk": 101, "mix": 4},
        # prompts at the 7B dimensions, positions of a context stretched by parts
        {"name": "rope_prompt_8000", "op": "rope", "tokens": 8000, "hq": 28, "hkv": 4, "dh": 128, "rot": 128, "interleaved": False,
         "scaling": "by_parts", "src": "bf16", "dst": "bf16", "chunk": 2000, "mix": 5},
        # decode of the talker: 16 short sequences, latency
        {"name": "decode_talker_16", "op": "attention", "seqs": 16, "hq": 16, "hkv": 4, "dh": 64, "type": "bf16", "q_lo": 1, "q_hi": 1,
         "kv_lo": 128, "kv_hi": 1024, "cap": 30.0, "window": 0, "prefix": 0, "bias": False, "mix": 6},
        # decode at the 7B dimensions with capped scores: the cache's bytes
        {"name": "decode_7b_64", "op": "attention", "seqs": 64, "hq": 28, "hkv": 4, "dh": 128, "type": "bf16", "q_lo": 1, "q_hi": 1,
         "kv_lo": 512, "kv_hi": 4096, "cap": 50.0, "window": 0, "prefix": 0, "bias": False, "mix": 7},
        # few long documents with a distance bias, fp16 cache: work split over the cache's length
        {"name": "decode_long_3", "op": "attention", "seqs": 3, "hq": 16, "hkv": 2, "dh": 128, "type": "f16", "q_lo": 1, "q_hi": 1,
         "kv_lo": 20001, "kv_hi": 32768, "cap": 0.0, "window": 0, "prefix": 0, "bias": True, "mix": 8},
        # eight prompt chunks under a sliding window of 512 keys with capped scores
        {"name": "chunk_window_8", "op": "attention", "seqs": 8, "hq": 16, "hkv": 2, "dh": 128, "type": "bf16", "q_lo": 128, "q_hi": 1024,
         "kv_lo": 128, "kv_hi": 2048, "cap": 50.0, "window": 512, "prefix": 0, "bias": False, "mix": 9},
        # a long prompt's second chunk at the 7B dimensions behind an image prefix that every token sees
        {"name": "chunk_prefix_1", "op": "attention", "seqs": 1, "hq": 28, "hkv": 4, "dh": 128, "type": "bf16", "q_lo": 2048, "q_hi": 2048,
         "kv_lo": 4095, "kv_hi": 4095, "cap": 50.0, "window": 0, "prefix": 576, "bias": False, "mix": 10},
        # sampled tokens of a decode tick with twenty alternatives, fp32 logits as the head leaves them
        {"name": "logprobs_decode_64", "op": "logprobs", "rows": 64, "vocab": 152064, "type": "f32", "top": 20, "mix": 11},
        # prompt scoring: every row of a chunk, bf16 logits
        {"name": "logprobs_prompt_2047", "op": "logprobs", "rows": 2047, "vocab": 152064, "type": "bf16", "top": 5, "mix": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tables", "rope", "decode", "decode", "chunk", "logprobs"))
    mix = rng.randrange(1 << 30)
    if op == "tables":
        n = _log(rng, 1, 1000)
        chunks = rng.randrange(0, min(n, 24) + 1)
        return {"op": "tables", "seqs": n, "ctx_lo": 0, "ctx_hi": _log(rng, 16, 4096), "chunks": chunks, "chunk_hi": _log(rng, 2, 1024), "mix": mix}
    if op == "rope":
        dh = rng.choice((64, 128))
        hkv = rng.choice((1, 2, 4, 8))
        return {"op": "rope", "tokens": _log(rng, 1, 8000), "hq": hkv * rng.choice((1, 2, 4, 7)), "hkv": hkv, "dh": dh,
                "rot": rng.choice((dh, dh // 2)), "interleaved": rng.random() < 0.5, "scaling": rng.choice(("none", "linear", "by_parts")),
                "src": rng.choice(("f32", "bf16", "f16")), "dst": rng.choice(("bf16", "f16")), "chunk": _log(rng, 1, 2000), "mix": mix}
    if op in ("decode", "chunk"):
        dh = rng.choice((64, 128))
        hq, hkv = rng.choice(((28, 4), (16, 2), (16, 4), (16, 16), (12, 1), (5, 5)))
        case = {"op": "attention", "hq": hq, "hkv": hkv, "dh": dh, "type": rng.choice(("bf16", "f16")), "cap": rng.choice((0.0, 30.0, 50.0)),
                "window": rng.choice((0, 0, _log(rng, 64, 2048))), "prefix": rng.choice((0, 0, _log(rng, 4, 600))), "bias": rng.random() < 0.4, "mix": mix}
        if op == "decode":
            hi = _log(rng, 64, 32768)
            most = max(1, min(64, 200000 * 16 // (hi * max(hkv, 4))))
            return dict(case, seqs=_log(rng, 1, most), q_lo=1, q_hi=1, kv_lo=max(1, hi // rng.choice((1, 4, 16))), kv_hi=hi)
        q_hi = _log(rng, 2, 1024)
        return dict(case, seqs=_log(rng, 1, max(1, 4096 // q_hi if q_hi > 400 else 10)), q_lo=max(1, q_hi // rng.choice((1, 8))), q_hi=q_hi,
                    kv_lo=q_hi, kv_hi=q_hi + _log(rng, 1, 2048))
    v = rng.choice((152064, _log(rng, 1000, 152064)))
    return {"op": "logprobs", "rows": _log(rng, 1, 2047), "vocab": v, "type": rng.choice(("f32", "bf16", "f16")) if v < 40000 else rng.choice(("f32", "bf16")),
            "top": rng.choice((0, 1, 5, 20)), "mix": mix} if rng.random() < 0.7 else {
            "op": "logprobs", "rows": _log(rng, 1, 64), "vocab": v, "type": "f32", "top": rng.choice((1, 5, 20)), "mix": mix}


# ------------------------------------------------------------------------------------------- lengths of a case
def _pages(n):
    return -(-n // PAGE)


def _table_lengths(case):
    r = random.Random(case["mix"])
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    q = [1] * case["seqs"]
    for s in r.sample(range(case["seqs"]), case["chunks"]):
        q[s] = r.randint(1, case["chunk_hi"])
    return ctx, q


def _attention_lengths(case):
    """(new tokens, keys with them) of each sequence."""
    r = random.Random(case["mix"])
    q = [r.randint(case["q_lo"], case["q_hi"]) for _ in range(case["seqs"])]
    return q, [max(n, r.randint(case["kv_lo"], case["kv_hi"])) for n in q]


def _rope_lengths(case):
    """Token counts and first positions of the sequences that the rows belong to."""
    r, left, parts = random.Random(case["mix"]), case["tokens"], []
    while left > 0:
        n = min(left, r.randint(max(1, case["chunk"] // 2), case["chunk"]))
        parts.append((n, r.randint(0, 4096)))
        left -= n
    return parts


# ------------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 17)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _common(st):
    st["workspace"] = torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return st


def _random_tables(g, pages, width, num_pages):
    """Block tables of sequences that own `pages` pages each, -1 behind them, and the free pages, in a random order."""
    order = torch.randperm(num_pages, generator=g, device="cuda").to(torch.int32)
    owned = _i32(pages)
    begin = torch.cumsum(owned, 0, dtype=torch.int32) - owned
    col = torch.arange(width, device="cuda", dtype=torch.int32)
    at = (begin[:, None] + col[None]).clamp(max=num_pages - 1).long()
    return torch.where(col[None] < owned[:, None], order[at], torch.full_like(col, -1)[None]), order[sum(pages):].contiguous()


def prepare(case, seed):
    return _common({"tables": _prepare_tables, "rope": _prepare_rope, "attention": _prepare_attention, "logprobs": _prepare_logprobs}[case["op"]](case, _gen(seed)))


def _prepare_tables(case, g):
    ctx, q = _table_lengths(case)
    pages = [_pages(c) for c in ctx]
    after = [_pages(c + n) for c, n in zip(ctx, q)]
    width, tokens = max(after) + 3, sum(q)
    max_tokens = _pages(tokens) * PAGE               # a captured step has room for a whole number of tiles
    num_pages = sum(after) + 100
    tables, free = _random_tables(g, pages, width, num_pages)
    empty = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"op": "tables", "ctx_len": _i32(ctx), "q_len": _i32(q), "block_tables": tables.contiguous(),
            "free_list": torch.cat([free, torch.zeros(num_pages - free.numel(), dtype=torch.int32, device="cuda")]), "free_count": _i32([free.numel()]),
            "num_pages": num_pages, "max_tokens": max_tokens, "kv_len": empty(len(q)), "tok_begin": empty(len(q) + 1), "tok_seq": empty(max_tokens),
            "tok_pos": empty(max_tokens), "tok_slot": empty(max_tokens), "free_count_out": empty(1)}


def _frequencies(case):
    """Angles per position of the rotated pairs in 64 bits, and the factor on both cos and sin."""
    rot, base, factor, trained = case["rot"], 10000.0, 4.0, 4096
    inv = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if case["scaling"] == "linear":
        return inv / factor, 1.0
    if case["scaling"] == "by_parts":                # slow pairs are stretched, fast ones are not, a ramp between
        turns = trained * inv / (2 * math.pi)
        keep = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        return inv * keep + inv / factor * (1 - keep), 0.1 * math.log(factor) + 1.0
    return inv, 1.0


def _prepare_rope(case, g):
    parts, dt = _rope_lengths(case), TYPES[case["dst"]]
    hq, hkv, dh, t = case["hq"], case["hkv"], case["dh"], case["tokens"]
    max_position = max(p + n for n, p in parts)
    inv, mag = _frequencies(case)
    angle = torch.arange(max_position, device="cuda", dtype=torch.float64)[:, None] * torch.from_numpy(inv).cuda()[None]
    rope = torch.stack([angle.cos() * mag, angle.sin() * mag], -1).float().contiguous()
    pages = [_pages(p + n) for n, p in parts]
    num_pages = sum(pages) + 5
    tables, _ = _random_tables(g, pages, max(pages), num_pages)
    seq = torch.repeat_interleave(torch.arange(len(parts), device="cuda"), torch.tensor([n for n, _ in parts], device="cuda"))
    first = torch.tensor([p for _, p in parts], device="cuda")
    begin = torch.tensor(np.concatenate([[0], np.cumsum([n for n, _ in parts])[:-1]]), device="cuda")
    pos = first[seq] + torch.arange(t, device="cuda") - begin[seq]
    slot = tables[seq, pos // PAGE].long() * PAGE + pos % PAGE
    if t > 32:
        slot[-3:] = -1                               # rows that pad a captured step: rotated, not stored
    qkv = torch.randn(t, (hq + 2 * hkv) * dh, generator=g, device="cuda").to(TYPES[case["src"]])
    return {"op": "rope", "q": qkv[:, :hq * dh].unflatten(1, (hq, dh)), "k": qkv[:, hq * dh:(hq + hkv) * dh].unflatten(1, (hkv, dh)),
            "v": qkv[:, (hq + hkv) * dh:].unflatten(1, (hkv, dh)), "tok_pos": pos.int(), "tok_slot": slot.int(), "rope": rope,
            "rot": case["rot"], "interleaved": case["interleaved"], "layer": 1,
            "kv_pool": torch.randn(2, 2, num_pages, hkv, PAGE, dh, generator=g, device="cuda").to(dt), "q_out": torch.empty(t, hq, dh, dtype=dt, device="cuda")}


def _prepare_attention(case, g):
    q_len, kv_len = _attention_lengths(case)
    hq, hkv, dh, dt = case["hq"], case["hkv"], case["dh"], TYPES[case["type"]]
    pages = [_pages(n) for n in kv_len]
    num_pages = sum(pages) + 5
    tables, _ = _random_tables(g, pages, max(pages), num_pages)
    t = sum(q_len)
    slopes = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda", dtype=torch.float32) / hq) if case["bias"] else None
    return {"op": "attention", "q": (3.0 * torch.randn(t, hq, dh, generator=g, device="cuda")).to(dt), "layer": 0,
            "kv_pool": torch.randn(1, 2, num_pages, hkv, PAGE, dh, generator=g, device="cuda").to(dt), "block_tables": tables.contiguous(),
            "kv_len": _i32(kv_len), "tok_begin": _i32([0] + list(np.cumsum(q_len))), "max_q_len": max(q_len), "max_kv_len": max(kv_len),
            "prefix_len": _i32([min(case["prefix"], n) for n in kv_len]) if case["prefix"] else None, "slopes": slopes, "scale": dh ** -0.5, "cap": case["cap"],
            "window": case["window"], "o": torch.empty(t, hq, dh, dtype=dt, device="cuda"), "lse": torch.empty(t, hq, dtype=torch.float32, device="cuda")}


def _prepare_logprobs(case, g):
    n, v, dt = case["rows"], case["vocab"], TYPES[case["type"]]
    x = torch.empty(n, v, dtype=dt, device="cuda")
    for i in range(0, n, 256):                       # a trained head's logits: a broad body and a few strong candidates per row
        part = 2.0 * torch.randn(min(256, n - i), v, generator=g, device="cuda")
        part += 12.0 * (torch.rand(part.shape, generator=g, device="cuda") < 8.0 / v)
        x[i:i + 256] = part.to(dt)
    targets = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    if n > 1:
        targets[-1] = -1                             # a prompt's last row has no next token
    k = case["top"]
    f = lambda *s: torch.empty(*s, dtype=torch.float32, device="cuda")  # noqa: E731
    i = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"op": "logprobs", "logits": x, "targets": targets, "top": k, "scale": 1.25, "logprob": f(n), "entropy": f(n), "rank": i(n),
            "top_ids": i(n, k) if k else None, "top_logprobs": f(n, k) if k else None}


# --------------------------------------------------------------------------------------------------------- run
def run(state):
    if own:
        from paper_2608_01785_b200 import device_ops as ops
        return _own(ops, state)
    return {"tables": _plain_tables, "rope": _plain_rope, "attention": _plain_attention, "logprobs": _plain_logprobs}[state["op"]](state)


def _own(ops, s):
    if s["op"] == "tables":
        ops.step_tables(s["ctx_len"], s["q_len"], s["free_list"], s["free_count"], s["block_tables"], s["kv_len"], s["tok_begin"], s["tok_seq"],
                        s["tok_pos"], s["tok_slot"], s["free_count_out"], s["workspace"], s["status"])
        return {k: s[k] for k in ("kv_len", "tok_begin", "tok_seq", "tok_pos", "tok_slot", "block_tables", "free_count_out")}
    if s["op"] == "rope":
        ops.rope_cache(s["q"], s["k"], s["v"], s["tok_pos"], s["tok_slot"], s["rope"], s["q_out"], s["kv_pool"], s["layer"], s["status"],
                       interleaved=s["interleaved"])
        return {"q": s["q_out"], "cache": s["kv_pool"][s["layer"]]}
    if s["op"] == "attention":
        ops.paged_attention(s["q"], s["kv_pool"], s["layer"], s["block_tables"], s["kv_len"], s["o"], s["workspace"], s["status"], lse=s["lse"],
                            tok_begin=s["tok_begin"], max_q_len=s["max_q_len"], prefix_len=s["prefix_len"], slopes=s["slopes"], scale=s["scale"],
                            cap=s["cap"], window=s["window"])
        return {"o": s["o"], "lse": s["lse"]}
    ops.token_logprobs(s["logits"], s["targets"], s["logprob"], s["workspace"], s["status"], entropy=s["entropy"], rank=s["rank"], top_ids=s["top_ids"],
                       top_logprobs=s["top_logprobs"], scale=s["scale"])
    return {k: s[k] for k in ("logprob", "entropy", "rank", "top_ids", "top_logprobs") if s[k] is not None}


# ------------------------------------------------------------------------------------------------- plain forms
def _plain_tables(s):
    ctx, q, mt = s["ctx_len"], s["q_len"], s["max_tokens"]
    owned, kv = (ctx + PAGE - 1) // PAGE, ctx + q
    need = (kv + PAGE - 1) // PAGE - owned
    tok_end, page_begin = torch.cumsum(q, 0), torch.cumsum(need, 0) - need
    col = torch.arange(s["block_tables"].shape[1], device="cuda")
    new = (col[None] >= owned[:, None]) & (col[None] < (owned + need)[:, None])
    pop = s["free_count"].long() - 1 - (page_begin[:, None] + col[None] - owned[:, None])
    tables = torch.where(new, s["free_list"][pop.clamp(0, s["num_pages"] - 1)], s["block_tables"])
    t = torch.arange(mt, device="cuda")
    real = t < tok_end[-1]
    seq = torch.searchsorted(tok_end, t, right=True).clamp(max=ctx.numel() - 1)
    pos = ctx[seq] + t - (tok_end - q)[seq]
    slot = tables[seq, (pos // PAGE).clamp(0, tables.shape[1] - 1)].long() * PAGE + pos % PAGE
    mark = lambda x: torch.where(real, x, torch.full_like(x, -1)).int()  # noqa: E731
    return {"kv_len": kv, "tok_begin": torch.cat([torch.zeros_like(tok_end[:1]), tok_end]).int(), "tok_seq": mark(seq), "tok_pos": mark(pos),
            "tok_slot": mark(slot), "block_tables": tables, "free_count_out": (s["free_count"] - need.sum()).int()}


def _rotate(x, c, sn, rot, interleaved):
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    lo, hi = a * c - b * sn, a * sn + b * c
    r = torch.stack([lo, hi], -1).flatten(-2) if interleaved else torch.cat([lo, hi], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _plain_rope(s):
    cs = s["rope"][s["tok_pos"].long()][:, None]
    c, sn = cs[..., 0], cs[..., 1]
    dt = s["q_out"].dtype
    s["q_out"].copy_(_rotate(s["q"].float(), c, sn, s["rot"], s["interleaved"]).to(dt))
    keep = s["tok_slot"] >= 0
    slot = s["tok_slot"][keep].long()
    cache = s["kv_pool"][s["layer"]]
    cache[0][slot // PAGE, :, slot % PAGE] = _rotate(s["k"].float(), c, sn, s["rot"], s["interleaved"]).to(dt)[keep]
    cache[1][slot // PAGE, :, slot % PAGE] = s["v"].float().to(dt)[keep]
    return {"q": s["q_out"], "cache": cache}


def _plain_attention(s):
    n, lq, lk = s["kv_len"].numel(), s["max_q_len"], s["max_kv_len"]
    t, hq, dh = s["q"].shape
    hkv = s["kv_pool"].shape[3]
    begin, end, kv = s["tok_begin"][:-1].long(), s["tok_begin"][1:].long(), s["kv_len"].long()
    j = torch.arange(lq, device="cuda")
    row = begin[:, None] + j[None]                                               # [n, lq] token rows, padded
    real = row < end[:, None]
    row = row.clamp(max=t - 1)
    pos = kv[:, None] - (end - begin)[:, None] + j[None]                         # absolute positions
    tables = s["block_tables"].long().clamp(min=0)
    keys = s["kv_pool"][s["layer"], 0][tables].transpose(2, 3).flatten(1, 2)[:, :lk].float()
    values = s["kv_pool"][s["layer"], 1][tables].transpose(2, 3).flatten(1, 2)[:, :lk].float()
    q = s["q"][row].float().unflatten(2, (hkv, hq // hkv))                       # [n, lq, hkv, g, dh]
    x = torch.matmul(q.permute(0, 2, 3, 1, 4).flatten(2, 3), keys.permute(0, 2, 3, 1)).unflatten(2, (hq // hkv, lq)) * s["scale"]
    if s["cap"]:
        x = s["cap"] * torch.tanh(x / s["cap"])
    key = torch.arange(keys.shape[1], device="cuda")
    far = pos[:, :, None] - key[None, None]                                      # [n, lq, lk]
    if s["slopes"] is not None:
        x = x - s["slopes"].view(1, hkv, -1, 1, 1) * far.abs()[:, None, None].float()
    seen = far >= 0
    if s["window"]:
        seen &= far < s["window"]
    if s["prefix_len"] is not None:
        seen |= (key[None] < s["prefix_len"][:, None])[:, None]
    seen &= (key[None] < kv[:, None])[:, None]
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), values.transpose(1, 2)).unflatten(2, (hq // hkv, lq)) / total.clamp(min=1e-30)
    lse = (top + torch.log(total))[..., 0]
    pick = real.flatten().nonzero()[:, 0] if lq > 1 else slice(None)
    o = o.permute(0, 3, 1, 2, 4).reshape(n * lq, hq, dh)[pick]
    return {"o": o.to(s["o"].dtype), "lse": lse.permute(0, 3, 1, 2).reshape(n * lq, hq)[pick].contiguous()}


def _plain_logprobs(s):
    x, t = s["logits"].float() * s["scale"], s["targets"].long()
    raw = s["logits"].float()
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1)
    lse = top[:, 0] + torch.log(total)
    entropy = torch.log(total) - (e * (x - top)).sum(1) / total
    some, at = t >= 0, t.clamp(min=0)[:, None]
    out = {"logprob": torch.where(some, x.gather(1, at)[:, 0] - lse, torch.zeros_like(lse)), "entropy": entropy,
           "rank": torch.where(some, (raw > raw.gather(1, at)).sum(1), torch.full_like(t, -1)).int()}
    if s["top"]:
        order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :s["top"]]
        out["top_ids"] = order.int()
        out["top_logprobs"] = x.gather(1, order) - lse[:, None]
    return out


# -------------------------------------------------------------------------------------------------------- work
def _visible(case):
    """Pairs (token, key) that the mask leaves, and keys that some token of their sequence sees."""
    pairs = keys = 0
    for q, kv in zip(*_attention_lengths(case)):
        pos = np.arange(kv - q, kv, dtype=np.int64)
        prefix = min(case["prefix"], kv)
        lo = np.maximum(pos - case["window"] + 1, 0) if case["window"] else np.zeros_like(pos)
        pairs += int((np.maximum(pos + 1 - np.maximum(lo, prefix), 0) + prefix).sum())
        keys += prefix + max(0, kv - max(int(lo[0]), prefix))
    return pairs, keys


def work(case):
    if case["op"] == "tables":
        ctx, q = _table_lengths(case)
        n, t = len(q), sum(q)
        new = sum(_pages(c + m) - _pages(c) for c, m in zip(ctx, q))
        return {"bytes": 4 * (2 * n + 2 * n + 3 * _pages(t) * PAGE + 2 * new + n), "flops": 0}
    if case["op"] == "rope":
        src, dst = TYPES[case["src"]].itemsize, TYPES[case["dst"]].itemsize
        row = (case["hq"] + 2 * case["hkv"]) * case["dh"]
        return {"bytes": case["tokens"] * (row * (src + dst) + 8 + 4 * case["rot"]), "flops": 3 * case["tokens"] * (case["hq"] + case["hkv"]) * case["rot"]}
    if case["op"] == "attention":
        pairs, keys = _visible(case)
        t = sum(_attention_lengths(case)[0])
        return {"bytes": keys * case["hkv"] * case["dh"] * 4 + t * case["hq"] * (4 * case["dh"] + 4), "flops": 4 * pairs * case["hq"] * case["dh"]}
    return {"bytes": case["rows"] * (case["vocab"] * TYPES[case["type"]].itemsize + 16 + 8 * case["top"]), "flops": 6 * case["rows"] * case["vocab"]}


# ------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _exact_tables, "rope": _exact_rope, "attention": _exact_attention, "logprobs": _exact_logprobs}[case["op"]](case, s)


def _exact_tables(case, s):
    ctx, q = _table_lengths(case)
    tables, free = s["block_tables"].cpu().numpy().copy(), s["free_list"].cpu().numpy()
    left = int(s["free_count"].item())
    seq, pos, slot, begin = [], [], [], [0]
    for i, (c, n) in enumerate(zip(ctx, q)):
        for page in range(_pages(c), _pages(c + n)):
            left -= 1
            tables[i, page] = free[left]
        for p in range(c, c + n):
            seq.append(i)
            pos.append(p)
            slot.append(int(tables[i, p // PAGE]) * PAGE + p % PAGE)
        begin.append(begin[-1] + n)
    pad = [-1] * (s["max_tokens"] - len(seq))
    a = lambda v: np.array(v, dtype=np.int32)  # noqa: E731
    return {"kv_len": a([c + n for c, n in zip(ctx, q)]), "tok_begin": a(begin), "tok_seq": a(seq + pad), "tok_pos": a(pos + pad), "tok_slot": a(slot + pad),
            "block_tables": tables, "free_count_out": a([left])}


def _exact_rope(case, s):
    table, pos = s["rope"].double(), s["tok_pos"].long()
    z = torch.complex(table[pos, :, 0], table[pos, :, 1])[:, None]               # a pair turns by multiplication with cos + i sin
    rot = case["rot"]

    def turn(x):
        x = x.double().clone()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        w = torch.complex(x[..., first], x[..., second]) * z
        x[..., first], x[..., second] = w.real, w.imag
        return x

    cache = s["kv_pool"][s["layer"]].double()
    slots, k, v = s["tok_slot"].tolist(), turn(s["k"]), s["v"].double()
    rows = [i for i, x in enumerate(slots) if x >= 0]
    pages, offsets = [slots[i] // PAGE for i in rows], [slots[i] % PAGE for i in rows]
    cache[0, pages, :, offsets] = k[rows]
    cache[1, pages, :, offsets] = v[rows]
    return {"q": turn(s["q"]), "cache": cache}


def _exact_attention(case, s):
    q_len, kv_len = _attention_lengths(case)
    hq, hkv, dh = case["hq"], case["hkv"], case["dh"]
    outs, lses, at = [], [], 0
    for i, (n, kv) in enumerate(zip(q_len, kv_len)):
        pages = s["block_tables"][i, :_pages(kv)].long()
        k, v = (s["kv_pool"][0, w][pages].double().permute(1, 0, 2, 3).reshape(hkv, -1, dh)[:, :kv] for w in (0, 1))
        pos = torch.arange(kv - n, kv, device="cuda")[:, None]
        key = torch.arange(kv, device="cuda")[None]
        seen = (key <= pos) & (pos - key < (case["window"] or kv + 1)) | (key < min(case["prefix"], kv))
        for h in range(hq):
            x = (s["q"][at:at + n, h].double() @ k[h * hkv // hq].T) / math.sqrt(dh)
            if case["cap"]:
                x = torch.tanh(x / case["cap"]) * case["cap"]
            if case["bias"]:
                x = x - 2.0 ** (-8.0 * (h + 1) / hq) * (pos - key).abs()
            x = torch.where(seen, x, torch.full_like(x, -math.inf))
            lses.append(torch.logsumexp(x, 1))
            outs.append(torch.softmax(x, 1) @ v[h * hkv // hq])
        at += n
    pick = lambda parts: torch.cat([torch.stack(parts[i * hq:(i + 1) * hq], 1) for i in range(len(q_len))])  # noqa: E731
    return {"o": pick(outs), "lse": pick(lses)}


def _exact_logprobs(case, s):
    got = []
    for i in range(0, case["rows"], 64):
        raw = s["logits"][i:i + 64].double()
        lp = torch.log_softmax(raw * s["scale"], 1)
        t = s["targets"][i:i + 64].long()
        some, row = t >= 0, torch.arange(raw.shape[0], device="cuda")
        part = {"logprob": torch.where(some, lp[row, t], torch.zeros_like(lp[:, 0])), "entropy": -(lp.exp() * lp).sum(1),
                "rank": torch.where(some, (raw > raw[row, t][:, None]).sum(1), -torch.ones_like(t)).int()}
        if case["top"]:
            order = torch.argsort(-raw, dim=1, stable=True)[:, :case["top"]]
            part["top_ids"], part["top_logprobs"] = order.int(), torch.gather(lp, 1, order)
        got.append(part)
    return {k: torch.cat([p[k] for p in got]) for k in got[0]}
