"""The operators of horizonserve_device.h on a B200 against their plain 64-bit definitions (device_ref.py), at the sizes and masks
where they can go wrong, at several SM budgets, and their refusals."""
import math

import numpy as np
import pytest
import torch

from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_ops as ops
from tests import device_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN = float("nan")
STATUS = {None: 0, "INVALID_ARG": B.HS_ERR_INVALID_ARG, "OUT_OF_PAGES": B.HS_ERR_OUT_OF_PAGES, "BAD_BLOCK_TABLE": B.HS_ERR_BAD_BLOCK_TABLE}


def i32(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device=DEV)


@pytest.fixture(scope="module")
def ws():
    return ops.workspace(DEV)


@pytest.fixture()
def status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def control_words_are_zero(ws):
    return int(ws[: 64 << 10].to(torch.int32).sum()) == 0


# ------------------------------------------------------------------------------------------------------------ page tables
def run_tables(ctx, q, free, free_count, tables, num_pages, cap, ws, status, budget=None, in_place=False):
    n = len(ctx)
    c, t = i32(ctx), i32(tables)
    fl, fc = i32(list(free) + [0] * (num_pages - len(free))), i32([free_count])
    kv = c if in_place else torch.full((n,), -7, dtype=torch.int32, device=DEV)
    fo = fc if in_place else torch.full((1,), -7, dtype=torch.int32, device=DEV)
    out = [torch.full((m,), -7, dtype=torch.int32, device=DEV) for m in (n + 1, cap, cap, cap)]
    ops.step_tables(c, i32(q), fl, fc, t, kv, *out, fo, ws, status, sm_budget=budget)
    torch.cuda.synchronize()
    assert control_words_are_zero(ws)
    return {"kv_len": kv.tolist(), "tok_begin": out[0].tolist(), "tok_seq": out[1].tolist(), "tok_pos": out[2].tolist(), "tok_slot": out[3].tolist(),
            "block_tables": t.cpu().numpy(), "free_count": int(fo)}


def same(got, want):
    for k in want:
        assert np.array_equal(np.asarray(got[k]), np.asarray(want[k])), k


@pytest.mark.parametrize("n,ctx_hi,q_hi,cap_extra", [(1, 1, 1, 0), (1, 0, 40, 3), (3, 33, 17, 5), (64, 200, 1, 0), (65, 40, 70, 1), (1025, 60, 3, 100), (4096, 20, 2, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_step_tables(n, ctx_hi, q_hi, cap_extra, in_place, ws, status):
    rng = np.random.default_rng(n + q_hi)
    ctx = rng.integers(0, ctx_hi + 1, n).tolist()
    q = rng.integers(0, q_hi + 1, n).tolist()
    if sum(q) == 0:
        q[0] = 1
    num_pages = sum(ref.pages(c + m) for c, m in zip(ctx, q)) + 2
    tables, free = ref.random_tables(rng, ctx, ref.pages(ctx_hi + q_hi) + 1, num_pages)
    cap = sum(q) + cap_extra
    why, want = ref.step_tables(ctx, q, free, len(free), tables, num_pages, cap)
    assert why is None
    for budget in (None, 1, 5):
        same(run_tables(ctx, q, free, len(free), tables, num_pages, cap, ws, status, budget, in_place), want)
    assert int(status) == 0


@pytest.mark.parametrize("what", ["negative ctx", "negative q", "row too short", "too many tokens", "free count", "out of pages", "bad popped page", "bad owned page"])
def test_step_tables_that_cannot_be_done(what, ws, status):
    rng = np.random.default_rng(5)
    ctx, q, width, num_pages, cap = [20, 0, 47, 5], [1, 33, 2, 0], 5, 20, 40
    tables, free = ref.random_tables(rng, ctx, width, num_pages)
    free, count = free.tolist(), len(free)
    if what == "negative ctx":
        ctx[1] = -1
    elif what == "negative q":
        q[3] = -2
    elif what == "row too short":
        q[2] = 34
    elif what == "too many tokens":
        cap = 35
    elif what == "free count":
        count = 21
    elif what == "out of pages":
        count = 3
    elif what == "bad popped page":
        free[count - 2] = num_pages
    elif what == "bad owned page":
        tables[2, 2] = -3
    why, want = ref.step_tables(ctx, q, free, count, tables, num_pages, cap)
    assert why is not None
    for in_place in (False, True):
        status.zero_()
        same(run_tables(ctx, q, free, count, tables, num_pages, cap, ws, status, None, in_place), want)
        assert int(status) == STATUS[why]


def test_tables_follow_the_host_allocator(ws, status):
    """A few steps and a release on the device give the block tables that hs_kv_alloc / hs_kv_free give on the host."""
    from paper_2608_01785_b200 import workloads as wl
    cfg = B.make_config(wl.DIMS["c1_tiny"], 64, 256, 16, 8, 128, device=-1)
    host = B.hs_stage_create(cfg, None, 0, 0)
    n, width, pool = 5, 8, 64
    ctx, tables = i32([0] * n), torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    free, count = i32(list(range(pool))[::-1]), i32([pool])
    outs = [torch.empty(m, dtype=torch.int32, device=DEV) for m in (n + 1, 200, 200, 200)]
    lens = np.zeros(n, dtype=int)
    rng = np.random.default_rng(0)
    for step in range(4):
        q = rng.integers(0, 25, n)
        ops.step_tables(ctx, i32(q), free, count, tables, ctx, *outs, count, ws, status)
        lens += q
        rows = [B.hs_kv_alloc(host, s, int(lens[s]), 8) if lens[s] else [] for s in range(n)]
        got = tables.cpu().numpy()
        for s in range(n):
            assert got[s, :len(rows[s])].tolist() == rows[s] and (got[s, len(rows[s]):] == -1).all()
        assert ctx.tolist() == lens.tolist() and int(count) == B.hs_kv_free_pages(host)
        if step == 1:
            ops.release_pages(i32([0, 1, 0, 3, 0]), ctx, tables, free, count, ws, status)
            for s in (1, 3):
                B.hs_kv_free(host, s)
                lens[s] = 0
            assert ctx.tolist() == lens.tolist() and int(count) == B.hs_kv_free_pages(host)
    assert int(status) == 0 and control_words_are_zero(ws)
    B.hs_stage_destroy(host)


@pytest.mark.parametrize("n", [1, 7, 2000])
def test_release_pages(n, ws, status):
    rng = np.random.default_rng(n)
    ctx = rng.integers(0, 100, n)
    num_pages = sum(ref.pages(c) for c in ctx) + 3
    tables, free = ref.random_tables(rng, ctx, 7, num_pages)
    done = rng.integers(0, 2, n)
    pad = free.tolist() + [-5] * (num_pages - len(free))
    want = ref.release_pages(done, ctx, tables, pad, len(free))
    for budget in (None, 1, 3):
        t = [i32(done), i32(ctx), i32(tables), i32(pad), i32([len(free)])]
        ops.release_pages(*t, ws, status, sm_budget=budget)
        assert t[1].tolist() == [int(x) for x in want[0]] and np.array_equal(t[2].cpu().numpy(), want[1])
        assert t[3].tolist() == [int(x) for x in want[2]] and int(t[4]) == want[3]
    assert int(status) == 0
    # more pages than the stack has room for: nothing changes
    if done.any() and ctx[done != 0].sum() > 0:
        t = [i32(done), i32(ctx), i32(tables), i32(pad), i32([num_pages])]
        ops.release_pages(*t, ws, status)
        assert t[1].tolist() == ctx.tolist() and np.array_equal(t[2].cpu().numpy(), tables) and t[3].tolist() == pad and int(t[4]) == num_pages
        assert int(status) == B.HS_ERR_INVALID_ARG
    assert control_words_are_zero(ws)


# ------------------------------------------------------------------------------------------------------------------- rope
@pytest.mark.parametrize("scaling,kw", [("plain", {}), ("linear", {"factor": 4.0}), ("base", {"factor": 8.0}),
                                        ("by_parts", {"factor": 16.0, "trained": 4096, "slow": 1.0, "fast": 32.0})])
@pytest.mark.parametrize("rot,positions,magnitude", [(16, 1, 1.0), (64, 1000, 1.0), (128, 70001, 1.2773)])
def test_rope_table(scaling, kw, rot, positions, magnitude):
    code = {"plain": ops.ROPE_PLAIN, "linear": ops.ROPE_LINEAR, "base": ops.ROPE_BASE, "by_parts": ops.ROPE_BY_PARTS}[scaling]
    table = torch.full((positions, rot // 2, 2), NAN, device=DEV)
    ops.rope_table(table, 1e6, code, kw.get("factor", 1.0), kw.get("trained", 0), kw.get("slow", 1.0), kw.get("fast", 32.0), magnitude)
    w = ref.frequencies(rot, 1e6, scaling, **kw)
    angle = np.arange(positions, dtype=np.float64)[:, None] * w[None]
    want = np.stack([np.cos(angle), np.sin(angle)], -1) * magnitude
    # one rounding to fp32 (2^-24 of at most the magnitude) and 64-bit angles of up to 7e4, formed twice
    assert np.abs(table.cpu().numpy().astype(np.float64) - want).max() <= magnitude * (2.0 ** -24 + 1e-10)
    other = torch.empty_like(table)
    ops.rope_table(other, 1e6, code, kw.get("factor", 1.0), kw.get("trained", 0), kw.get("slow", 1.0), kw.get("fast", 32.0), magnitude, sm_budget=3)
    assert torch.equal(table, other)


@pytest.mark.parametrize("tokens,hq,hkv,dim,rot", [(1, 1, 1, 64, 64), (3, 28, 4, 128, 128), (37, 16, 4, 64, 32), (300, 5, 5, 96, 48), (19, 12, 1, 128, 64),
                                                    (9, 3, 2, 16, 16), (40, 4, 2, 256, 240)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("src,dst", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float16)])
def test_rope_cache(tokens, hq, hkv, dim, rot, interleaved, src, dst, status):
    g = torch.Generator().manual_seed(tokens + dim)
    layers, pages, positions, layer = 2, tokens // 16 + 3, 500, 1
    extra = 16                                         # rows are slices of a wider matrix
    qkv = torch.randn(tokens, (hq + 2 * hkv) * dim + extra, generator=g).to(src)
    q, k, v = (qkv[:, a * dim:b * dim].unflatten(1, (b - a, dim)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    pos = torch.randint(0, positions, (tokens,), generator=g, dtype=torch.int32)
    slot = torch.randperm(pages * 16, generator=g)[:tokens].to(torch.int32)
    padding = []
    if tokens > 5:
        padding = [2, tokens - 1]
        slot[padding] = -1
        pos[tokens - 1] = -1                           # a padding row without a position: zeros, and no complaint
    table = torch.empty(positions, rot // 2, 2, device=DEV)
    ops.rope_table(table)
    pool = torch.randn(layers, 2, pages, hkv, 16, dim, generator=g).to(dst)
    want_pool = pool[layer].double()
    p = pos.clamp(min=0).tolist()
    want_q, want_k = ref.rotate(q.double(), table.cpu(), p, interleaved), ref.rotate(k.double(), table.cpu(), p, interleaved)
    for t in range(tokens):
        if int(pos[t]) < 0:
            want_q[t] = 0
        if int(slot[t]) >= 0:
            want_pool[0, int(slot[t]) // 16, :, int(slot[t]) % 16] = want_k[t]
            want_pool[1, int(slot[t]) // 16, :, int(slot[t]) % 16] = v[t].double()
    got = []
    for budget in (None, 1, 7):
        d_qkv, d_pool = qkv.to(DEV), pool.to(DEV)
        dq, dk, dv = (d_qkv[:, a * dim:b * dim].unflatten(1, (b - a, dim)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
        out = torch.full((tokens, hq, dim), NAN, dtype=dst, device=DEV)
        ops.rope_cache(dq, dk, dv, pos.to(DEV), slot.to(DEV), table, out, d_pool, layer, status, interleaved=interleaved, sm_budget=budget)
        got.append((out, d_pool))
    assert int(status) == 0
    for out, d_pool in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(d_pool, got[0][1])
    out, d_pool = got[0]
    # one rounding of the result to the cache's type, and two products and a sum in fp32 of values up to sqrt(x^2 + y^2)
    u = 2.0 ** -8 if dst == torch.bfloat16 else 2.0 ** -11
    for a, b in ((out.cpu().double(), want_q), (d_pool[layer].cpu().double(), want_pool)):
        assert bool(((a - b).abs() <= u * b.abs() * 1.01 + 3 * 2.0 ** -24 * 6 + 2.0 ** -25).all())
    assert torch.equal(d_pool[0].cpu(), pool[0])       # the other layer is as it was


def test_rope_cache_reports_rows_it_cannot_place(status):
    table = torch.empty(10, 32, 2, device=DEV)
    ops.rope_table(table)
    pool = torch.zeros(1, 2, 2, 1, 16, 64, dtype=torch.bfloat16, device=DEV)
    x = torch.ones(4, 1, 64, device=DEV)
    out = torch.full((4, 1, 64), NAN, dtype=torch.bfloat16, device=DEV)
    for pos, slot in (([0, 10, 1, 2], [0, 1, 2, 3]), ([0, -1, 1, 2], [0, 1, 2, 3]), ([0, 3, 1, 2], [0, 32, 2, 3])):
        status.zero_()
        pool.zero_()
        ops.rope_cache(x, x, x, i32(pos), i32(slot), table, out, pool, 0, status)
        assert int(status) == B.HS_ERR_INVALID_ARG
        assert pool[0, 1, 0, 0, :, 0].tolist() == [1, 0, 1, 1] + [0] * 12 and bool((pool[0, :, 1] == 0).all())
        assert bool((out[1] == 0).all()) == (pos[1] in (10, -1))


def test_rope_cache_in_place(status):
    table = torch.empty(64, 64, 2, device=DEV)
    ops.rope_table(table)
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.randn(50, 6, 128, generator=g, device=DEV).bfloat16()
    k = torch.randn(50, 2, 128, generator=g, device=DEV).bfloat16()
    pool = torch.zeros(1, 2, 4, 2, 16, 128, dtype=torch.bfloat16, device=DEV)
    pos, slot, out = i32(list(range(50))), i32(list(range(50))), torch.empty_like(q)
    ops.rope_cache(q, k, k, pos, slot, table, out, pool, 0, status)
    ops.rope_cache(q, k, k, pos, slot, table, q, pool, 0, status)
    assert torch.equal(q, out) and int(status) == 0


# -------------------------------------------------------------------------------------------------------------- attention
def attention_case(seed, kv_len, q_len, hq, hkv, dim, dtype, cap, window, prefix, bias, poison=True):
    """Random inputs; cache rows that no row of the call sees hold NaN, tables of pages that nobody sees hold rubbish."""
    rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    n, t = len(kv_len), sum(q_len)
    num_pages, width = sum(ref.pages(x) for x in kv_len) + 2, max(max(ref.pages(x) for x in kv_len), 1) + 1
    tables, _ = ref.random_tables(rng, kv_len, width, num_pages)
    q = torch.randn(t, hq, dim, generator=g).mul(3).to(dtype)
    pool = torch.randn(2, 2, num_pages, hkv, 16, dim, generator=g).to(dtype)
    pre = [int(rng.integers(0, max(1, min(x, prefix)) + 1)) for x in kv_len] if prefix else None
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]) if bias else None
    if poison:
        seen = torch.zeros(num_pages, 16, dtype=torch.bool)
        for s in range(n):
            first = kv_len[s] - q_len[s]
            lo = max(first - window + 1, 0) if window else 0
            used = set()
            for j in range(kv_len[s]):
                if q_len[s] and (j >= lo or (pre and j < pre[s])):
                    seen[tables[s, j // 16], j % 16] = True
                    used.add(j // 16)
            for i in range(width):
                if i not in used:
                    tables[s, i] = (-1, num_pages + 5)[i % 2]
        pool[1, :, ~seen.unsqueeze(1).expand(-1, hkv, -1)] = NAN
        pool[0] = NAN
    return {"q": q, "pool": pool, "tables": tables, "kv_len": kv_len, "q_len": q_len, "prefix": pre, "slopes": slopes, "scale": dim ** -0.5, "cap": cap, "window": window}


def run_attention(c, ws, status, budget=None, strided=True, stream=None):
    t, hq, dim = c["q"].shape
    wide = torch.zeros(t, hq * dim + 24, dtype=c["q"].dtype, device=DEV)
    q = wide[:, :hq * dim].unflatten(1, (hq, dim)) if strided else torch.empty(t, hq, dim, dtype=c["q"].dtype, device=DEV)
    q.copy_(c["q"])
    o_wide = torch.full((t, hq * dim + 8), 77.0, dtype=c["q"].dtype, device=DEV)
    o = o_wide[:, :hq * dim].unflatten(1, (hq, dim))
    lse = torch.full((t, hq), NAN, device=DEV)
    begin = i32([0] + list(np.cumsum(c["q_len"])))
    ops.paged_attention(q, c["pool"].to(DEV), 1, i32(c["tables"]), i32(c["kv_len"]), o, ws, status, lse=lse, tok_begin=begin,
                        max_q_len=max(c["q_len"]), prefix_len=None if c["prefix"] is None else i32(c["prefix"]),
                        slopes=None if c["slopes"] is None else c["slopes"].to(DEV), scale=c["scale"], cap=c["cap"], window=c["window"], sm_budget=budget)
    torch.cuda.synchronize()
    assert bool((o_wide[:, hq * dim:] == 77.0).all())
    return o.contiguous(), lse


def check_attention(c, ws, status):
    o, lse = run_attention(c, ws, status)
    assert int(status) == 0 and control_words_are_zero(ws)
    want_o, want_lse = ref.attention(c["q"].double(), c["pool"][1].double(), c["tables"], c["kv_len"], c["q_len"], c["prefix"],
                                     None if c["slopes"] is None else c["slopes"].double(), c["scale"], c["cap"], c["window"])
    # Weights and outputs are rounded to the cache's type once each (u of at most max |v|); a score is off by the fp32 sum of dim products
    # (dim 2^-24 sum |q k| scale, below 2e-4 at these inputs) and by 2e-7 cap, which moves o by twice that of max |v| and lse by that.
    u = 2.0 ** -8 if c["q"].dtype == torch.bfloat16 else 2.0 ** -11
    v = c["pool"][1, 1].double()
    vmax = float(v[~v.isnan()].abs().max()) if bool((~v.isnan()).any()) else 0.0
    o, lse = o.cpu().double(), lse.cpu().double()
    assert not bool(o.isnan().any()) and float((o - want_o).abs().max()) <= (2 * u + 5e-4) * vmax
    empty = want_lse == -math.inf
    assert bool((lse[empty] == -math.inf).all()) and bool((o[empty] == 0).all())
    assert bool(((lse - want_lse)[~empty].abs() <= 3e-4).all())
    for budget in (1, 9, 37):
        o2, lse2 = run_attention(c, ws, status, budget)
        assert torch.equal(o2.cpu().double(), o) and torch.equal(lse2.cpu().double(), lse), f"budget {budget}"


MASKS = [(0.0, 0, 0, False), (30.0, 0, 0, False), (0.0, 0, 0, True), (50.0, 40, 0, True), (0.0, 17, 21, False), (20.0, 1, 0, False), (0.0, 0, 90, False)]
HEADS = [(28, 4, 128), (16, 4, 64), (5, 5, 64), (12, 1, 128), (34, 2, 64), (20, 1, 64)]


@pytest.mark.parametrize("cap,window,prefix,bias", MASKS)
@pytest.mark.parametrize("hq,hkv,dim", HEADS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_decode_attention(cap, window, prefix, bias, hq, hkv, dim, dtype, ws, status):
    kv = [1, 15, 16, 17, 0, 33, 100, 250]
    check_attention(attention_case(3, kv, [1, 1, 1, 1, 1, 1, 0, 1], hq, hkv, dim, dtype, cap, window, prefix, bias), ws, status)


@pytest.mark.parametrize("kv", [[1], [16], [3001], [0], [0, 0, 0], [2000, 1], [1, 2500], [700] * 3, list(range(1, 120))])
@pytest.mark.parametrize("hq,hkv", [(7, 1), (16, 1), (4, 2)])
def test_decode_lengths(kv, hq, hkv, ws, status):
    check_attention(attention_case(len(kv), kv, [1] * len(kv), hq, hkv, 128, torch.bfloat16, 0.0, 0, 0, False), ws, status)


def test_decode_of_many_sequences(ws, status):
    rng = np.random.default_rng(1)
    kv = rng.integers(0, 30, 1500).tolist()
    check_attention(attention_case(2, kv, [int(x) for x in rng.integers(0, 2, 1500)], 2, 1, 64, torch.bfloat16, 30.0, 0, 0, False), ws, status)


@pytest.mark.parametrize("cap,window,prefix,bias", MASKS)
@pytest.mark.parametrize("hq,hkv,dim", HEADS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_chunk_attention(cap, window, prefix, bias, hq, hkv, dim, dtype, ws, status):
    q = [1, 2, 0, 7, 33, 16, 70]
    kv = [1, 40, 12, 7, 130, 16, 75]
    check_attention(attention_case(4, kv, q, hq, hkv, dim, dtype, cap, window, prefix, bias), ws, status)


@pytest.mark.parametrize("q,kv", [([2], [2]), ([64], [64]), ([65], [1000]), ([300], [300]), ([129, 3], [129, 700]), ([5, 3], [3, 0]), ([2, 0], [9, 9])])
@pytest.mark.parametrize("hq,hkv,window", [(7, 1, 0), (16, 1, 100), (4, 2, 0), (3, 3, 64)])
def test_chunk_lengths(q, kv, hq, hkv, window, ws, status):
    """Among them a sequence with more rows than keys, whose first rows see nothing."""
    check_attention(attention_case(5, kv, q, hq, hkv, 128, torch.bfloat16, 0.0, window, 0, False), ws, status)


def test_chunk_of_single_tokens_agrees_with_decode(ws, status):
    """The chunk form on a batch of single tokens, a row's worth of rounding apart from the decode form."""
    c = attention_case(6, [40, 300, 17], [1, 1, 1], 16, 2, 128, torch.bfloat16, 30.0, 0, 0, True)
    o, lse = run_attention(c, ws, status)
    c["q_len"] = [1, 1, 1]
    begin = i32([0, 1, 2, 3])
    o2 = torch.empty(3, 16, 128, dtype=torch.bfloat16, device=DEV)
    ops.paged_attention(c["q"].to(DEV), c["pool"].to(DEV), 1, i32(c["tables"]), i32(c["kv_len"]), o2, ws, status, tok_begin=begin, max_q_len=2,
                        slopes=c["slopes"].to(DEV), scale=c["scale"], cap=c["cap"])
    v = c["pool"][1, 1].double()
    assert float((o.double() - o2.double()).abs().max()) <= 4 * 2.0 ** -8 * float(v[~v.isnan()].abs().max())
    ops.paged_attention(c["q"].to(DEV), c["pool"].to(DEV), 1, i32(c["tables"]), i32(c["kv_len"]), o2, ws, status, slopes=c["slopes"].to(DEV), scale=c["scale"],
                        cap=c["cap"])                  # and without tok_begin: row s is sequence s's
    assert torch.equal(o, o2) and int(status) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_of_large_scores(dtype, ws, status):
    """Scores far beyond the cap and far apart: tanh saturates, weights underflow."""
    for q in ([1, 1, 1], [3, 20, 1]):
        c = attention_case(7, [30, 64, 200], q, 4, 2, 64, dtype, 5.0, 0, 0, False)
        c["q"] *= 60
        check_attention(c, ws, status)


def test_attention_reports_bad_tables(ws, status):
    for q, what in (([1, 1], "page"), ([4, 3], "page"), ([1, 1], "length"), ([4, 3], "length"), ([4, 3], "rows"), ([1, 1], "rows")):
        c = attention_case(8, [40, 50], q, 2, 1, 64, torch.bfloat16, 0.0, 0, 0, False)
        args = [c["q"].to(DEV), c["pool"].to(DEV), 1]
        tables, kv, begin = c["tables"].copy(), list(c["kv_len"]), [0, q[0], q[0] + q[1]]
        if what == "page":
            tables[1, 1] = 1000
        elif what == "length":
            kv[1] = 10000
        else:
            begin[2] = q[0] + q[1] + 5
        status.zero_()
        want = torch.full((sum(q), 2, 64), 5.0, dtype=torch.bfloat16, device=DEV)
        got = want.clone()
        ops.paged_attention(*args, i32(c["tables"]), i32(c["kv_len"]), want, ws, status, tok_begin=i32([0, q[0], q[0] + q[1]]), max_q_len=max(q))
        assert int(status) == 0
        ops.paged_attention(*args, i32(tables), i32(kv), got, ws, status, tok_begin=i32(begin), max_q_len=max(q))
        torch.cuda.synchronize()
        assert int(status) == (B.HS_ERR_INVALID_ARG if what == "rows" else B.HS_ERR_BAD_BLOCK_TABLE)
        # the other sequence's rows are right (in a decode batch its share of the device may differ, and so the order of its sums)
        assert float((got[:q[0]].double() - want[:q[0]].double()).abs().max()) <= 4 * 2.0 ** -8 * 6
        if what == "rows":
            assert bool((got[q[0]:] == 5.0).all())
        assert control_words_are_zero(ws)


# ---------------------------------------------------------------------------------------------------------- log probabilities
def run_logprobs(x, targets, n_top, scale, ws, status, budget=None):
    n = x.shape[0]
    out = {"logprob": torch.full((n,), NAN, device=DEV), "entropy": torch.full((n,), NAN, device=DEV), "rank": torch.full((n,), -9, dtype=torch.int32, device=DEV)}
    if n_top:
        out["top_ids"] = torch.full((n, n_top), -9, dtype=torch.int32, device=DEV)
        out["top_logprobs"] = torch.full((n, n_top), NAN, device=DEV)
    ops.token_logprobs(x, i32(targets), out["logprob"], ws, status, entropy=out["entropy"], rank=out["rank"], top_ids=out.get("top_ids"),
                       top_logprobs=out.get("top_logprobs"), scale=scale, sm_budget=budget)
    torch.cuda.synchronize()
    assert control_words_are_zero(ws)
    return out


def check_logprobs(x, targets, n_top, scale, ws, status, budgets=(1, 6)):
    got = run_logprobs(x, targets, n_top, scale, ws, status)
    want = ref.logprobs(x.cpu().double(), targets, n_top, scale)
    # d = k x - k max in fp32 is off by 2^-23 of |k x|, |k max| and itself, exp2 by 2^-22, and sums of V terms by far less than V 2^-24 of
    # themselves (they are added by 512 threads and more): in all below 1e-5 + 4e-7 of the largest |scale x| that counts
    big = float(x[x > -math.inf].abs().max()) * scale if bool((x > -math.inf).any()) else 0.0
    tol = 1e-5 + 4e-7 * big
    for k in ("logprob", "entropy") + (("top_logprobs",) if n_top else ()):
        a, b = got[k].cpu().double(), torch.tensor(want[k], dtype=torch.float64).float().double()      # (beyond fp32: infinity)
        dead = b == -math.inf
        assert bool((a[dead] == -math.inf).all()) and bool(((a - b)[~dead].abs() <= tol).all()), k
    assert got["rank"].tolist() == want["rank"]
    if n_top:
        assert got["top_ids"].tolist() == want["top_ids"]
    for budget in budgets:
        again = run_logprobs(x, targets, n_top, scale, ws, status, budget)
        for k in got:
            assert torch.equal(got[k], again[k]), (k, budget)
    return got


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 5), (3, 33), (2, 1023), (1, 1024), (5, 1025), (70, 3001), (1, 20000), (3, 50003), (200, 2049), (1, 152064)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n_top", [0, 1, 20, 32])
def test_token_logprobs(rows, vocab, dtype, n_top, ws, status):
    g = torch.Generator().manual_seed(rows * 7 + vocab)
    wide = (3 * torch.randn(rows, vocab + 5, generator=g)).to(dtype).to(DEV)      # odd strides and beginnings
    x = wide[:, 3:3 + vocab]
    targets = torch.randint(0, vocab, (rows,), generator=g).tolist()
    if rows > 1:
        targets[1] = -1
    check_logprobs(x, targets, min(n_top, vocab), 0.7, ws, status, budgets=(1, 6) if vocab < 10000 else (50,))
    assert int(status) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("what", ["constant", "two values", "ascending", "descending", "one lane", "masked", "all masked", "few left", "lowest", "zeros", "spike"])
def test_token_logprobs_of_unusual_rows(what, dtype, ws, status):
    vocab = 30011
    x = torch.randn(4, vocab, generator=torch.Generator().manual_seed(3))
    i = torch.arange(vocab)
    if what == "constant":
        x[:] = -2.5
    elif what == "two values":
        x[:] = (i % 2).float()
    elif what == "ascending":
        x[:] = i / vocab * 8
    elif what == "descending":
        x[:] = -i / vocab * 8
    elif what == "one lane":
        x[:, i % 128 < 4] += 20                       # all large values where one lane of every warp reads
    elif what == "masked":
        x[:, 100:30000] = -math.inf
    elif what == "all masked":
        x[1] = -math.inf
        x[3] = -math.inf
    elif what == "few left":
        x[:] = -math.inf
        x[:, [5, 17000, 30010]] = torch.tensor([1.0, 3.0, 2.0])
        x[2, 5] = -math.inf
    elif what == "lowest":
        x[:, ::3] = torch.finfo(dtype).min
    elif what == "zeros":
        x[:] = 0
        x[:, ::2] = -0.0
    elif what == "spike":
        x[:, 29000] = 3000.0 if dtype != torch.float16 else 900.0
    check_logprobs(x.to(dtype).to(DEV), [0, vocab - 1, 17000, 29000], 20, 1.3, ws, status)
    assert int(status) == 0


def test_token_logprobs_of_rows_that_are_not_numbers(ws, status):
    x = torch.randn(3, 5000, generator=torch.Generator().manual_seed(3))
    want = run_logprobs(x.to(DEV), [1, 2, 3], 5, 1.0, ws, status)
    x[0, 4321] = NAN
    x[2, 77] = math.inf
    got = run_logprobs(x.to(DEV), [1, 2, 3], 5, 1.0, ws, status)
    for r in (0, 2):
        assert math.isnan(float(got["logprob"][r])) and math.isnan(float(got["entropy"][r]))
        assert all(-1 <= t < 5000 for t in got["top_ids"][r].tolist())
    for k in got:
        assert torch.equal(got[k][1], want[k][1])


def test_token_logprobs_of_a_target_that_is_none(ws, status):
    x = torch.randn(2, 100, generator=torch.Generator().manual_seed(3)).to(DEV)
    got = run_logprobs(x, [100, -5], 0, 1.0, ws, status)
    assert got["logprob"].tolist() == [0, 0] and got["rank"].tolist() == [-1, -1] and int(status) == B.HS_ERR_INVALID_ARG


# ------------------------------------------------------------------------------------------------------ streams and refusals
def test_operators_on_another_stream(ws, status):
    c = attention_case(9, [300, 40], [1, 1], 8, 2, 64, torch.bfloat16, 0.0, 0, 0, False)
    o, lse = run_attention(c, ws, status)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, lse2 = run_attention(c, ops.workspace(DEV), status)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_refusals(ws, status):
    def refused(code, fn):
        with pytest.raises(B.HsError) as e:
            fn()
        assert e.value.status == code

    x = torch.zeros(2, 50, device=DEV)
    lp, t = torch.zeros(2, device=DEV), i32([0, 1])
    refused(B.HS_ERR_INVALID_BUDGET, lambda: ops.token_logprobs(x, t, lp, ws, status, sm_budget=0))
    refused(B.HS_ERR_INVALID_BUDGET, lambda: ops.token_logprobs(x, t, lp, ws, status, sm_budget=1000))
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.token_logprobs(x, t, lp, ws, status, scale=0.0))
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.token_logprobs(x, t, None, ws, status))
    many = torch.zeros(2, 33, dtype=torch.int32, device=DEV)
    refused(B.HS_ERR_UNSUPPORTED_SHAPE, lambda: ops.token_logprobs(x, t, lp, ws, status, top_ids=many, top_logprobs=many.float()))
    with pytest.raises(ValueError):
        ops.token_logprobs(x, t.long(), lp, ws, status)
    with pytest.raises(ValueError):
        ops.token_logprobs(x.t(), t, lp, ws, status)
    with pytest.raises(ValueError):
        ops.token_logprobs(x, t, lp, ws[1000:], status)

    c = attention_case(1, [20, 30], [1, 1], 4, 2, 64, torch.bfloat16, 0.0, 0, 0, False)
    q, pool, bt, kv = c["q"].to(DEV), c["pool"].to(DEV), i32(c["tables"]), i32(c["kv_len"])
    o = torch.empty_like(q)
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.paged_attention(q, pool, 1, bt, kv, o, ws, status, max_q_len=2))
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.paged_attention(q, pool, 1, bt, kv, o, ws, status, cap=-1.0))
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.paged_attention(q, pool, 1, bt, kv, o, ws, status, window=-1))
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.paged_attention(q, pool, 1, bt, kv, o, ws, status, scale=NAN))
    refused(B.HS_ERR_INVALID_BUDGET, lambda: ops.paged_attention(q, pool, 1, bt, kv, o, ws, status, sm_budget=149))
    with pytest.raises(ValueError):
        ops.paged_attention(q.float(), pool, 1, bt, kv, o, ws, status)
    with pytest.raises(ValueError):
        ops.paged_attention(q, pool, 2, bt, kv, o, ws, status)
    odd = torch.zeros(1, 2, 4, 1, 16, 96, dtype=torch.bfloat16, device=DEV)
    z = torch.zeros(2, 1, 96, dtype=torch.bfloat16, device=DEV)
    refused(B.HS_ERR_UNSUPPORTED_SHAPE, lambda: ops.paged_attention(z, odd, 0, bt, kv, z, ws, status))
    three = torch.zeros(2, 3, 64, dtype=torch.bfloat16, device=DEV)
    refused(B.HS_ERR_UNSUPPORTED_SHAPE, lambda: ops.paged_attention(three, pool, 1, bt, kv, three, ws, status))

    table = torch.empty(10, 32, 2, device=DEV)
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.rope_table(table, base=-1.0))
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.rope_table(table, scaling=7))
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.rope_table(table, scaling=ops.ROPE_BY_PARTS, factor=2.0))
    refused(B.HS_ERR_UNSUPPORTED_SHAPE, lambda: ops.rope_table(torch.empty(10, 12, 2, device=DEV)))
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=DEV)
    wide = torch.empty(10, 40, 2, device=DEV)
    refused(B.HS_ERR_UNSUPPORTED_SHAPE, lambda: ops.rope_cache(q, k, k, t, t, wide, o, pool, 1, status))
    shifted = torch.zeros(2 * 4 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(2, 4, 64)
    refused(B.HS_ERR_INVALID_ARG, lambda: ops.rope_cache(shifted, k, k, t, t, table, o, pool, 1, status))
    with pytest.raises(ValueError):
        ops.rope_cache(q, k.float(), k, t, t, table, o, pool, 1, status)

    ctx, free, count = i32([0] * 3), i32([0, 1]), i32([2])
    out = [torch.empty(m, dtype=torch.int32, device=DEV) for m in (4, 8, 8, 8)]
    bt3 = torch.full((3, 2), -1, dtype=torch.int32, device=DEV)
    refused(B.HS_ERR_INVALID_BUDGET, lambda: ops.step_tables(ctx, ctx, free, count, bt3, ctx, *out, count, ws, status, sm_budget=-1))
    big = i32([0] * 4097)
    refused(B.HS_ERR_UNSUPPORTED_SHAPE, lambda: ops.release_pages(big, big, torch.zeros(4097, 1, dtype=torch.int32, device=DEV), free, count, ws, status))
    with pytest.raises(ValueError):
        ops.step_tables(ctx, ctx[:2], free, count, bt3, ctx, *out, count, ws, status)
    torch.cuda.synchronize()
    assert int(status) == 0


# ------------------------------------------------------------------------------------------------- how work is divided over the device
@pytest.mark.parametrize("cap,window,prefix,bias", [(0.0, 0, 0, False), (30.0, 900, 0, True), (0.0, 1000, 1200, False)])
@pytest.mark.parametrize("hq,hkv,dim", [(7, 1, 128), (16, 2, 64), (12, 1, 128), (34, 2, 64)])
@pytest.mark.parametrize("q,kv", [([4], [2000]), ([1, 30], [3000, 50]), ([20, 0], [5003, 800]), ([3, 70, 40], [1500, 70, 900]), ([2, 2], [0, 1400])])
def test_chunks_of_few_rows_divide_long_sequences(cap, window, prefix, bias, hq, hkv, dim, q, kv, ws, status):
    check_attention(attention_case(sum(kv), kv, q, hq, hkv, dim, torch.bfloat16, cap, window, prefix, bias), ws, status)


@pytest.mark.parametrize("cap,window,prefix,bias", [(0.0, 0, 0, False), (30.0, 700, 0, True), (0.0, 500, 650, False)])
@pytest.mark.parametrize("hq,hkv,dim,kv", [
    (16, 16, 64, [40, 7, 0, 33, 64, 1, 90, 16, 17, 31]),     # whole groups, several a share
    (8, 1, 64, [9000, 100, 0, 700]),                          # parts of groups, most groups with fewer than the longest
    (12, 2, 128, [2000, 1999, 3]),                            # and with two tiles of heads
    (2, 2, 64, [2400] * 79 + [5]),                            # more groups than shares, too long to stay whole: cut anywhere
])
def test_decode_by_groups_parts_and_pieces(cap, window, prefix, bias, hq, hkv, dim, kv, ws, status):
    check_attention(attention_case(len(kv), kv, [1] * len(kv), hq, hkv, dim, torch.bfloat16, cap, window, prefix, bias), ws, status)


@pytest.mark.parametrize("rows,vocab,dtype,n_top", [(149, 152064, torch.bfloat16, 20), (3, 152064, torch.float32, 32), (20, 60001, torch.float16, 1), (300, 20000, torch.float32, 5),
                                                    (64, 152064, torch.float32, 20), (1, 300001, torch.bfloat16, 32)])
def test_token_logprobs_of_whole_and_divided_rows(rows, vocab, dtype, n_top, ws, status):
    g = torch.Generator().manual_seed(rows + vocab)
    x = (3 * torch.randn(rows, vocab, generator=g)).to(dtype).to(DEV)
    check_logprobs(x, torch.randint(0, vocab, (rows,), generator=g).tolist(), n_top, 0.9, ws, status, budgets=(11,))


@pytest.mark.parametrize("dtype,large", [(torch.float32, 3e38), (torch.bfloat16, 3e38), (torch.float16, 65504.0)])
@pytest.mark.parametrize("vocab", [100, 3000, 70000])
def test_token_logprobs_of_logits_near_the_types_limits(dtype, large, vocab, ws, status):
    """Rows with a few logits at the largest values of the type, of either sign: only those at the top have a probability."""
    x = torch.randn(3, vocab, generator=torch.Generator().manual_seed(5))
    x[0, 17] = x[0, vocab - 3] = large
    x[1] = -large
    x[1, 40] = x[1, 41] = x[1, vocab // 2] = x[1, vocab - 1] = -large / 2
    x[2, ::2] = -large
    x[2, 50] = large
    x = x.to(dtype).to(DEV)
    got = run_logprobs(x, [17, 41, 50], 4, 1.0, ws, status)
    want = torch.tensor([-math.log(2), -math.log(4), 0.0])
    # the values at the top are equal, and the others' weights are 0: sums of 2, 4 and 1
    assert float((got["logprob"].cpu() - want).abs().max()) <= 1e-6 and float((got["entropy"].cpu() + want).abs().max()) <= 1e-6
    assert got["rank"].tolist() == [0, 0, 0]
    assert got["top_ids"][0, :2].tolist() == [17, vocab - 3] and got["top_ids"][1].tolist() == [40, 41, vocab // 2, vocab - 1] and int(got["top_ids"][2, 0]) == 50
    assert int(status) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [1e-4, 0.05, 60.0, 1e4])
def test_token_logprobs_of_unusual_scales(dtype, scale, ws, status):
    g = torch.Generator().manual_seed(8)
    x = 3 * torch.randn(4, 40000, generator=g)
    x[:, ::3] = -math.inf
    x = x.to(dtype).to(DEV)
    check_logprobs(x, [1, 3, 20000, 39998], 7, scale, ws, status)
