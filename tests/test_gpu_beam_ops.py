"""The operators of horizonserve_beams.h on a B200 against their plain definitions (beam_ref.py, device_ref.py), at the sizes, masks and orders where
they can go wrong, at several SM budgets, on other streams and in graphs, and what they refuse on the device."""
import math

import numpy as np
import pytest
import torch

from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_ops as ops
from tests import beam_ref as ref
from tests import device_ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN, INF = float("nan"), float("inf")
STATUS = {None: 0, "INVALID_ARG": B.HS_ERR_INVALID_ARG, "OUT_OF_PAGES": B.HS_ERR_OUT_OF_PAGES, "BAD_BLOCK_TABLE": B.HS_ERR_BAD_BLOCK_TABLE}
PAGE_BITS = (1 << 24) // 8


def i32(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device=DEV)


@pytest.fixture(scope="module")
def ws():
    return ops.workspace(DEV)


@pytest.fixture()
def status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def control_words_are_zero(ws):
    return not bool(ws[: 64 << 10].any()) and not bool(ws[-PAGE_BITS:].any())


# ------------------------------------------------------------------------------------------------------------ page tables
def run_fork(parent, ctx, tables, shares, free, count, num_pages, ws, status, budget=None):
    n = len(parent)
    t = [i32(x) for x in (parent, ctx, tables, shares, list(free) + [-5] * (num_pages - len(free)), [count])]
    copies = [torch.full((n,), -7, dtype=torch.int32, device=DEV) for _ in range(3)]
    ops.fork_pages(*t, *copies, ws, status, sm_budget=budget)
    torch.cuda.synchronize()
    assert control_words_are_zero(ws)
    return {"ctx_len": t[1].tolist(), "block_tables": t[2].cpu().numpy(), "shares": t[3].tolist(), "free_list": t[4].tolist(), "free_count": int(t[5]),
            "copy_src": copies[0].tolist(), "copy_dst": copies[1].tolist(), "copy_len": copies[2].tolist()}


def same(got, want):
    for k in want:
        assert np.array_equal(np.asarray(got[k]), np.asarray(want[k])), k


def pad(free, num_pages):
    return list(free) + [-5] * (num_pages - len(free))


@pytest.mark.parametrize("n,beams,most", [(1, 1, 0), (1, 1, 40), (1, 5, 100), (3, 2, 17), (7, 8, 300), (40, 32, 60), (1, 32, 16 * 70), (2048, 2, 20), (4096, 1, 5)])
def test_fork_pages(n, beams, most, ws, status):
    rng = np.random.default_rng(n * beams + most)
    ctx, tables, shares, free, num_pages = ref.shared_rows(rng, n, beams, [int(x) for x in rng.integers(0, most + 1, n)], n * beams + 40)
    rows = n * beams
    parents = {"beams": [r * beams + int(x) for r in range(n) for x in rng.integers(0, beams, beams)], "as they are": list(range(rows)), "ended": [-1] * rows,
               "some ended": [-1 if rng.random() < 0.3 else r // beams * beams + int(rng.integers(beams)) for r in range(rows)], "one": [rows // 2] * rows}
    if rows <= 256:                                      # rows of other requests too
        parents["any"] = rng.integers(-1, rows, rows).tolist()
        parents["turned round"] = list(range(rows))[::-1]
    for what, parent in parents.items():
        if what == "one" and rows > 512:
            continue
        why, want = ref.fork(parent, ctx, tables, shares, pad(free, num_pages), len(free), num_pages)
        assert why is None, what
        for budget in (None, 1, 5):
            same(run_fork(parent, ctx, tables, shares, free, len(free), num_pages, ws, status, budget), want)
    assert int(status) == 0


@pytest.mark.parametrize("what", ["parent too large", "parent too small", "negative length", "length beyond the row", "free count", "out of pages", "bad popped page", "bad owned page",
                                  "bad last page"])
def test_fork_pages_that_cannot_be_done(what, ws, status):
    rng = np.random.default_rng(8)
    ctx, tables, shares, free, num_pages = ref.shared_rows(rng, 2, 4, [37, 20], 10)
    parent, count = [1, 1, 2, 1, 4, 5, 4, -1], len(free)
    if what == "parent too large":
        parent[7] = 8
    elif what == "parent too small":
        parent[0] = -2
    elif what == "negative length":
        ctx[5] = -1
    elif what == "length beyond the row":
        ctx[5] = tables.shape[1] * 16 + 1
    elif what == "free count":
        count = num_pages + 1
    elif what == "out of pages":
        count = 2
    elif what == "bad popped page":
        free[count - 2] = num_pages
    elif what == "bad owned page":
        tables[0, 0] = tables[1, 0] = -3
    elif what == "bad last page":
        tables[4, 1] = 1 << 30
    why, want = ref.fork(parent, ctx, tables, shares, pad(free, num_pages), count, num_pages)
    assert why is not None
    for budget in (None, 1):
        status.zero_()
        same(run_fork(parent, ctx, tables, shares, free, count, num_pages, ws, status, budget), want)
        assert int(status) == STATUS[why]


def test_fork_keeps_what_lies_behind_the_rows(ws, status):
    """Rubbish behind a row's pages, and rows longer than any length, stay."""
    tables = np.full((3, 300), 12345, dtype=np.int32)
    tables[0, :2], tables[1, :1] = [4, 2], [7]
    why, want = ref.fork([0, 0, 1], [20, 5, 0], tables, [0] * 9, pad([1, 3, 5], 9), 3, 9)
    assert why is None and want["block_tables"][1, 2] == 12345
    same(run_fork([0, 0, 1], [20, 5, 0], tables, [0] * 9, [1, 3, 5], 3, 9, ws, status), want)


def test_pages_that_rows_outside_the_call_hold_stay(ws, status):
    """A cached prompt holds its pages through their count: the rows end, the pages stay out of the stack."""
    tables = np.full((2, 4), -1, dtype=np.int32)
    tables[:, :2] = [3, 1]
    got = run_fork([-1, -1], [32, 32], tables, [0, 2, 0, 1, 0], [0, 2], 2, 5, ws, status)
    assert got["shares"] == [0, 0, 0, 0, 0] and got["free_count"] == 3 and got["free_list"][:3] == [0, 2, 3] and got["ctx_len"] == [0, 0]


# ----------------------------------------------------------------------------------------------------------------- copies
@pytest.mark.parametrize("layers,heads,dim", [(1, 1, 8), (2, 3, 64), (3, 4, 128), (2, 2, 72), (1, 5, 256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1, 7, 60])
def test_copy_pages(layers, heads, dim, dtype, n, status):
    rng = np.random.default_rng(n + dim)
    pool = torch.from_numpy(rng.integers(0, 1 << 15, (layers, 2, 2 * n + 1, heads, 16, dim)).astype(np.int16)).view(dtype).to(DEV)
    order = rng.permutation(2 * n + 1)
    src, dst, length = order[:n].tolist(), order[n:2 * n].tolist(), rng.integers(0, 17, n).tolist()
    if n > 2:
        src[1], dst[2] = -1, -1
    for lens in (None, length):
        for budget in (None, 1, 3):
            got, want = pool.clone(), pool.clone()
            ops.copy_pages(got, i32(src), i32(dst), status, length=None if lens is None else i32(lens), sm_budget=budget)
            for i, (a, b) in enumerate(zip(src, dst)):
                if a >= 0 and b >= 0:
                    k = 16 if lens is None else lens[i]
                    want[:, :, b, :, :k] = pool[:, :, a, :, :k]
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)) and int(status) == 0


@pytest.mark.parametrize("src,dst,length,why", [(5, 1, 3, "BAD_BLOCK_TABLE"), (1, 5, 3, "BAD_BLOCK_TABLE"), (-2, 1, 3, "BAD_BLOCK_TABLE"), (1, -2, 3, "BAD_BLOCK_TABLE"),
                                                (1, 2, 17, "INVALID_ARG"), (1, 2, -1, "INVALID_ARG")])
def test_copies_that_are_refused_are_skipped(src, dst, length, why, status):
    pool = torch.randn(2, 2, 5, 1, 16, 64, device=DEV).bfloat16()
    got, want = pool.clone(), pool.clone()
    ops.copy_pages(got, i32([src, 3]), i32([dst, 4]), status, length=i32([length, 16]))
    want[:, :, 4] = pool[:, :, 3]
    assert torch.equal(got, want) and int(status) == STATUS[why]


# ------------------------------------------------------------------------------------------------------------- compaction
def run_compact(keep, ctx, tables, shares, free, count, num_pages, copies, ws, status, budget=None):
    t = [i32(x) for x in (ctx, tables, shares, pad(free, num_pages), [count])]
    out = [torch.full((copies,), -7, dtype=torch.int32, device=DEV) for _ in range(2)]
    ops.compact_pages(keep, *t, *out, ws, status, sm_budget=budget)
    torch.cuda.synchronize()
    assert control_words_are_zero(ws) and int(t[4]) == count
    return {"block_tables": t[1].cpu().numpy(), "shares": t[2].tolist(), "free_list": t[3].tolist(), "copy_src": out[0].tolist(), "copy_dst": out[1].tolist()}


@pytest.mark.parametrize("n,beams,most,spare", [(1, 1, 0, 1), (1, 1, 40, 33), (3, 2, 200, 64), (20, 8, 500, 700), (64, 4, 3000, 9000), (1000, 1, 30, 5)])
def test_compact_pages(n, beams, most, spare, ws, status):
    rng = np.random.default_rng(n + spare)
    ctx, tables, shares, free, num_pages = ref.shared_rows(rng, n, beams, [int(x) for x in rng.integers(0, most + 1, n)], spare)
    for keep in {num_pages, num_pages - 1, num_pages - spare // 2, num_pages - spare}:
        why, want = ref.compact(keep, ctx, tables, shares, pad(free, num_pages), len(free), num_pages, num_pages - keep + 3)
        assert why is None
        for budget in (None, 1, 7):
            same(run_compact(keep, ctx, tables, shares, free, len(free), num_pages, num_pages - keep + 3, ws, status, budget), want)
    assert int(status) == 0


@pytest.mark.parametrize("n,beams,most,spare", [(2, 3, 400, 8150), (2, 3, 400, 8300), (40, 8, 600, 5000), (300, 1, 900, 30000), (8, 8, 2000, 70001)])
def test_compact_pages_of_larger_pools(n, beams, most, spare, ws, status):
    test_compact_pages(n, beams, most, spare, ws, status)


@pytest.mark.parametrize("what", ["too many moves", "out of pages", "negative length", "length beyond the row", "free count", "a page twice", "a page outside", "bad entry", "a free entry"])
@pytest.mark.parametrize("spare", [40, 20000])
def test_compaction_that_cannot_be_done(what, spare, ws, status):
    rng = np.random.default_rng(9)
    ctx, tables, shares, free, num_pages = ref.shared_rows(rng, 3, 2, [100, 40, 64], spare)
    keep, copies, count = num_pages - spare // 2, 20, len(free)
    if what == "too many moves":
        copies = sum(p not in free for p in range(keep, num_pages)) - 1
    elif what == "out of pages":
        keep = 5
        copies = num_pages
    elif what == "negative length":
        ctx[2] = -1
    elif what == "length beyond the row":
        ctx[2] = tables.shape[1] * 16 + 1
    elif what == "free count":
        count = -1
    elif what == "a page twice":
        free[0] = free[1]
    elif what == "a page outside":
        free[0] = num_pages
    elif what == "bad entry":
        tables[1, 0] = num_pages
    elif what == "a free entry":
        tables[1, 0] = max(free)
    assert copies >= 0 and max(free) >= keep
    why, want = ref.compact(keep, ctx, tables, shares, pad(free, num_pages), count, num_pages, copies)
    assert why is not None
    for budget in (None, 1):
        status.zero_()
        same(run_compact(keep, ctx, tables, shares, free, count, num_pages, copies, ws, status, budget), want)
        assert int(status) == STATUS[why]


# -------------------------------------------------------------------------------------------------------------- selection
def run_select(x, scores, n_out, ws, status, done=None, weight=None, end=-1, scale=1.0, budget=None, shift=0, gap=0, full=True):
    """x on the GPU; its rows are copied `shift` elements off a boundary, `gap` more than their length apart."""
    n, b = scores.shape
    if shift or gap:
        wide = torch.full((x.shape[0] * (x.shape[1] + gap) + shift,), NAN, dtype=x.dtype, device=DEV)
        rows = wide[shift:].unflatten(0, (x.shape[0], x.shape[1] + gap))[:, :x.shape[1]]
        rows.copy_(x)
        x = rows
    score, parent, token, over = torch.full((n, n_out), 7.0, device=DEV), *(torch.full((n, n_out), -7, dtype=torch.int32, device=DEV) for _ in range(3))
    lse = torch.full((n * b,), 7.0, device=DEV)
    ops.beam_select(x, torch.tensor(scores, dtype=torch.float32, device=DEV), score, parent, token, ws, status, done=None if done is None else i32(done),
                    weight=None if weight is None else torch.tensor(weight, dtype=torch.float32, device=DEV), out_done=over if full else None, lse=lse if full else None,
                    end_token=end, scale=scale, sm_budget=budget)
    torch.cuda.synchronize()
    assert control_words_are_zero(ws)
    return score, parent, token, over, lse


def check_select(x, scores, n_out, ws, status, done=None, weight=None, end=-1, scale=1.0, exact_order=False, **how):
    """scores and weight are fp32 numbers in numpy arrays, x a tensor on the CPU."""
    got = run_select(x.to(DEV), scores, n_out, ws, status, done, weight, end, scale, **how)
    score, parent, token, over, lse = (t.cpu().double().numpy() for t in got)
    (n, b), x64 = scores.shape, x.double().numpy()
    want, want_lse = ref.select(x64, scores, done, weight, n_out, end, float(np.float32(scale)))
    # An exponential is off by 2^-22 of itself and by its argument's rounding, 2^-24 of at most 32 (ln 2 of it); a tile's sum of 32 by 2^-22, the sum of
    # tiles by 2^-23: log sum is off by 2.5e-6 at most.  A score is rounded once.
    span = 2.5e-6
    for r in range(n):
        for i in range(b):
            a, w = lse[r * b + i], want_lse[r * b + i]
            assert (math.isnan(a) and math.isnan(w)) or a == w or abs(a - w) <= span + 2.0 ** -23 * abs(w), (r, i, a, w)
        keys = [(int(parent[r, k]), int(token[r, k])) for k in range(n_out)]
        k = len(want[r])
        assert keys[k:] == [(-1, -1)] * (n_out - k) and (score[r, k:] == -INF).all() and (over[r, k:] == 0).all()
        assert len(set(keys[:k])) == k
        exact = {}
        for i in {p for p, _ in keys[:k]}:
            assert r * b <= i < (r + 1) * b
            i -= r * b
            row, s = x64[r * b + i], float(scores[r, i])
            if done is not None and done[r, i]:
                exact[i] = None
            else:
                top = row.max()
                exact[i] = s + (float(np.float32(scale)) * (row - top) - math.log(np.exp(float(np.float32(scale)) * (row - top)).sum()))
        for j, (ranked, i, v, s, ended) in enumerate(want[r]):
            assert abs(score[r, j] - s) <= span + 2.0 ** -23 * abs(s) + (0 if exact_order else span), (r, j, score[r, j], s)
            pi, pv = keys[j][0] - r * b, keys[j][1]
            mine = float(scores[r, pi]) if exact[pi] is None else exact[pi][pv]
            w = 1.0 if weight is None else float(weight[r, pi])
            if exact_order:
                assert (pi, pv) == (i, v), (r, j)
            else:                                        # (candidates nearer to one another than the error may change places)
                assert abs(w * mine - ranked) <= 2 * span * max(w, 1.0), (r, j)
            assert over[r, j] == (exact[pi] is None or pv == end)
    for budget in (1, 9):
        again = run_select(x.to(DEV), scores, n_out, ws, status, done, weight, end, scale, budget, **how)
        assert all(torch.equal(p.view(torch.int32), q.view(torch.int32)) for p, q in zip(got, again)), f"budget {budget}"


def logits(g, rows, vocab, dtype, spread=2.0):
    return (spread * torch.randn(rows, vocab, generator=g) + 8.0 * (torch.rand(rows, vocab, generator=g) < 6.0 / vocab)).to(dtype)


def beam_scores(rng, n, b):
    return (-10.0 - 2.0 * rng.random((n, b))).astype(np.float32)


@pytest.mark.parametrize("n,b,vocab,n_out", [(1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 7, 32), (1, 4, 1000, 8), (3, 2, 4096, 5), (5, 32, 257, 32), (2, 1, 70001, 16), (40, 8, 997, 16),
                                             (1, 1, 152064, 32), (300, 1, 33, 2), (2, 8, 20000, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_beam_select(n, b, vocab, n_out, dtype, ws, status):
    g, rng = torch.Generator().manual_seed(vocab + n), np.random.default_rng(vocab + n)
    check_select(logits(g, n * b, vocab, dtype), beam_scores(rng, n, b), n_out, ws, status, scale=0.8)
    assert int(status) == 0


@pytest.mark.parametrize("dtype,shift,gap", [(torch.float32, 1, 3), (torch.float32, 3, 1), (torch.bfloat16, 1, 1), (torch.bfloat16, 5, 8), (torch.float16, 7, 2)])
@pytest.mark.parametrize("vocab", [1, 3, 9, 4097, 30011])
def test_beam_select_of_rows_anywhere(dtype, shift, gap, vocab, ws, status):
    g, rng = torch.Generator().manual_seed(vocab), np.random.default_rng(vocab)
    check_select(logits(g, 6, vocab, dtype), beam_scores(rng, 2, 3), 4, ws, status, shift=shift, gap=gap)


@pytest.mark.parametrize("n,b,n_out", [(6, 4, 4), (9, 8, 8), (3, 1, 3), (2, 32, 20)])
def test_beam_select_with_ended_beams(n, b, n_out, ws, status):
    g, rng = torch.Generator().manual_seed(n), np.random.default_rng(n)
    done = (rng.random((n, b)) < 0.5).astype(np.int32)
    done[0] = 1                                          # nothing but ended beams
    done[-1] = 0
    weight = ((5 + rng.integers(0, 20, (n, b))) ** -0.6).astype(np.float32)
    scores = beam_scores(rng, n, b)
    x = logits(g, n * b, 3001, torch.bfloat16)
    x[torch.from_numpy(done.ravel()) > 0] = NAN          # (not read)
    x[:, 17] += 6.0
    check_select(x, scores, n_out, ws, status, done=done, weight=weight, end=17)
    check_select(x, scores, n_out, ws, status, done=done, end=17)
    got = run_select(x.to(DEV), scores, n_out, ws, status, done=done, end=17, full=False)
    assert bool((got[3] == -7).all()) and bool((got[4] == 7.0).all())


def test_equal_logits_go_by_their_tokens(ws, status):
    """Rows of few different values, rows of one value, rows that rise and fall, and beams that are exactly alike."""
    x = torch.zeros(6, 20000)
    g = torch.Generator().manual_seed(3)
    x[0] = torch.randint(0, 3, (20000,), generator=g).float()
    x[1] = 4.0
    x[2] = torch.arange(20000) / 1000.0
    x[3] = -torch.arange(20000) / 1000.0
    x[4, ::2] = 1.0
    x[5, 19990:] = 5.0
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for n_out in (1, 5, 32):
            check_select(x.to(dtype), np.zeros((6, 1), dtype=np.float32), n_out, ws, status, exact_order=True)
    same_rows = x[:1].repeat(4, 1)
    score, parent, token, _, _ = run_select(same_rows.to(DEV), np.full((1, 4), -3.0, dtype=np.float32), 32, ws, status)
    first = torch.nonzero(x[0] == 2.0)[:, 0][:32]
    assert parent.unique().tolist() == [0] and token[0].tolist() == first.tolist() and score.unique().numel() == 1
    few = torch.full((4, 3), 2.0)
    _, parent, token, _, _ = run_select(few.to(DEV), np.zeros((1, 4), dtype=np.float32), 12, ws, status)
    assert parent[0].tolist() == [0] * 3 + [1] * 3 + [2] * 3 + [3] * 3 and token[0].tolist() == [0, 1, 2] * 4


def test_more_ties_than_the_lists_hold(ws, status):
    """32 beams with one logit each in many parts: every candidate of the request ties."""
    x = torch.full((32, 152064), 1.5, dtype=torch.bfloat16)
    score, parent, token, _, _ = run_select(x.to(DEV), np.full((1, 32), -1.0, dtype=np.float32), 32, ws, status)
    assert parent[0].tolist() == [0] * 32 and token[0].tolist() == list(range(32))
    assert abs(float(score[0, 0]) + 1.0 + math.log(152064)) < 1e-5
    # all of one thread's pieces: what reaches the first bound is more than the list holds
    x = torch.zeros(1, 152064)
    at = (torch.arange(152064) // 4) % 1024 % 256 == 9
    x[0, at] = 3.0 + torch.arange(int(at.sum())) / 4096.0
    check_select(x, np.zeros((1, 1), dtype=np.float32), 32, ws, status, exact_order=True)


@pytest.mark.parametrize("b,vocab", [(8, 16000), (8, 152064), (32, 4097), (2, 152064), (3, 30000)])
@pytest.mark.parametrize("last", [0.0, -20.0, -1e4])
def test_a_beam_behind_all_others(b, vocab, last, ws, status):
    """A bound that holds for every part's first keys says little where one beam is far behind: most candidates of the others reach it."""
    scores = np.full((2, b), -1.0, dtype=np.float32) - 0.001 * np.arange(b, dtype=np.float32)
    scores[0, -1] += last
    scores[1, 0] += last
    check_select(logits(torch.Generator().manual_seed(b), 2 * b, vocab, torch.float32), scores, 32, ws, status, scale=0.8)
    assert int(status) == 0


@pytest.mark.parametrize("bad", [0.0, -0.5, NAN])
def test_a_weight_that_is_not_above_zero_gives_no_continuation(bad, ws, status):
    scores = np.zeros((2, 3), dtype=np.float32)
    weight, plain = np.ones((2, 3), dtype=np.float32), scores.copy()
    weight[1, 1], plain[1, 1] = bad, -INF
    x = logits(torch.Generator().manual_seed(8), 6, 3000, torch.bfloat16)
    done = np.array([[0, 0, 0], [0, 1, 0]], dtype=np.int32)
    for over in (None, done):
        status.zero_()
        got = run_select(x.to(DEV), scores, 5, ws, status, weight=weight, done=over)
        assert int(status) == STATUS["INVALID_ARG"]
        status.zero_()
        want = run_select(x.to(DEV), plain, 5, ws, status, done=over)
        assert int(status) == 0 and all(torch.equal(a, b) for a, b in zip(got[:4], want[:4]))
    status.zero_()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_masked_logits(dtype, scale, ws, status):
    """Rows masked with -infinity or with the type's lowest value, in part and from end to end; NaN, +infinity and beams that are not in use."""
    g = torch.Generator().manual_seed(1)
    low = torch.finfo(dtype).min
    x = logits(g, 12, 9001, dtype)
    x[0, 100:] = -INF
    x[1, :8990] = -INF
    x[2] = -INF
    x[3, 100:] = low
    x[4, :8990] = low
    x[5] = low
    x[5, 3] = -INF
    x[6, 4000] = NAN
    x[7, 4000] = INF
    x[8] = -INF
    x[8, 77] = -3.0
    x[9] = torch.finfo(dtype).max
    scores = np.full((12, 1), -1.5, dtype=np.float32)
    scores[10], scores[11] = -INF, NAN
    check_select(x, scores, 8, ws, status, scale=scale)
    assert int(status) == 0
    # the same as one request's beams: those without continuations do not disturb the others
    check_select(x, scores.reshape(1, 12), 32, ws, status, scale=scale)


@pytest.mark.parametrize("offset", [3e5, -3e5, 5e6, -5e6, 1e30, -1e30])
def test_logits_far_from_zero(offset, ws, status):
    x = torch.full((3, 5000), offset)
    x[0, 7] += abs(offset) * 2.0 ** -20
    x[1, ::3] -= abs(offset) * 2.0 ** -22
    x[2, 5:] = -INF
    check_select(x, beam_scores(np.random.default_rng(1), 3, 1), 6, ws, status)


# -------------------------------------------------------------------------------------------------------------- attention
def attention_case(seed, groups, hq, hkv, dim, dtype, cap=0.0, bias=False, scale=None, layer=1):
    """groups: (shared keys, [own keys of each sequence]).  Keys that no sequence has hold NaN, table entries behind them rubbish."""
    rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    kv = [s + n for s, own in groups for n in own]
    width = max(max(ref.pages(x) for x in kv), 1) + 1
    tables, num_pages = ref.grouped_tables(rng, groups, width)
    q = torch.randn(len(kv), hq, dim, generator=g).mul(3).to(dtype)
    pool = torch.randn(2, 2, num_pages, hkv, 16, dim, generator=g).to(dtype)
    seen = torch.zeros(num_pages, 16, dtype=torch.bool)
    for s, n in enumerate(kv):
        for j in range(n):
            seen[tables[s, j // 16], j % 16] = True
        for i in range(ref.pages(n), width):
            tables[s, i] = (-1, num_pages + 5)[i % 2]
    pool[layer, :, ~seen.unsqueeze(1).expand(-1, hkv, -1)] = NAN
    pool[1 - layer] = NAN
    return {"q": q, "pool": pool, "tables": tables, "kv": kv, "begin": np.cumsum([0] + [len(own) for _, own in groups]).tolist(), "shared": [s for s, _ in groups],
            "slopes": torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]) if bias else None, "scale": dim ** -0.5 if scale is None else scale, "cap": cap,
            "layer": layer}


def run_attention(c, ws, status, budget=None, strided=True, **change):
    c = c | change
    n, hq, dim = c["q"].shape
    wide = torch.full((n, hq * dim + 24), NAN, dtype=c["q"].dtype, device=DEV)
    q = wide[:, :hq * dim].unflatten(1, (hq, dim)) if strided else torch.empty(n, hq, dim, dtype=c["q"].dtype, device=DEV)
    q.copy_(c["q"])
    o_wide = torch.full((n, hq * dim + 8), 77.0, dtype=c["q"].dtype, device=DEV)
    o = o_wide[:, :hq * dim].unflatten(1, (hq, dim))
    lse = torch.full((n, hq), 55.0, device=DEV)
    ops.shared_attention(q, c["pool"].to(DEV), c["layer"], i32(c["tables"]), i32(c["kv"]), i32(c["begin"]), i32(c["shared"]), o, ws, status, lse=lse,
                         slopes=None if c["slopes"] is None else c["slopes"].to(DEV), scale=c["scale"], cap=c["cap"], sm_budget=budget)
    torch.cuda.synchronize()
    assert control_words_are_zero(ws) and bool((o_wide[:, hq * dim:] == 77.0).all())
    return o.contiguous(), lse


def check_attention(c, ws, status):
    o, lse = run_attention(c, ws, status)
    assert int(status) == 0
    kv = c["kv"]
    want_o, want_lse = device_ref.attention(c["q"].double(), c["pool"][c["layer"]].double(), c["tables"], kv, [1] * len(kv), None,
                                            None if c["slopes"] is None else c["slopes"].double(), c["scale"], c["cap"])
    # Weights and outputs are rounded to the cache's type once each (u of at most max |v|); a score is off by the fp32 sum of dim products
    # (dim 2^-24 sum |q k| scale, below 2e-4 at these inputs) and by 2e-7 cap, which moves o by twice that of max |v| and lse by that.
    u = 2.0 ** -8 if c["q"].dtype == torch.bfloat16 else 2.0 ** -11
    v = c["pool"][c["layer"], 1].double()
    vmax = float(v[~v.isnan()].abs().max()) if bool((~v.isnan()).any()) else 0.0
    o64, lse64 = o.cpu().double(), lse.cpu().double()
    assert not bool(o64.isnan().any()) and float((o64 - want_o).abs().max()) <= (2 * u + 5e-4) * vmax
    empty = want_lse == -INF
    assert bool((lse64[empty] == -INF).all()) and bool((o64[empty] == 0).all())
    assert bool(((lse64 - want_lse)[~empty].abs() <= 3e-4).all())
    for budget in (1, 9, 37):
        o2, lse2 = run_attention(c, ws, status, budget, strided=False)
        assert torch.equal(o2, o) and torch.equal(lse2, lse), f"budget {budget}"
    return o, lse


HEADS = [(28, 4, 128), (16, 4, 64), (5, 5, 64), (12, 1, 128), (34, 2, 64), (150, 1, 64), (16, 16, 128)]


@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, False), (0.0, True), (50.0, True)])
@pytest.mark.parametrize("hq,hkv,dim", HEADS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_shared_attention(cap, bias, hq, hkv, dim, dtype, ws, status):
    groups = [(40, [1, 9, 30]), (0, [5]), (100, [1]), (16, [0, 20, 0]), (130, [70, 1, 15, 16, 17]), (15, [1, 2])]
    check_attention(attention_case(3, groups, hq, hkv, dim, dtype, cap, bias), ws, status)


@pytest.mark.parametrize("groups", [[(0, [1])], [(1, [0])], [(0, [0])], [(0, [0, 0]), (0, [0])], [(16, [0])], [(64, [0, 0, 0])], [(2000, [1])], [(2000, [3] * 5)], [(0, [900, 3])],
                                    [(48, [0, 1, 16, 17, 64])], [(700, [1] * 40)], [(0, list(range(0, 60)))], [(33, [40] * 7), (900, [2] * 3), (5, [1] * 20)],
                                    [(1024, [64] * 19)], [(63, [1]), (64, [1]), (65, [1]), (127, [2]), (128, [2])]])
@pytest.mark.parametrize("hq,hkv", [(7, 1), (16, 1), (4, 4)])
def test_shared_attention_lengths(groups, hq, hkv, ws, status):
    check_attention(attention_case(len(groups), groups, hq, hkv, 128, torch.bfloat16), ws, status)


def test_shared_attention_of_many_sequences(ws, status):
    rng = np.random.default_rng(2)
    groups = [(int(rng.integers(0, 40)), rng.integers(0, 20, int(rng.integers(0, 9))).tolist()) for _ in range(500)]
    groups = [g for g in groups if g[1]]
    check_attention(attention_case(5, groups, 4, 2, 64, torch.float16), ws, status)
    check_attention(attention_case(6, [(20, rng.integers(0, 9, 1500).tolist())], 2, 1, 64, torch.bfloat16), ws, status)


@pytest.mark.parametrize("scale", [-0.1, 0.0, 3.0])
def test_shared_attention_scales(scale, ws, status):
    check_attention(attention_case(7, [(100, [5, 6]), (20, [40])], 8, 2, 64, torch.float16, scale=scale / 8), ws, status)


def test_shared_attention_agrees_with_paged_attention(ws, status):
    """The same rows by hs_op_paged_attention, which reads every sequence by itself; and with shared lengths left out, or counted too high."""
    c = attention_case(8, [(500, [20, 3, 60, 8]), (90, [300, 2])], 28, 4, 128, torch.bfloat16, cap=30.0)
    o, lse = run_attention(c, ws, status)
    want, want_lse = torch.empty_like(o), torch.empty_like(lse)
    ops.paged_attention(c["q"].to(DEV), c["pool"].to(DEV), 1, i32(c["tables"]), i32(c["kv"]), want, ws, status, lse=want_lse, scale=c["scale"], cap=30.0)
    for shared in (c["shared"], [0, 0], [100, 17]):
        o, lse = run_attention(c, ws, status, shared=shared)
        # both are within 2^-8 of max |v| (about 4.5) for the weights and as much for the output of the exact one
        assert float((o.float() - want.float()).abs().max()) <= 4 * 2.0 ** -8 * 5.0 and float((lse - want_lse).abs().max()) <= 6e-4
    high = run_attention(c, ws, status, shared=[503, 92])          # (the shortest sequences' own keys count, down to whole pages)
    assert torch.equal(high[0], run_attention(c, ws, status)[0]) and int(status) == 0


def test_sequences_outside_the_groups_are_left_alone(ws, status):
    c = attention_case(9, [(40, [3, 4]), (40, [5, 6, 7]), (0, [9])], 8, 2, 64, torch.float16)
    whole, whole_lse = run_attention(c, ws, status)
    o, lse = run_attention(c, ws, status, begin=[2, 2, 5], shared=[40, 40])
    # Where tiles are cut follows from the lengths of all of a call's sequences, so the two calls may join other parts.  Each is within (2 u + 5e-4) max |v| of the exact
    # outputs, u = 2^-11, and 3e-4 of the exact lse (check_attention), so they are within twice that of one another.
    v = c["pool"][1, 1].float()
    assert float((o[2:5].float() - whole[2:5].float()).abs().max()) <= 2 * (2 * 2.0 ** -11 + 5e-4) * float(v[~v.isnan()].abs().max())
    assert float((lse[2:5] - whole_lse[2:5]).abs().max()) <= 6e-4
    for rest in (slice(0, 2), slice(5, 6)):
        assert bool((o[rest] == 77.0).all()) and bool((lse[rest] == 55.0).all())
    o, _ = run_attention(c, ws, status, begin=[3, 3, 3], shared=[1, 1])
    assert bool((o == 77.0).all()) and int(status) == 0


@pytest.mark.parametrize("change", [dict(begin=[0, 3, 2, 6]), dict(begin=[-1, 2, 5, 6]), dict(begin=[0, 2, 5, 7]), dict(shared=[40, -1, 0])])
def test_shared_attention_refuses_groups_on_the_device(change, ws, status):
    c = attention_case(10, [(40, [3, 4]), (40, [5, 6, 7]), (0, [9])], 8, 2, 64, torch.float16)
    o, lse = run_attention(c, ws, status, **change)
    assert int(status) == B.HS_ERR_INVALID_ARG and bool((o == 77.0).all()) and bool((lse == 55.0).all())


@pytest.mark.parametrize("what", ["a shared page", "an own page", "a negative length", "a length beyond the row"])
def test_shared_attention_with_bad_tables(what, ws, status):
    c = attention_case(11, [(40, [3, 4]), (40, [5, 6, 7]), (0, [9])], 8, 2, 64, torch.float16)
    want, _ = run_attention(c, ws, status)
    tables, kv = c["tables"].copy(), list(c["kv"])
    if what == "a shared page":
        tables[2, 0] = 1 << 29
    elif what == "an own page":
        tables[3, 2] = -9
    elif what == "a negative length":
        kv[4] = -5
    else:
        kv[4] = tables.shape[1] * 16 + 1
    o, _ = run_attention(c, ws, status, tables=tables, kv=kv)
    assert int(status) == B.HS_ERR_BAD_BLOCK_TABLE
    assert torch.equal(o[:2], want[:2]) and torch.equal(o[5:], want[5:])


# ------------------------------------------------------------------------------------------------- streams, graphs, a loop
def test_on_other_streams_and_in_a_graph(ws, status):
    """All five on a side stream, captured once and replayed on other inputs, give what single calls give."""
    rng, g = np.random.default_rng(12), torch.Generator().manual_seed(12)
    c = attention_case(12, [(40, [3, 4, 5]), (300, [5, 6, 7])], 8, 2, 64, torch.float16)
    ctx, tables, shares, free, num_pages = ref.shared_rows(rng, 2, 3, [50, 23], 20)
    x = logits(g, 6, 5003, torch.bfloat16).to(DEV)

    def make():
        s = {"x": x.clone(), "scores": torch.tensor(beam_scores(np.random.default_rng(1), 2, 3), device=DEV), "score": torch.empty(2, 3, device=DEV),
             "parent": torch.empty(2, 3, dtype=torch.int32, device=DEV), "token": torch.empty(2, 3, dtype=torch.int32, device=DEV), "ctx": i32(ctx), "tables": i32(tables),
             "shares": i32(shares), "free": i32(pad(free, num_pages)), "count": i32([len(free)]), "copies": [torch.empty(6, dtype=torch.int32, device=DEV) for _ in range(3)],
             "pool": torch.randn(1, 2, num_pages, 2, 16, 64, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).half(),
             "moves": [torch.empty(9, dtype=torch.int32, device=DEV) for _ in range(2)], "q": c["q"].to(DEV), "cpool": c["pool"].to(DEV), "ctables": i32(c["tables"]),
             "kv": i32(c["kv"]), "begin": i32(c["begin"]), "shared": i32(c["shared"]), "o": torch.zeros_like(c["q"], device=DEV)}
        return s

    def step(s, ws):
        ops.shared_attention(s["q"], s["cpool"], 1, s["ctables"], s["kv"], s["begin"], s["shared"], s["o"], ws, status)
        ops.beam_select(s["x"], s["scores"], s["score"], s["parent"], s["token"], ws, status)
        ops.fork_pages(s["parent"].view(-1), s["ctx"], s["tables"], s["shares"], s["free"], s["count"], *s["copies"], ws, status)
        ops.copy_pages(s["pool"], s["copies"][0], s["copies"][1], status, length=s["copies"][2])
        ops.compact_pages(num_pages - 9, s["ctx"], s["tables"], s["shares"], s["free"], s["count"], *s["moves"], ws, status)
        ops.copy_pages(s["pool"], *s["moves"], status)

    def outputs(s):
        return [t.clone() for v in s.values() for t in (v if isinstance(v, list) else [v])]

    single = make()
    want = []
    for i in range(3):
        step(single, ws)
        want.append(outputs(single))
        single["x"].copy_(single["x"].roll(i + 1, 0))
    other_ws, side = ops.workspace(DEV), torch.cuda.Stream()
    captured = make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured, other_ws)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outputs(captured), want[i]):
            assert torch.equal(a.view(torch.int16) if a.dtype != torch.int32 else a, b.view(torch.int16) if b.dtype != torch.int32 else b)
        captured["x"].copy_(captured["x"].roll(i + 1, 0))
    assert int(status) == 0 and control_words_are_zero(other_ws)


@pytest.mark.parametrize("offset", [5e6, -5e6, 1e8])
@pytest.mark.parametrize("scale", [1.0, 0.8, 0.3, 3.7])
@pytest.mark.parametrize("below", [(0, 1), (0, 1, 2), (0, 9, 9, 9, 9, 9, 9), (0, 3, 5, 11, 17)])
def test_many_logits_far_from_zero(offset, scale, below, ws, status):
    """Whole rows (one for each team of threads of the device, so that none is cut) of few different logits, whose distances are small multiples of their type's step there: equal numbers are added up, so
    what each addition rounds away has one sign."""
    rows, vocab, step = 4 * ops.sm_count(0), 152064, float(np.spacing(np.float32(abs(offset))))
    away = step * torch.tensor(below, dtype=torch.float64)[torch.arange(vocab) % len(below)]
    x = (offset - away).float()
    assert bool((x.double() == offset - away).all())
    score, parent, token, over, _ = run_select(x.to(DEV).expand(rows, vocab).contiguous(), np.zeros((rows, 1), dtype=np.float32), 8, ws, status, scale=scale)
    assert torch.equal(token, torch.nonzero(x == offset)[:8, 0].int().to(DEV).expand(rows, 8)) and torch.equal(parent, torch.arange(rows, device=DEV).int()[:, None].expand(rows, 8))
    # log sum is off by 2.5e-6 at most (check_select), as a thread adds up at most 16 numbers before the sum goes on in more bits, and a score is rounded once
    want = -math.log(float(torch.exp(-float(np.float32(scale)) * away).sum()))
    assert float((score.double() - want).abs().max()) <= 2.5e-6 + 2.0 ** -24 * abs(want) and int(status) == 0


@pytest.mark.parametrize("scale,largest", [(1e-30, 2e31), (1e-36, 1e37), (1e-37, 2e38), (3e-38, 3e38), (1e-40, 3e38)])
@pytest.mark.parametrize("vocab", [7, 5000])
def test_small_scales_of_large_logits(scale, largest, vocab, ws, status):
    x = (largest / 4 * torch.randn(6, vocab, generator=torch.Generator().manual_seed(vocab))).clamp(-largest, largest)
    x[1, ::3] = -INF
    x[2, :] = largest
    check_select(x, beam_scores(np.random.default_rng(2), 3, 2), 5, ws, status, scale=scale)
    assert int(status) == 0


@pytest.mark.parametrize("weighted", [False, True])
def test_scores_beyond_fp32_are_held_to_its_largest_number(weighted, ws, status):
    """Masked with the type's lowest value, sharpened, few tokens left: the continuations behind those have scores, though none that fp32 holds."""
    most, x = float(torch.finfo(torch.float32).max), torch.full((4, 900), torch.finfo(torch.float32).min)
    x[:, 5], x[:, 7], x[2] = 1.0, 2.0, most
    scores = np.array([[-1.0, -2.0], [-3.0, -most]], dtype=np.float32)
    weight = np.full((2, 2), 0.25, dtype=np.float32) if weighted else None
    score, parent, token, _, lse = run_select(x.to(DEV), scores, 6, ws, status, weight=weight, scale=2.0)
    want, _ = ref.select(x.double().numpy(), scores, None, weight, 6, -1, 2.0)
    assert [(int(p), int(t)) for p, t in zip(parent.flatten(), token.flatten())] == [(2 * r + i, v) for r in range(2) for _, i, v, _, _ in want[r]]
    exact = torch.tensor([[s for _, _, _, s, _ in w] for w in want], dtype=torch.float64)
    assert float(exact.min()) < -most
    held = exact.clamp(-most, most)
    assert bool(((score.cpu().double() - held).abs() <= 2.5e-6 + 2.0 ** -24 * held.abs()).all()) and bool(score.isfinite().all())
    assert float(lse[2]) == most and int(status) == 0     # (2 * most and the logarithm of 900)


@pytest.mark.parametrize("b,vocab,n_out", [(1, 152064, 8), (4, 152064, 8), (32, 152064, 32), (3, 50, 5), (8, 9000, 32), (2, 40, 32)])
@pytest.mark.parametrize("start", [-1e30, float(np.finfo(np.float32).min), 1e30])
def test_beams_so_far_away_that_their_continuations_tie(b, vocab, n_out, start, ws, status):
    """A score next to which differences of logits vanish, in 64 bits too: the order is that of the exact scores, beam by beam and from the largest logit down."""
    x = logits(torch.Generator().manual_seed(vocab), 2 * b, vocab, torch.float32)
    x[:, 3] = x.amax(1)                                   # (a logit that a row has twice: the lower token first)
    scores = np.full((2, b), start, dtype=np.float32)
    scores[1, -1] *= 2.0 if start == -1e30 else 0.5       # (one beam of the second request is behind the others or in front of them)
    over = np.zeros((2, b), dtype=np.int32)
    over[0, b // 2] = int(b > 2)
    score, parent, token, _, _ = run_select(x.to(DEV), scores, n_out, ws, status, done=over, end=5)
    order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices
    for r in range(2):
        want = []
        for i in sorted(range(b), key=lambda i: -float(scores[r, i])):
            want += [(r * b + i, 5)] if over[r, i] else [(r * b + i, int(v)) for v in order[r * b + i][:n_out]]
        got = list(zip(parent[r].tolist(), token[r].tolist()))
        assert got[:len(want)] == want[:n_out] and set(got[len(want):]) <= {(-1, -1)}
        assert all(s == scores[r, p - r * b] for s, p in zip(score[r].cpu().numpy(), parent[r].tolist()) if p >= 0)
    assert int(status) == 0


BAD_V = [("an own key", NAN), ("an own key", INF), ("a coordinate", -INF), ("a coordinate", NAN), ("two sequences", INF), ("a shared key", NAN), ("the last key", INF)]


@pytest.mark.parametrize("what,bad", BAD_V)
@pytest.mark.parametrize("groups,hq,hkv,dim,dtype,cap,bias", [
    ([(40, [5, 9, 30]), (100, [1]), (130, [70, 4, 15, 16, 17]), (0, [7, 8])], 28, 4, 128, torch.bfloat16, 0.0, False),
    ([(40, [5, 9, 30]), (100, [1]), (130, [70, 4, 15, 16, 17]), (0, [7, 8])], 16, 4, 64, torch.float16, 30.0, True),
    ([(3000, [40, 9, 100])], 4, 1, 128, torch.float16, 0.0, False), ([(0, [0, 40, 9, 0])], 4, 1, 64, torch.bfloat16, 0.0, False), ([(900, [30] * 40)], 7, 1, 64, torch.bfloat16, 50.0, False),
    ([(0, [700, 3, 64, 90]), (2000, [64] * 9)] * 3, 6, 2, 128, torch.bfloat16, 0.0, True), ([(60, [20, 40])], 150, 1, 64, torch.bfloat16, 0.0, False)])
def test_a_v_that_is_no_number_stays_with_the_rows_that_see_it(what, bad, groups, hq, hkv, dim, dtype, cap, bias, ws, status):
    """Infinities and NaN in v at keys of one sequence or two (one tile, tiles that two teams have, tiles cut between shares): the others are as the definition has them."""
    c = attention_case(21, groups, hq, hkv, dim, dtype, cap, bias)
    v = c["pool"][c["layer"], 1]
    for s in range(1, min(3, len(c["kv"])) if what == "two sequences" else 2):
        kv = c["kv"][s]
        j = {"a shared key": min(20, kv - 1), "the last key": kv - 1}.get(what, max(kv - 2, 0))
        at = v[int(c["tables"][s, j // 16]), :, j % 16]
        at[..., 3 if what == "a coordinate" else slice(None)] = bad
    o, lse = run_attention(c, ws, status)
    want_o, want_lse = device_ref.attention(c["q"].double(), c["pool"][c["layer"]].double(), c["tables"], c["kv"], [1] * len(c["kv"]), None,
                                            None if c["slopes"] is None else c["slopes"].double(), cap=c["cap"], scale=c["scale"])
    whole, o64 = want_o.isfinite(), o.cpu().double()
    assert (bool(whole.any()) or what == "a shared key") and not bool(whole.all())     # (a key that all rows share reaches all of them)
    assert torch.equal(o64.isfinite(), whole) and torch.equal(o64.isnan(), want_o.isnan())
    assert torch.equal(o64[o64.isinf()], want_o[want_o.isinf()])
    u, most = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11, float(v.double()[v.isfinite()].abs().max())       # (bounds of check_attention)
    assert float((o64 - want_o)[whole].abs().amax(dim=0) if bool(whole.any()) else 0.0) <= (2 * u + 5e-4) * most
    some = want_lse > -INF
    assert bool((lse.cpu()[~some] == -INF).all()) and float((lse.cpu().double() - want_lse)[some].abs().max()) <= 3e-4
    for budget in (1, 9, 37):
        o2, lse2 = run_attention(c, ws, status, budget, strided=False)
        assert torch.equal(o2.view(torch.int16), o.view(torch.int16)) and torch.equal(lse2, lse), f"budget {budget}"
    assert int(status) == 0
