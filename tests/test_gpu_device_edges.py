"""Arguments at their ends, on a B200: scales and caps of every size, lengths up to the limit, page tables and logits that hold what they should not."""
import math

import numpy as np
import pytest
import torch

from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_ops as ops
from tests import device_ref as ref
from tests.test_gpu_device_ops import DEV, NAN, attention_case, check_attention, control_words_are_zero, i32, run_attention, run_logprobs, status, ws  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [-0.125, 0.0, 1e-39, -1e-3])
@pytest.mark.parametrize("q,kv", [([1, 1, 1], [75, 40, 200]), ([70, 3, 16], [75, 40, 200]), ([4], [2000])])
@pytest.mark.parametrize("cap,window,prefix,bias", [(0.0, 0, 0, False), (0.0, 17, 21, False), (30.0, 0, 0, False), (0.0, 0, 0, True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_of_scales_that_are_not_positive(scale, q, kv, cap, window, prefix, bias, dtype, ws, status):
    """The smallest key's score is the largest, or all are alike; masked keys stay at -infinity.  (No scale is above head_dim^-1/2, which check_attention's
    tolerance is made for.)"""
    c = attention_case(11, kv, q, 8, 2, 64, dtype, cap, window, prefix, bias)
    c["scale"] = scale
    check_attention(c, ws, status)


@pytest.mark.parametrize("scale,cap", [(128 ** -0.5, 50.0), (1 / 128, 100.0), (1 / 64, 300.0), (128 ** -0.5, 1000.0), (128 ** -0.5, 2000.0), (0.01, 40000.0)])
@pytest.mark.parametrize("q", [[1] * 6, [40, 1, 2, 33, 64, 7]])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_attention_of_caps_of_every_size(scale, cap, q, bias, dtype, ws, status):
    """Scores up to a given share y of the cap, of either sign, one sequence for each y: the sum of a row is that of its largest score."""
    ys, dim, kv = [0.2, 0.345, 0.5, 0.6, 0.69, 0.95], 128, [200, 130, 77, 300, 64, 140]
    c = attention_case(12, kv, q, 4, 2, dim, dtype, cap, 0, 0, bias, poison=False)
    c["scale"] = scale
    u = torch.tensor([1.0, -1.0, -1.0, 1.0] * (dim // 4))
    row = 0
    for s, y in enumerate(ys):
        want = y * cap / (scale * dim)                     # of the products of a coordinate of q and of k
        a = torch.tensor(2.0 ** round(math.log2(want) / 2))
        c["q"][row:row + q[s]] = (a * u).to(dtype)
        row += q[s]
        for j in range(kv[s]):
            share = (1.0, -0.8, 0.0, 0.5, -1.0, 0.7, 0.1)[j % 7]
            c["pool"][1, 0, int(c["tables"][s, j // 16]), :, j % 16] = (want / a * share * u).to(dtype)
    o, lse = run_attention(c, ws, status)
    want_o, want_lse = ref.attention(c["q"].double(), c["pool"][1].double(), c["tables"], kv, q, None, None if c["slopes"] is None else c["slopes"].double(), scale, cap, 0)
    # q . k is exact in fp32 (128 equal products of 16 bits and a sign).  The capped score is within 4e-9 cap of the polynomial, which is added up in at
    # most seven roundings of about its value (or 3e-7 cap by the exponential), and the bias, the maximum's distance and the change to natural
    # logarithms round four times more: 11 of 2^-24 of at most 0.75 cap + 2^-8 of the bias's slope, below 1e-6 cap.  Weights and outputs as in check_attention.
    tol = 1e-6 * cap + 3e-5
    vmax, r = float(c["pool"][1, 1].abs().max()), 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    assert float((lse.cpu().double() - want_lse).abs().max()) <= tol
    assert float((o.cpu().double() - want_o).abs().max()) <= (2 * r + 2 * tol) * vmax
    assert int(status) == 0


@pytest.mark.parametrize("scale,cap", [(0.125, 1e-40), (1e20, 1e-25), (-1e20, 1e-25)])
@pytest.mark.parametrize("q", [[1, 1], [9, 70]])
def test_attention_of_caps_far_below_the_scale(scale, cap, q, ws, status):
    """scale / cap is beyond fp32; every score is the cap or, where q . k is 0, 0."""
    c = attention_case(13, [40, 130], q, 4, 2, 64, torch.bfloat16, cap, 0, 0, False)
    c["scale"] = scale
    c["q"][0] = 0
    c["q"][-1, 1] = 0
    check_attention(c, ws, status)


@pytest.mark.parametrize("q", [[40], [200], [3, 70]])
@pytest.mark.parametrize("cap,bias", [(0.0, False), (30.0, False), (0.0, True)])
def test_chunks_do_not_depend_on_the_width_of_the_block_table(q, cap, bias, ws, status):
    """The same call with columns behind every sequence's pages, by which the launch takes the kernel that can divide items: the same bits."""
    c = attention_case(15, [448, 300][:len(q)], q, 8, 2, 64, torch.bfloat16, cap, 0, 0, bias)
    o, lse = run_attention(c, ws, status)
    c["tables"] = np.concatenate([c["tables"], np.full((len(q), 60), -1, dtype=np.int32)], 1)
    wide_o, wide_lse = run_attention(c, ws, status)
    assert torch.equal(o, wide_o) and torch.equal(lse, wide_lse) and int(status) == 0


LONGEST = 2 ** 31 - 64                                      # of a sequence


def test_the_longest_block_table_row(ws, status):
    """One request whose row has all the pages that a call can have: short and longest lengths, and one beyond."""
    width = 1 << 27
    tables = torch.full((1, width), -1, dtype=torch.int32, device=DEV)
    free, count = i32([7, 6, 5]), i32([3])
    outs = [torch.empty(m, dtype=torch.int32, device=DEV) for m in (2, 40, 40, 40)]
    kv = i32([0])
    ops.step_tables(i32([0]), i32([20]), free, count, tables, kv, *outs, count, ws, status)
    assert int(status) == B.HS_ERR_BAD_BLOCK_TABLE            # (pages 5 and 6 of a pool of three)
    status.zero_()
    count.fill_(3)
    free = i32([2, 1, 0])
    ctx = i32([0])
    ops.step_tables(ctx, i32([20]), free, count, tables, ctx, *outs, count, ws, status)
    assert int(status) == 0 and int(ctx) == 20 and int(count) == 1 and tables[0, :3].tolist() == [0, 1, -1]
    assert outs[3][:20].tolist() == list(range(20)) and outs[3][20:].tolist() == [-1] * 20
    ops.release_pages(i32([1]), ctx, tables, free, count, ws, status)
    assert int(status) == 0 and int(ctx) == 0 and free.tolist() == [2, 1, 0] and tables[0, :3].tolist() == [-1] * 3
    tables[0, -5:] = 2
    ctx.fill_(LONGEST - 3)
    for q, why in ((3, 0), (4, B.HS_ERR_INVALID_ARG), (2 ** 31 - 1, B.HS_ERR_INVALID_ARG)):
        status.zero_()
        kv.fill_(-9)
        outs[2].fill_(-9)
        ops.step_tables(ctx, i32([q]), free, count, tables, kv, *outs, count, ws, status)
        assert int(status) == why and int(kv) == LONGEST - (0 if why == 0 else 3)
        assert outs[2][:4].tolist() == ([LONGEST - 3, LONGEST - 2, LONGEST - 1, -1] if why == 0 else [-1] * 4)
    assert control_words_are_zero(ws)


@pytest.mark.parametrize("q,cap", [([1], 0.0), ([40], 0.0), ([40], 30.0), ([200], 0.0)])
def test_attention_at_the_longest_length(q, cap, ws, status):
    """Under a window, so that a sequence of 2^31 - 64 keys looks at the pages of one of 448."""
    near, width = 448, 1 << 27
    c = attention_case(14, [near], q, 8, 2, 64, torch.bfloat16, cap, 100, 0, False)
    o, lse = run_attention(c, ws, status)
    tables = torch.full((1, width), -1, dtype=torch.int32, device=DEV)
    tables[0, (LONGEST - near) // 16:LONGEST // 16] = i32(c["tables"][0, :near // 16])
    args = [c["q"].to(DEV), c["pool"].to(DEV), 1, tables]
    begin = i32([0, q[0]])
    got, got_lse = torch.empty_like(args[0]), torch.empty_like(lse)
    ops.paged_attention(*args, i32([LONGEST]), got, ws, status, lse=got_lse, tok_begin=begin, max_q_len=q[0], scale=c["scale"], cap=cap, window=100)
    assert int(status) == 0 and torch.equal(got, o) and torch.equal(got_lse, lse)
    ops.paged_attention(*args, i32([LONGEST + 1]), got, ws, status, tok_begin=begin, max_q_len=q[0], scale=c["scale"], cap=cap, window=100)
    assert int(status) == B.HS_ERR_BAD_BLOCK_TABLE and control_words_are_zero(ws)


def test_a_step_with_room_for_almost_all_tokens_that_a_number_counts(ws, status):
    """Per-token arrays of 2^31 - 100 entries (8.6 GB each), which no whole number of the grid's threads fits below 2^31."""
    cap = 2 ** 31 - 100
    tok = [torch.zeros(cap, dtype=torch.int32, device=DEV) for _ in range(3)]
    count, kv = i32([3]), i32([0, 0])
    ops.step_tables(i32([0, 0]), i32([20, 1]), i32([0, 1, 2]), count, torch.full((2, 4), -1, dtype=torch.int32, device=DEV), kv, i32([0] * 3), *tok, count, ws, status)
    assert int(status) == 0 and kv.tolist() == [20, 1] and int(count) == 0
    # (pages 2 and 1 for the first request, 0 for the second)
    assert [t[19:23].tolist() for t in tok] == [[0, 1, -1, -1], [19, 0, -1, -1], [19, 0, -1, -1]]
    for t in tok:
        for i in range(21, cap, 1 << 28):
            assert bool((t[i:i + (1 << 28)] == -1).all())
    assert control_words_are_zero(ws)


@pytest.mark.parametrize("n", [3, 1500])
@pytest.mark.parametrize("wrong", [-1, "beyond"])
def test_release_of_a_row_that_holds_no_page(n, wrong, ws, status):
    """A page id outside the pool is not put on the stack: nothing is given back, and the status says why."""
    rng = np.random.default_rng(n)
    ctx = rng.integers(1, 100, n)
    num_pages = sum(ref.pages(c) for c in ctx) + 3
    tables, free = ref.random_tables(rng, ctx, 7, num_pages)
    done = rng.integers(0, 2, n)
    done[1] = 1
    pad = free.tolist() + [-5] * (num_pages - len(free))
    keep = int(tables[1, ref.pages(ctx[1]) - 1])
    tables[1, ref.pages(ctx[1]) - 1] = num_pages if wrong == "beyond" else wrong
    for budget in (None, 1, 5):
        status.zero_()
        t = [i32(done), i32(ctx), i32(tables), i32(pad), i32([len(free)])]
        ops.release_pages(*t, ws, status, sm_budget=budget)
        assert int(status) == B.HS_ERR_BAD_BLOCK_TABLE
        assert t[1].tolist() == ctx.tolist() and np.array_equal(t[2].cpu().numpy(), tables) and int(t[4]) == len(free) and t[3][:len(free)].tolist() == free.tolist()
        assert control_words_are_zero(ws)
        # and mended, the same call is done
        status.zero_()
        t[2][1, ref.pages(ctx[1]) - 1] = keep
        whole = tables.copy()
        whole[1, ref.pages(ctx[1]) - 1] = keep
        want = ref.release_pages(done, ctx, whole, pad, len(free))
        ops.release_pages(*t, ws, status, sm_budget=budget)
        assert int(status) == 0 and t[1].tolist() == [int(x) for x in want[0]] and np.array_equal(t[2].cpu().numpy(), want[1])
        assert int(t[4]) == want[3] and t[3][:want[3]].tolist() == [int(x) for x in want[2][:want[3]]] and control_words_are_zero(ws)


@pytest.mark.parametrize("rows,vocab", [(3, 9), (2, 5001), (4, 5001), (3, 152064), (150, 40000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rank_in_rows_that_are_not_numbers(rows, vocab, dtype, ws, status):
    """The logits above the target are counted whatever else the row holds; none is above a target that is not a number."""
    g = torch.Generator().manual_seed(vocab)
    x = (3 * torch.randn(rows, vocab, generator=g)).to(dtype)
    targets = torch.randint(0, vocab, (rows,), generator=g).tolist()
    for r in range(rows - 1):
        x[r, torch.randint(0, vocab, (vocab // 500 + 1,), generator=g)] = NAN
        x[r, torch.randint(0, vocab, (2,), generator=g)] = math.inf
    targets[0] = int(x[0].isnan().nonzero()[0])
    got = run_logprobs(x.to(DEV), targets, 5, 1.0, ws, status)
    assert got["rank"].tolist() == [int((x[r] > x[r, t]).sum()) for r, t in enumerate(targets)]
    assert bool(got["logprob"][:rows - 1].isnan().all()) and bool(got["logprob"][rows - 1:].isfinite().all()) and int(status) == 0


def test_token_logprobs_of_long_rows_that_one_warp_looks_through(ws, status):
    """Rows whose first tile is masked, and so long that the warp that finds their alternatives takes longer than the 2 s of an ordinary wait; blocks of three rows each,
    whose readers wait for it meanwhile."""
    rows, vocab, last = 148, 220_000_000, 4096
    x = torch.full((rows, vocab), -math.inf, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(9)
    x[:, vocab - last:] = (3 * torch.randn(rows, last, generator=g, device=DEV)).bfloat16()
    got = run_logprobs(x, [vocab - 1 - r for r in range(rows)], 3, 1.0, ws, status, budget=50)
    assert int(status) == 0
    part = x[:, vocab - last:].cpu().double()
    lp = torch.log_softmax(part, 1)
    for r in range(rows):
        order = torch.sort(-part[r], stable=True).indices[:3]
        assert got["top_ids"][r].tolist() == (order + vocab - last).tolist() and int(got["rank"][r]) == int((part[r] > part[r, last - 1 - r]).sum())
        # (as in check_logprobs: logits below 20)
        assert abs(float(got["logprob"][r]) - float(lp[r, last - 1 - r])) <= 2e-5
    del x
    torch.cuda.empty_cache()
