"""The beam search loop on the CPU: its operators are the plain definitions here, its model is a table of the tokens that the cache holds, so that a page that is
forked, copied or moved wrongly changes what is generated."""
import math
import zlib

import numpy as np
import pytest
import torch

from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_loop
from paper_2608_01785_b200 import device_ops as ops
from paper_2608_01785_b200.device_loop import BeamLoop, LoopDims, make_weights
from tests import beam_ref as R

DIMS = LoopDims(n_layers=1, d_model=64, n_q_heads=1, n_kv_heads=1, head_dim=64, vocab=64)
STATUS = {"OUT_OF_PAGES": B.HS_ERR_OUT_OF_PAGES, "INVALID_ARG": B.HS_ERR_INVALID_ARG}


def logits_of(tokens):
    return 2 * torch.randn(DIMS.vocab, generator=torch.Generator().manual_seed(zlib.crc32(bytes(tokens))))


def set_status(st, name):
    if name:
        st.fill_(STATUS[name])


def step_tables(ctx, q, free_list, free_count, tables, kv_len, begin, seq, pos, slot, free_out, ws, st, sm_budget=None):
    for t in (seq, pos, slot):
        t.fill_(-1)
    need = sum(R.pages(int(c + k)) - R.pages(int(c)) for c, k in zip(ctx, q))
    kv_len.copy_(ctx)
    begin.zero_()
    if need > int(free_count):
        return set_status(st, "OUT_OF_PAGES")
    t = 0
    for s in range(len(ctx)):
        for i in range(int(ctx[s]), int(ctx[s] + q[s])):
            if i % 16 == 0:
                free_count -= 1
                tables[s, i // 16] = free_list[int(free_count)]
            seq[t], pos[t], slot[t] = s, i, int(tables[s, i // 16]) * 16 + i % 16
            t += 1
        begin[s + 1] = t
    kv_len.copy_(ctx + q)


def beam_select(logits, scores, out_score, out_parent, out_token, ws, st, done=None, weight=None, out_done=None, lse=None, end_token=-1, scale=1.0, sm_budget=None):
    n, b = scores.shape
    chosen, _ = R.select(logits.double().numpy(), scores.double().numpy(), done.numpy() if done is not None else None, weight.double().numpy() if weight is not None else None,
                         out_score.shape[1], end_token, scale)
    out_score.fill_(-math.inf)
    out_parent.fill_(-1)
    out_token.fill_(-1)
    out_done.fill_(0)
    for r in range(n):
        for i, (_, beam, token, score, over) in enumerate(chosen[r]):
            out_score[r, i], out_parent[r, i], out_token[r, i], out_done[r, i] = score, r * b + beam, token, int(over)


def fork_pages(parent, ctx, tables, shares, free_list, free_count, src, dst, length, ws, st, sm_budget=None):
    name, left = R.fork(parent.tolist(), ctx.tolist(), tables.numpy().astype(np.int64), shares.tolist(), free_list.tolist(), int(free_count), shares.numel())
    set_status(st, name)
    for t, k in ((ctx, "ctx_len"), (tables, "block_tables"), (shares, "shares"), (free_list, "free_list"), (src, "copy_src"), (dst, "copy_dst"), (length, "copy_len")):
        t.copy_(torch.as_tensor(np.asarray(left[k])))
    free_count.fill_(left["free_count"])


def copy_pages(pool, src, dst, st, length=None, sm_budget=None):
    for i, (a, b) in enumerate(zip(src.tolist(), dst.tolist())):
        if a >= 0 and b >= 0:
            n = 16 if length is None else int(length[i])
            pool[:, :, b, :, :n] = pool[:, :, a, :, :n]


def compact_pages(keep, ctx, tables, shares, free_list, free_count, src, dst, ws, st, sm_budget=None):
    name, left = R.compact(keep, ctx.tolist(), tables.numpy().astype(np.int64), shares.tolist(), free_list.tolist(), int(free_count), shares.numel(), src.numel())
    set_status(st, name)
    for t, k in ((tables, "block_tables"), (shares, "shares"), (free_list, "free_list"), (src, "copy_src"), (dst, "copy_dst")):
        t.copy_(torch.as_tensor(np.asarray(left[k])))


class Loop(BeamLoop):
    """With a model whose logits follow from the tokens that the cache holds for a row."""

    def _layers(self, b, max_q_len):
        for slot, token in zip(b["slot"].tolist(), b["tokens"].tolist()):
            if slot >= 0:
                self.pool[0, 0, slot // 16, 0, slot % 16, 0] = token
        self.decodes = max_q_len == 1

    def _head(self, b, n):
        for i in range(n):
            row = i if self.decodes else i * self.n_beams
            held = [int(self.pool[0, 0, int(self.tables[row, j // 16]), 0, j % 16, 0]) for j in range(int(b["kv_len"][row]))]
            b["logits"][i] = logits_of(held)

    def step(self):
        self._decode()


@pytest.fixture()
def plain(monkeypatch):
    for f in (step_tables, beam_select, fork_pages, copy_pages, compact_pages):
        monkeypatch.setattr(ops, f.__name__, f)
    monkeypatch.setattr(ops, "rope_table", lambda *a, **k: None)
    monkeypatch.setattr(ops, "workspace", lambda d: torch.zeros(1))
    monkeypatch.setattr(B, "make_head_config", lambda *a: None)
    monkeypatch.setattr(B, "hs_head_workspace_bytes", lambda cfg: 256)
    monkeypatch.setattr(B, "hs_head_create", lambda *a: 1)
    monkeypatch.setattr(B, "hs_head_destroy", lambda h: None)


def search(prompt, beams, steps, end_token=-1, penalty=0.0):
    """Beam search from its definition: [(score, tokens)], best first."""
    hyps = [(0.0, [], False)]
    for _ in range(steps):
        new = []
        for score, tokens, over in hyps:
            if over:
                new.append((score, tokens, True))
                continue
            lp = torch.log_softmax(logits_of(prompt + tokens).double(), 0)
            new += [(score + float(lp[v]), tokens + [v], v == end_token) for v in range(DIMS.vocab)]
        hyps = sorted(new, key=lambda h: -h[0] / len(h[1]) ** penalty)[:beams]
    return [(s, t) for s, t, _ in hyps]


def prompts(*lens):
    g = torch.Generator().manual_seed(5)
    return [torch.randint(0, DIMS.vocab, (n,), generator=g).tolist() for n in lens]


def check_pages(loop):
    """Every page is free or held, `shares` counts the holders behind the first, and a last page that is not full has one."""
    num, held, last = loop.shares.numel(), {}, []
    for row, c in zip(loop.tables.tolist(), loop.ctx_len.tolist()):
        for i in range(R.pages(c)):
            held[row[i]] = held.get(row[i], 0) + 1
        if c % 16:
            last.append(row[c // 16])
    assert sorted(list(held) + loop.free_list[:int(loop.free_count)].tolist()) == list(range(num))
    assert loop.shares.tolist() == [max(held.get(p, 0) - 1, 0) for p in range(num)]
    assert all(held[p] == 1 for p in last)


def same(got, want):
    assert [t for _, t in got] == [t for _, t in want]
    for (a, _), (b, _) in zip(got, want):
        assert abs(a - b) <= 2e-5 * (1 + abs(b))          # (scores are kept in fp32: some twenty roundings of 2^-24)


@pytest.mark.parametrize("beams", [1, 2, 5])
@pytest.mark.parametrize("end_token,penalty", [(-1, 0.0), (7, 0.0), (7, 0.8), (-1, 1.0)])
def test_the_beams_are_those_of_the_definition(plain, beams, end_token, penalty):
    p = prompts(1, 15, 16, 33)
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 4, beams, 80, 64, sum(map(len, p)), 20, end_token=end_token, length_penalty=penalty)
    loop.prefill(p)
    for step in range(1, 21):
        assert int(loop.status) == 0
        check_pages(loop)
        if step in (1, 2, 18, 20):
            for r, got in enumerate(loop.hypotheses()):
                same(got, search(p[r], beams, step, end_token, penalty))
        loop.step()
    same(loop.hypotheses()[0], search(p[0], beams, 20, end_token, penalty))         # steps behind max_tokens change nothing
    assert loop.q_len.tolist() == [0] * loop.n
    loop.finish(torch.ones(4, dtype=torch.int32))
    assert int(loop.free_count) == 80 and loop.hypotheses() == [[], [], [], []]
    loop.close()


@pytest.mark.parametrize("copies", [16384, 3])
def test_a_request_ends_while_others_go_on_in_a_smaller_pool(plain, copies, monkeypatch):
    monkeypatch.setattr(device_loop, "COPIES", copies)     # (pages that move at a time)
    p = prompts(20, 3, 40)
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 3, 3, 60, 80, sum(map(len, p)), 30)
    loop.prefill(p)
    for _ in range(9):
        loop.step()
    loop.finish(torch.tensor([0, 1, 0], dtype=torch.int32))
    check_pages(loop)
    used = 60 - int(loop.free_count)
    with pytest.raises(B.HsError):
        loop.shrink(used - 1)
    check_pages(loop)
    loop.shrink(used + 8)
    assert loop.pool.shape[2] == used + 8 and loop.free_list.numel() == used + 8
    check_pages(loop)
    for _ in range(9):
        loop.step()
    check_pages(loop)
    assert int(loop.status) == 0
    got = loop.hypotheses()
    assert got[1] == []
    for r in (0, 2):
        same(got[r], search(p[r], 3, 19))
    loop.close()


def test_fewer_tokens_than_beams_leave_rows_without_a_hypothesis(plain, monkeypatch):
    # (the two tokens are the further apart the shorter the text: no two texts are equally likely)
    monkeypatch.setitem(globals(), "logits_of", lambda tokens: torch.where(torch.arange(64) < 2, torch.arange(64.0) * 20 / len(tokens), -math.inf))
    p = prompts(17)
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 1, 5, 20, 40, 17, 8)
    loop.prefill(p)
    for n in (2, 4, 5, 5):
        got = loop.hypotheses()[0]
        assert len(got) == n
        same(got, search(p[0], 5, int(loop.steps))[:n])
        check_pages(loop)
        loop.step()
    loop.close()


@pytest.mark.parametrize("pages,steps", [(5, 0), (6, 1), (7, 1), (9, 14)])
def test_a_step_that_finds_no_page_leaves_the_hypotheses(plain, pages, steps):
    p = prompts(20, 40)                                   # 5 pages, and 4 copies
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 2, 3, pages, 64, 60, 30)
    loop.prefill(p)
    before = None
    for _ in range(25):
        if int(loop.status) != 0:
            break
        before = loop.hypotheses()
        loop.step()
    assert int(loop.status) == B.HS_ERR_OUT_OF_PAGES
    stopped = loop.hypotheses()
    if before is not None:
        assert stopped == before
    else:
        assert stopped == [[], []]
    check_pages(loop)
    for _ in range(2):
        loop.step()
    assert loop.hypotheses() == stopped
    check_pages(loop)
    loop.finish(torch.ones(2, dtype=torch.int32))
    assert int(loop.free_count) == pages
    loop.close()


@pytest.mark.parametrize("kw,word", [(dict(n_beams=0), "n_beams"), (dict(n_beams=33), "n_beams"), (dict(n_requests=0), "n_requests"), (dict(n_requests=513), "n_requests"),
                                     (dict(max_tokens=0), "max_tokens"), (dict(dims=LoopDims(window=5)), "window")])
def test_what_the_operators_do_not_take_is_refused_at_once(plain, kw, word):
    a = dict(dims=DIMS, weights=make_weights(DIMS, device="cpu"), n_requests=2, n_beams=4, num_pages=8, max_positions=16, max_prompt_tokens=8, max_tokens=4)
    with pytest.raises(ValueError, match=word):
        BeamLoop(**dict(a, **kw))


@pytest.mark.parametrize("n_keep", [0, -1, 61])
def test_a_pool_of_no_size_is_refused(plain, n_keep):
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 1, 2, 60, 32, 8, 4)
    with pytest.raises(ValueError, match="n_keep"):
        loop.shrink(n_keep)
    loop.shrink(60)
    assert loop.pool.shape[2] == 60
    loop.close()


@pytest.mark.parametrize("steps", [3, 9])
@pytest.mark.parametrize("penalty", [0.0, 0.9])
def test_a_second_run_begins_like_the_first(plain, steps, penalty):
    """Requests that were ended leave nothing to those that are prefilled behind them, fewer steps than max_tokens or more."""
    first, second = prompts(20, 3), [p[::-1] for p in prompts(35, 18)]
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 2, 3, 60, 64, 60, 8, end_token=7, length_penalty=penalty)
    loop.prefill(first)
    for _ in range(steps):
        loop.step()
    loop.finish(torch.ones(2, dtype=torch.int32))
    assert int(loop.free_count) == 60
    for p in (second, first):
        loop.prefill(p)
        for step in range(1, 9):
            check_pages(loop)
            for r, got in enumerate(loop.hypotheses()):
                same(got, search(p[r], 3, step, 7, penalty))
            loop.step()
        assert int(loop.status) == 0 and int(loop.steps) == 8
        loop.finish(torch.ones(2, dtype=torch.int32))
    loop.close()


def test_a_run_is_not_begun_over_another(plain):
    p = prompts(20, 3)
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 2, 3, 60, 64, 60, 8)
    loop.prefill(p)
    loop.step()
    before = loop.hypotheses()
    for _ in range(2):
        with pytest.raises(RuntimeError, match="finish"):
            loop.prefill(p)
        assert loop.hypotheses() == before
        check_pages(loop)
        loop.finish(torch.tensor([0, 1], dtype=torch.int32))
        before = [before[0], []]
    loop.step()
    same(loop.hypotheses()[0], search(p[0], 3, 3))
    loop.close()


@pytest.mark.parametrize("penalty,tokens", [(40.0, 10), (-40.0, 10), (13.0, 1000), (-13.0, 1000), (math.nan, 4), (math.inf, 1), (-math.inf, 4), (200.0, 1)])
def test_a_length_penalty_whose_weights_leave_fp32_is_refused(plain, penalty, tokens):
    """Weights of 0 would end every beam, and infinite ones too."""
    with pytest.raises(ValueError, match="length_penalty"):
        Loop(DIMS, make_weights(DIMS, device="cpu"), 1, 2, 60, 64, 8, tokens, length_penalty=penalty)


@pytest.mark.parametrize("penalty", [30.0, -30.0])
def test_the_largest_length_penalties(plain, penalty):
    p = prompts(3)
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 1, 3, 60, 64, 8, 15, end_token=7, length_penalty=penalty)
    loop.prefill(p)
    for _ in range(14):
        loop.step()
    assert int(loop.status) == 0 and int(loop.steps) == 15
    same(loop.hypotheses()[0], search(p[0], 3, 15, 7, penalty))
    loop.close()


@pytest.mark.parametrize("keep,entry", [(40, 999), (40, -5), (5, None), (40, "free")])
def test_a_pool_that_cannot_shrink_changes_nothing(plain, monkeypatch, keep, entry):
    """No room, or a block table entry that is no page of the pool or a free one."""
    monkeypatch.setitem(STATUS, "BAD_BLOCK_TABLE", B.HS_ERR_BAD_BLOCK_TABLE)
    p = prompts(20, 3, 40)
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 3, 3, 60, 80, sum(map(len, p)), 30)
    # (pages from the pool's upper end, so that some have to move)
    loop.free_list.copy_(loop.free_list.flip(0))
    loop.prefill(p)
    for _ in range(5):
        loop.step()
    right = int(loop.tables[0, 0])
    if entry is not None:
        loop.tables[0, 0] = int(loop.free_list[:int(loop.free_count)].max()) if entry == "free" else entry
    names = ("ctx_len", "tables", "free_list", "free_count", "shares", "scores", "q_len", "status")
    before, pool, found = {k: getattr(loop, k).clone() for k in names}, loop.pool, loop.hypotheses()
    with pytest.raises(B.HsError):
        loop.shrink(keep)
    assert loop.pool is pool and all(torch.equal(getattr(loop, k), before[k]) for k in names) and loop.hypotheses() == found
    loop.tables[0, 0] = right
    loop.shrink(40)
    check_pages(loop)
    for _ in range(5):
        loop.step()
    for r in range(3):
        same(loop.hypotheses()[r], search(p[r], 3, 11))
    loop.close()


def test_a_run_is_not_begun_under_a_status(plain):
    """A status that a step has left would keep every further one from doing anything."""
    p = prompts(20, 40)
    loop = Loop(DIMS, make_weights(DIMS, device="cpu"), 2, 3, 9, 64, 60, 30)
    loop.prefill(p)
    while int(loop.status) == 0:
        loop.step()
    loop.finish(torch.ones(2, dtype=torch.int32))
    with pytest.raises(B.HsError):
        loop.prefill(p)
    assert int(loop.free_count) == 9 and loop.ctx_len.tolist() == [0] * 6
    loop.status.zero_()
    loop.prefill(p)
    for r, got in enumerate(loop.hypotheses()):
        same(got, search(p[r], 3, 1))
    loop.close()
