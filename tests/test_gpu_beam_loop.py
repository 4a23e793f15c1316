"""Beam search on the device: against a plain 64-bit run of its model, a replayed step against the same calls made one by one, and requests that end, pools that
shrink and pages that run out on the way."""
import math

import pytest
import torch

from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_ops as ops
from paper_2608_01785_b200.device_loop import BeamLoop, LoopDims, make_weights
from tests.test_gpu_device_loop import make, reference

pytestmark = pytest.mark.gpu


def check_pages(loop):
    """Every page is free or held, `shares` counts the holders behind the first, and a last page that is not full has one."""
    num, held, last = loop.shares.numel(), {}, []
    for row, c in zip(loop.tables.tolist(), loop.ctx_len.tolist()):
        for page in row[:-(-c // ops.PAGE)]:
            held[page] = held.get(page, 0) + 1
        if c % ops.PAGE:
            last.append(row[c // ops.PAGE])
    assert sorted(list(held) + loop.free_list[:int(loop.free_count)].tolist()) == list(range(num))
    assert loop.shares.tolist() == [max(held.get(p, 0) - 1, 0) for p in range(num)]
    assert all(held[p] == 1 for p in last)


@pytest.mark.parametrize("beams", [1, 4])
def test_beams_match_the_plain_model(beams):
    dims, w, prompts = make(n=4)
    loop = BeamLoop(dims, w, 4, beams, 80, 160, sum(map(len, prompts)), 8)
    loop.prefill(prompts)
    before = [[(0.0, [])] for _ in prompts]
    for step in range(1, 9):
        assert int(loop.status) == 0
        got = loop.hypotheses()
        for r, p in enumerate(prompts):
            assert len(got[r]) == beams and all(len(t) == step for _, t in got[r])
            rows = [reference(dims, w, p + t)[-1] for _, t in before[r]]
            # A log probability is within a tenth of the logits' spread of the plain one (the operands' roundings: test_loop_matches_the_plain_model of the greedy loop), so a
            # choice is at most twice that behind the one that it was preferred to.
            close = 0.1 * max(float(x.std()) for x in rows)
            lps = [torch.log_softmax(x, -1) for x in rows]
            every = torch.cat([lp + s for lp, (s, _) in zip(lps, before[r])])
            least = float(torch.topk(every, beams).values[-1])
            for s, t in got[r]:
                of = [i for i, (_, u) in enumerate(before[r]) if u == t[:-1]]
                assert len(of) == 1
                plain = before[r][of[0]][0] + float(lps[of[0]][t[-1]])
                assert abs(s - plain) <= close and plain >= least - 2 * close
            assert len({tuple(t) for _, t in got[r]}) == beams and sorted(got[r], key=lambda h: -h[0]) == got[r]
        before = got
        loop.step()
    check_pages(loop)
    loop.close()


def test_replay_is_the_same_as_the_calls():
    dims, w, prompts = make()
    loops = [BeamLoop(dims, w, 5, 3, 90, 160, sum(map(len, prompts)), 30, sm_budget=b) for b in (None, None, 40)]
    for loop in loops:
        loop.prefill(prompts)
    for _ in range(20):
        loops[0].step()
        loops[1]._decode()
        loops[2].step()
    torch.cuda.synchronize()
    for loop in loops:
        assert int(loop.status) == 0
        check_pages(loop)
    used = loops[0].tables[loops[0].tables >= 0].unique().long()
    for other in loops[1:]:
        for name in ("ctx_len", "tables", "free_count", "free_list", "shares", "scores", "done", "length", "past_parent", "past_token", "q_len", "steps"):
            assert torch.equal(getattr(loops[0], name), getattr(other, name)), name
        assert torch.equal(loops[0].last_token[:15], other.last_token[:15])
        for p in used.tolist():
            held = [(i, c) for i, row in enumerate(loops[0].tables.tolist()) for c, q in enumerate(row) if q == p]
            n = min(16, max(int(loops[0].ctx_len[i]) - 16 * c for i, c in held))
            assert torch.equal(loops[0].pool[:, :, p, :, :n], other.pool[:, :, p, :, :n])
    for loop in loops:
        loop.close()


def test_hypotheses_end_and_requests_are_ended_and_the_pool_shrinks():
    dims, w, prompts = make()
    n = sum(map(len, prompts))
    first = BeamLoop(dims, w, 5, 4, 120, 160, n, 12)
    first.prefill(prompts)
    for _ in range(5):
        first.step()
    end = first.hypotheses()[2][0][1][3]                  # a token that is generated
    first.close()
    whole, small = (BeamLoop(dims, w, 5, 4, 120, 160, n, 12, end_token=end, length_penalty=0.7) for _ in range(2))
    gone = torch.tensor([0, 1, 0, 0, 0], dtype=torch.int32, device="cuda")
    for loop in (whole, small):
        loop.prefill(prompts)
        for _ in range(6):
            loop.step()
        loop.finish(gone)
    assert int(small.done.sum()) > 0
    keep = 120 - int(small.free_count) + 25
    small.shrink(keep)
    assert small.pool.shape[2] == keep
    for loop in (whole, small):
        check_pages(loop)
        for _ in range(8):                                # (three steps more than there are tokens: they change nothing)
            loop.step()
        torch.cuda.synchronize()
        assert int(loop.status) == 0 and int(loop.steps) == 12
        check_pages(loop)
    assert whole.hypotheses() == small.hypotheses() and torch.equal(whole.scores, small.scores)
    for r, found in enumerate(whole.hypotheses()):
        assert len(found) == (0 if r == 1 else 4)
        for s, t in found:
            assert math.isfinite(s) and (len(t) == 12 or t[-1] == end) and end not in t[:-1]
    for loop in (whole, small):
        loop.finish(1 - gone)
        assert int(loop.free_count) == loop.shares.numel() and bool((loop.tables == -1).all()) and bool((loop.shares == 0).all())
        loop.close()


@pytest.mark.parametrize("pages", [12, 13, 20, 27])
def test_pages_run_out(pages):
    dims, w, prompts = make()                             # 13 pages, and copies for every beam but the first of four of the requests
    loop = BeamLoop(dims, w, 5, 3, pages, 160, sum(map(len, prompts)), 40)
    loop.prefill(prompts)
    before = loop.hypotheses()
    for _ in range(40):
        loop.step()
        if int(loop.status) != 0:
            break
        before = loop.hypotheses()
    assert int(loop.status) == B.HS_ERR_OUT_OF_PAGES
    assert loop.hypotheses() == before
    check_pages(loop)
    loop.step()
    assert loop.hypotheses() == before
    loop.finish(torch.ones(5, dtype=torch.int32, device="cuda"))
    assert int(loop.free_count) == pages
    loop.close()


def test_more_rows_than_the_head_samples_at_once():
    """40 requests of 8 beams: some against the same search of one request alone."""
    dims = LoopDims(n_layers=1)
    w = make_weights(dims, 3)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, dims.vocab, (int(torch.randint(1, 40, (1,), generator=g)),), generator=g).tolist() for _ in range(40)]
    loop = BeamLoop(dims, w, 40, 8, 900, 64, sum(map(len, prompts)), 6)
    loop.prefill(prompts)
    for _ in range(5):
        loop.step()
    assert int(loop.status) == 0
    check_pages(loop)
    for r in (0, 15, 16, 39):
        for s, t in loop.hypotheses()[r]:
            rows = reference(dims, w, prompts[r] + t[:-1])[-len(t):]
            lp = torch.log_softmax(rows, -1)[torch.arange(len(t)), torch.tensor(t)].sum()
            assert abs(s - float(lp)) <= 0.1 * float(rows.std()) * len(t)
    loop.close()


def test_command_runs(capsys):
    from paper_2608_01785_b200 import device_loop
    device_loop.main(["--requests", "3", "--tokens", "20", "--beams", "4"])
    out = capsys.readouterr().out
    assert "requests of 4 beams" in out and "pages free again" in out


def test_a_second_run_is_that_of_a_new_loop():
    """The captured step goes on with other prompts, behind a run that had come to its last token."""
    dims, w, prompts = make()
    others = [p[::-1] for p in prompts[::-1]]
    used, new = (BeamLoop(dims, w, 5, 3, 90, 160, sum(map(len, prompts)), 10, length_penalty=0.5) for _ in range(2))
    used.prefill(prompts)
    for _ in range(12):
        used.step()
    used.finish(torch.ones(5, dtype=torch.int32, device="cuda"))
    assert int(used.free_count) == 90
    for loop in (used, new):
        loop.prefill(others)
        for _ in range(9):
            loop.step()
        torch.cuda.synchronize()
        assert int(loop.status) == 0 and int(loop.steps) == 10
        check_pages(loop)
    assert used.hypotheses() == new.hypotheses()
    for name in ("ctx_len", "scores", "done", "length", "past_parent", "past_token", "q_len", "steps"):
        assert torch.equal(getattr(used, name), getattr(new, name)), name
    with pytest.raises(RuntimeError, match="finish"):
        used.prefill(others)
    for loop in (used, new):
        loop.close()
