"""The device-resident decoding loop: against a plain 64-bit run of its model, a replayed step against the same calls made one by one, and requests
that end while others go on."""
import math

import pytest
import torch

from paper_2608_01785_b200 import device_ops as ops
from paper_2608_01785_b200.device_loop import DeviceLoop, LoopDims, make_weights

pytestmark = pytest.mark.gpu


def reference(dims, w, tokens):
    """fp64 logits of every position of one request (bf16 where the loop stores bf16: the attention's operands)."""
    n, hq, hkv, dh = len(tokens), dims.n_q_heads, dims.n_kv_heads, dims.head_dim
    x = w["embed"].cpu().double()[tokens]
    pos = torch.arange(n, dtype=torch.float64)[:, None]
    angle = pos * dims.rope_base ** (-2.0 * torch.arange(dh // 2, dtype=torch.float64) / dh)[None]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turn(y):
        a, b = y[..., : dh // 2], y[..., dh // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

    for l in w["layers"]:
        h = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + dims.rms_eps)
        qkv = h @ l["w_qkv"].cpu().double().T
        q, k, v = qkv[:, :hq * dh].view(n, hq, dh), qkv[:, hq * dh:(hq + hkv) * dh].view(n, hkv, dh), qkv[:, (hq + hkv) * dh:].view(n, hkv, dh)
        q, k = turn(q), turn(k).repeat_interleave(hq // hkv, 1)
        s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(dh)
        s = dims.cap * torch.tanh(s / dims.cap)
        far = torch.arange(n)[:, None] - torch.arange(n)[None]
        seen = (far >= 0) & ((far < dims.window) if dims.window else True)
        s = s.masked_fill(~seen[None], -math.inf)
        o = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v.repeat_interleave(hq // hkv, 1))
        x = x + o.reshape(n, hq * dh) @ l["w_o"].cpu().double().T
    h = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + dims.rms_eps)
    return h @ w["w_vocab"].cpu().double().T


def make(window=0, n=5, seed=0):
    dims = LoopDims(window=window)
    w = make_weights(dims, seed)
    g = torch.Generator().manual_seed(seed + 1)
    prompts = [torch.randint(0, dims.vocab, (k,), generator=g).tolist() for k in (1, 16, 17, 40, 90)[:n]]
    return dims, w, prompts


@pytest.mark.parametrize("window", [0, 20])
def test_loop_matches_the_plain_model(window):
    dims, w, prompts = make(window)
    loop = DeviceLoop(dims, w, 5, 40, 160, sum(map(len, prompts)))
    loop.prefill(prompts)
    seqs = [list(p) for p in prompts]
    for step in range(6):
        torch.cuda.synchronize()
        assert int(loop.status) == 0
        for s in range(5):
            logits = reference(dims, w, seqs[s])[-1]
            lp = torch.log_softmax(logits, -1)
            token = int(loop.last_token[s])
            # The operands of two layers' products, q, K, V, P and the head's input are rounded to bf16: about ten roundings of at most 2^-8 each, spread
            # over sums of terms of either sign, so some 1 % of the logits' spread; a tenth of it (twice that between two tokens) leaves room for the largest of many.
            spread = float(logits.std())
            assert abs(float(loop.logprob[s]) - float(lp[token])) <= 0.1 * spread
            assert float(logits[token]) >= float(logits.max()) - 0.15 * spread
            assert int(loop.top_ids[s, 0]) == token
            seqs[s].append(token)
        loop.step()
    assert loop.ctx_len.tolist() == [len(p) + 6 for p in prompts]
    loop.close()


def test_replay_is_the_same_as_the_calls():
    dims, w, prompts = make()
    loops = [DeviceLoop(dims, w, 5, 40, 160, sum(map(len, prompts)), sm_budget=b) for b in (None, None, 40)]
    for loop in loops:
        loop.prefill(prompts)
    for _ in range(5):
        loops[0].step()
        loops[1]._decode()
        loops[2].step()
    torch.cuda.synchronize()
    for other in loops[1:]:
        for name in ("ctx_len", "tables", "free_count", "last_token", "logprob", "top_ids", "pool"):
            assert torch.equal(getattr(loops[0], name), getattr(other, name)), name
    for loop in loops:
        assert int(loop.status) == 0
        loop.close()


def test_requests_end_while_others_go_on():
    dims, w, prompts = make()
    alone, loop = DeviceLoop(dims, w, 5, 40, 160, 164), DeviceLoop(dims, w, 5, 40, 160, 164)
    for l in (alone, loop):
        l.prefill(prompts)
        for _ in range(3):
            l.step()
    done = torch.tensor([0, 1, 0, 1, 0], dtype=torch.int32, device="cuda")
    kept = loop.last_token.clone()
    loop.finish(done)
    for _ in range(4):
        alone.step()
        loop.step()
    torch.cuda.synchronize()
    assert int(loop.status) == 0
    for s in range(5):
        if done[s]:
            assert int(loop.ctx_len[s]) == 0 and int(loop.last_token[s]) == int(kept[s]) and bool((loop.tables[s] == -1).all())
        else:
            # the others' rows have moved up and the work is shared out differently: rounding apart
            assert int(loop.ctx_len[s]) == int(alone.ctx_len[s]) and abs(float(loop.logprob[s]) - float(alone.logprob[s])) <= 0.2
    pages = sum(-(-int(c) // ops.PAGE) for c in loop.ctx_len.tolist())
    assert int(loop.free_count) == 40 - pages
    owned = loop.tables[loop.tables >= 0]
    free = loop.free_list[: int(loop.free_count)]
    assert sorted(owned.tolist() + free.tolist()) == list(range(40))
    alone.close()
    loop.close()


def test_a_loop_without_pages_says_so():
    dims, w, prompts = make()
    loop = DeviceLoop(dims, w, 5, 13, 160, 164)           # 1 + 1 + 2 + 3 + 6 pages for the prompts, none to grow
    loop.prefill(prompts)
    before = [t.clone() for t in (loop.ctx_len, loop.tables, loop.free_count)]
    for _ in range(2):
        loop.step()                                       # the first step fits no page for the requests of 16 tokens
    torch.cuda.synchronize()
    from paper_2608_01785_b200 import binding as B
    assert int(loop.status) == B.HS_ERR_OUT_OF_PAGES
    for t, k in zip((loop.ctx_len, loop.tables, loop.free_count), before):
        assert torch.equal(t, k)
    loop.close()


def test_example_runs(capsys):
    from paper_2608_01785_b200 import device_loop
    device_loop.main(["--requests", "3", "--tokens", "8"])
    assert "pages free again" in capsys.readouterr().out


@pytest.mark.parametrize("pages,positions,status", [(12, 160, "OUT_OF_PAGES"), (40, 80, "INVALID_ARG")])
def test_prompts_that_do_not_fit_leave_the_requests_as_they_were(pages, positions, status):
    from paper_2608_01785_b200 import binding as B
    dims, w, prompts = make()                              # 13 pages, the longest 90 tokens
    loop = DeviceLoop(dims, w, 5, pages, positions, sum(map(len, prompts)))
    loop.last_token[:5] = torch.arange(5, dtype=torch.int32, device="cuda")
    names = ("ctx_len", "tables", "free_count", "free_list", "pool")
    before = {k: getattr(loop, k).clone() for k in names}
    loop.prefill(prompts)
    torch.cuda.synchronize()
    assert int(loop.status) == getattr(B, "HS_ERR_" + status)
    for k in names:
        assert torch.equal(getattr(loop, k), before[k]), k
    assert loop.last_token[:5].tolist() == [0, 1, 2, 3, 4] and loop.logprob[:5].tolist() == [0] * 5 and bool((loop.top_ids[:5] == 0).all())
    loop.close()


def test_more_requests_than_the_head_samples_at_once():
    """300 requests, three slices of the head's rows: some of each against the plain model, with the tolerances of test_loop_matches_the_plain_model."""
    dims = LoopDims(n_layers=1)
    w = make_weights(dims, 3)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, dims.vocab, (int(torch.randint(1, 30, (1,), generator=g)),), generator=g).tolist() for _ in range(300)]
    loop = DeviceLoop(dims, w, 300, 900, 64, sum(map(len, prompts)))
    loop.prefill(prompts)
    some = (0, 1, 127, 128, 129, 255, 256, 299)
    seqs = {s: list(prompts[s]) for s in some}
    for _ in range(3):
        torch.cuda.synchronize()
        assert int(loop.status) == 0
        for s in some:
            logits, token = reference(dims, w, seqs[s])[-1], int(loop.last_token[s])
            spread = float(logits.std())
            assert abs(float(loop.logprob[s]) - float(torch.log_softmax(logits, -1)[token])) <= 0.1 * spread
            assert float(logits[token]) >= float(logits.max()) - 0.15 * spread and int(loop.top_ids[s, 0]) == token
            seqs[s].append(token)
        loop.step()
    assert loop.ctx_len.tolist() == [len(p) + 3 for p in prompts]
    loop.close()
