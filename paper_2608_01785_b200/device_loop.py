"""A decoding loop that stays on the device: lengths, page tables, positions, sampled tokens and their log probabilities are device
tensors, and a decode step is one CUDA graph, captured once and replayed while requests grow, end and give their pages back.

The model is a small attention-only decoder (RMSNorm, attention with capped scores, output projection; a final norm and the vocabulary), enough
to run the operators of device_ops.py as they belong together:

    step_tables -> embedding -> [QKV product -> rope_cache -> paged_attention -> output product] per layer -> head -> token_logprobs

    python -m paper_2608_01785_b200.device_loop [--requests N] [--tokens N] [--beams N]

With beams every request keeps its N best continuations (BeamLoop): rows of the block tables that share the pages of what they have in common.
"""
from __future__ import annotations

import argparse
import math
from dataclasses import dataclass
from typing import List, Sequence

import torch

from . import binding as B
from . import device_ops as ops

HEAD_ROWS = 128                       # rows that one hs_head_step samples from
COPIES = 16384                        # pages that one copy_pages moves: any number of layers and heads fits


@dataclass(frozen=True)
class LoopDims:
    n_layers: int = 2
    d_model: int = 1024
    n_q_heads: int = 16
    n_kv_heads: int = 4
    head_dim: int = 64
    vocab: int = 4096
    rms_eps: float = 1e-6
    rope_base: float = 10000.0
    cap: float = 30.0                 # of the attention's scores
    window: int = 0                   # sliding window in keys, 0: none


def make_weights(dims: LoopDims, seed: int = 0, device="cuda"):
    """bf16 weights ~ N(0, 0.02), embeddings ~ N(0, 1); drawn on the CPU, so that every device has the same."""
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=0.02):
        return (std * torch.randn(*shape, generator=g)).to(torch.bfloat16).to(device)

    q, kv = dims.n_q_heads * dims.head_dim, dims.n_kv_heads * dims.head_dim
    return {"embed": normal(dims.vocab, dims.d_model, std=1.0), "g_final": torch.ones(dims.d_model, dtype=torch.bfloat16, device=device),
            "w_vocab": normal(dims.vocab, dims.d_model),
            "layers": [{"w_qkv": normal(q + 2 * kv, dims.d_model), "w_o": normal(dims.d_model, q)} for _ in range(dims.n_layers)]}


class DeviceLoop:
    """Requests decoded greedily under a KV pool of num_pages pages.  All state is on the device; `last_token`, `logprob` and `top_ids` hold what the last
    step sampled, request by request."""

    def __init__(self, dims: LoopDims, weights, n_requests: int, num_pages: int, max_positions: int, max_prompt_tokens: int, n_top: int = 5, sm_budget=None):
        if not 1 <= n_requests <= ops.MAX_SEQS:
            raise ValueError(f"n_requests: 1 .. {ops.MAX_SEQS} are possible")
        self.dims, self.w, self.n, self.budget = dims, weights, n_requests, sm_budget
        d = self.device = weights["embed"].device
        i32 = lambda *s, fill=0: torch.full(s, fill, dtype=torch.int32, device=d)  # noqa: E731
        self.ctx_len, self.q_len = i32(n_requests), i32(n_requests, fill=1)
        self.tables = i32(n_requests, -(-max_positions // ops.PAGE), fill=-1)
        self.free_list = torch.arange(num_pages - 1, -1, -1, dtype=torch.int32, device=d)
        self.free_count, self.status = i32(1, fill=num_pages), i32(1)
        self.workspace = ops.workspace(d)
        self.pool = torch.zeros(dims.n_layers, 2, num_pages, dims.n_kv_heads, ops.PAGE, dims.head_dim, dtype=torch.bfloat16, device=d)
        self.rope = torch.empty(max_positions, dims.head_dim // 2, 2, device=d)
        ops.rope_table(self.rope, dims.rope_base, sm_budget=sm_budget)
        # (one entry more, for the rows that pad a step)
        self.last_token, self.logprob = i32(n_requests + 1), torch.zeros(n_requests + 1, device=d)
        self.top_ids = i32(n_requests + 1, n_top)
        cfg = B.make_head_config(dims.d_model, dims.vocab, dims.rms_eps, min(n_requests, HEAD_ROWS), d.index or 0)
        self._head_ws = torch.zeros(B.hs_head_workspace_bytes(cfg) + 256, dtype=torch.uint8, device=d)
        at = (self._head_ws.data_ptr() + 255) // 256 * 256
        self.head = B.hs_head_create(cfg, weights["g_final"].data_ptr(), weights["w_vocab"].data_ptr(), at)
        self._decode_buffers, self._prompt_buffers = self._buffers(n_requests), self._buffers(max_prompt_tokens)
        self.graph = None

    def close(self) -> None:
        if self.head:
            self.graph = None
            B.hs_head_destroy(self.head)
            self.head = None

    def _buffers(self, tokens: int):
        d, q, kv = self.dims, self.dims.n_q_heads * self.dims.head_dim, self.dims.n_kv_heads * self.dims.head_dim
        dev, bf = self.device, torch.bfloat16
        i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=dev)  # noqa: E731
        return {"begin": i32(self.n + 1), "seq": i32(tokens), "pos": i32(tokens), "slot": i32(tokens), "kv_len": i32(self.n), "tokens": i32(tokens),
                "embedded": torch.zeros(tokens, d.d_model, dtype=bf, device=dev), "x": torch.zeros(tokens, d.d_model, device=dev),
                "qkv": torch.zeros(tokens, q + 2 * kv, device=dev), "q": torch.zeros(tokens, d.n_q_heads, d.head_dim, dtype=bf, device=dev),
                "o": torch.zeros(tokens, d.n_q_heads, d.head_dim, dtype=bf, device=dev), "rows": torch.arange(self.n, dtype=torch.int32, device=dev),
                "logits": torch.zeros(self.n, d.vocab, device=dev), "sampled": i32(self.n), "logprob": torch.zeros(self.n, device=dev),
                "top_ids": torch.zeros(self.n, self.top_ids.shape[1], dtype=torch.int32, device=dev),
                "top_logprobs": torch.zeros(self.n, self.top_ids.shape[1], device=dev)}

    def _stream(self) -> int:
        return torch.cuda.current_stream(self.device).cuda_stream

    def _budget(self) -> int:
        return self.budget or ops.sm_count(self.device.index or 0)

    def _layers(self, b, max_q_len: int) -> None:
        """b["tokens"] at b["pos"] through the layers; b["x"] is the residual stream."""
        d, t, budget = self.dims, b["tokens"].numel(), self._budget()
        hq, hkv, dh = d.n_q_heads, d.n_kv_heads, d.head_dim
        B.hs_op_embed(b["tokens"].data_ptr(), t, self.w["embed"].data_ptr(), d.vocab, d.d_model, b["embedded"].data_ptr(), budget, self.status.data_ptr(), self._stream())
        b["x"].copy_(b["embedded"])
        q, k, v = b["qkv"][:, :hq * dh], b["qkv"][:, hq * dh:(hq + hkv) * dh], b["qkv"][:, (hq + hkv) * dh:]
        for l, w in enumerate(self.w["layers"]):
            x = b["x"]
            h = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + d.rms_eps)).to(torch.bfloat16)
            B.hs_op_gemm_bf16(h.data_ptr(), w["w_qkv"].data_ptr(), 0, b["qkv"].data_ptr(), t, b["qkv"].shape[1], d.d_model, budget, self.status.data_ptr(), self._stream())
            ops.rope_cache(q.unflatten(1, (hq, dh)), k.unflatten(1, (hkv, dh)), v.unflatten(1, (hkv, dh)), b["pos"], b["slot"], self.rope, b["q"], self.pool, l,
                           self.status, sm_budget=self.budget)
            self._attend(b, l, max_q_len)
            B.hs_op_gemm_bf16(b["o"].data_ptr(), w["w_o"].data_ptr(), x.data_ptr(), x.data_ptr(), t, d.d_model, hq * dh, budget, self.status.data_ptr(), self._stream())

    def _attend(self, b, layer: int, max_q_len: int) -> None:
        ops.paged_attention(b["q"], self.pool, layer, self.tables, b["kv_len"], b["o"], self.workspace, self.status, tok_begin=b["begin"], max_q_len=max_q_len,
                            cap=self.dims.cap, window=self.dims.window, sm_budget=self.budget)

    def _head(self, b, n: int) -> None:
        """Logits and greedy tokens of the first n rows that b["rows"] names."""
        for i in range(0, n, HEAD_ROWS):
            B.hs_head_step(self.head, b["x"].data_ptr(), b["rows"][i:].data_ptr(), min(HEAD_ROWS, n - i), b["logits"][i:].data_ptr(), b["sampled"][i:].data_ptr(),
                           self._budget(), self._stream())

    def _sample(self, b, owner) -> None:
        """Greedy tokens of the rows b["rows"] of the residual stream, their log probabilities and alternatives, to the requests `owner`."""
        self._head(b, self.n)
        ops.token_logprobs(b["logits"], b["sampled"], b["logprob"], self.workspace, self.status, top_ids=b["top_ids"], top_logprobs=b["top_logprobs"],
                           sm_budget=self.budget)
        self.last_token.index_copy_(0, owner, b["sampled"])
        self.logprob.index_copy_(0, owner, b["logprob"])
        self.top_ids.index_copy_(0, owner, b["top_ids"])

    def prefill(self, prompts: Sequence[Sequence[int]]) -> None:
        """Runs all prompts as one chunk (at most max_prompt_tokens tokens) and samples each request's first token.  Prompts that do not fit the pool or the block
        tables leave a status and the requests as they were."""
        b, lens = self._prompt_buffers, [len(p) for p in prompts]
        assert len(lens) == self.n and min(lens) >= 1 and sum(lens) <= b["tokens"].numel()
        ops.step_tables(self.ctx_len, torch.tensor(lens, dtype=torch.int32, device=self.device), self.free_list, self.free_count, self.tables, b["kv_len"], b["begin"],
                        b["seq"], b["pos"], b["slot"], self.free_count, self.workspace, self.status, sm_budget=self.budget)
        flat = [t for p in prompts for t in p]
        b["tokens"].zero_()
        b["tokens"][:len(flat)] = torch.tensor(flat, dtype=torch.int32, device=self.device)
        self._layers(b, max(max(lens), 2))
        # (a request without rows -- every one of them, where the tables were refused -- has no last row: row 0 stands for it, and what that gives goes to the
        # spare entry)
        first, last = b["begin"][:-1], b["begin"][1:]
        b["rows"].copy_((last - 1).clamp(min=0))
        self._sample(b, torch.where(last > first, torch.arange(self.n, device=self.device), self.n))
        self.ctx_len.copy_(b["kv_len"])

    def _decode(self) -> None:
        b = self._decode_buffers
        ops.step_tables(self.ctx_len, self.q_len, self.free_list, self.free_count, self.tables, b["kv_len"], b["begin"], b["seq"], b["pos"], b["slot"],
                        self.free_count, self.workspace, self.status, sm_budget=self.budget)
        owner = torch.where(b["seq"] < 0, torch.full_like(b["seq"], self.n), b["seq"]).long()
        b["tokens"].copy_(self.last_token[owner])
        self._layers(b, 1)
        self._sample(b, owner)
        self.ctx_len.copy_(b["kv_len"])

    def _state(self):
        """What a step changes."""
        return self.ctx_len, self.tables, self.free_count, self.last_token, self.logprob, self.top_ids

    def step(self) -> None:
        """One token for every request whose q_len is 1, as a replay of the captured step (the first call captures it)."""
        if self.graph is None:
            # the first run of everything outside a capture, on state that is put back
            kept = [t.clone() for t in self._state()]
            side = torch.cuda.Stream(self.device)
            side.wait_stream(torch.cuda.current_stream(self.device))
            with torch.cuda.stream(side):
                self._decode()
            torch.cuda.current_stream(self.device).wait_stream(side)
            for t, k in zip(self._state(), kept):
                t.copy_(k)
            torch.cuda.synchronize(self.device)
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self._decode()
        self.graph.replay()

    def finish(self, done: torch.Tensor) -> None:
        """Ends the requests with done != 0 (int32 [n_requests], on the device): their pages go back, and they take no further part."""
        ops.release_pages(done, self.ctx_len, self.tables, self.free_list, self.free_count, self.workspace, self.status, sm_budget=self.budget)
        self.q_len.mul_((done == 0).to(torch.int32))


class BeamLoop(DeviceLoop):
    """Beam search: every request has the n_beams continuations with the largest log probability, each a row of the block tables (request r: rows r n_beams ..).
    Rows hold the pages of what they have in common together; a step is

        step_tables -> layers with shared_attention -> head -> beam_select -> fork_pages -> copy_pages

    `scores` [n_requests, n_beams] are the hypotheses' log probabilities, best first, `done` marks those that end in end_token; hypotheses() gives their tokens.  With a
    length_penalty they are ranked by the log probability divided by their number of tokens to that power.  A step that cannot be done leaves a status and the hypotheses as
    they were, and further steps change nothing; neither do steps behind max_tokens tokens."""

    def __init__(self, dims: LoopDims, weights, n_requests: int, n_beams: int, num_pages: int, max_positions: int, max_prompt_tokens: int, max_tokens: int,
                 end_token: int = -1, length_penalty: float = 0.0, sm_budget=None):
        if not 1 <= n_beams <= ops.MAX_BEAMS:
            raise ValueError(f"n_beams: 1 .. {ops.MAX_BEAMS} are possible")
        if not 1 <= n_requests * n_beams <= ops.MAX_SHARED_SEQS:
            raise ValueError(f"n_requests: 1 .. {ops.MAX_SHARED_SEQS} rows of all beams are possible")
        if max_tokens < 1:
            raise ValueError("max_tokens: at least 1")
        if not (math.isfinite(length_penalty) and abs(length_penalty) * math.log(max_tokens + 1) <= 87.0):     # (fp32 holds e^-87 .. e^87; steps behind max_tokens rank, too)
            raise ValueError("length_penalty: max_tokens + 1 to that power, and its inverse, have to be fp32 numbers")
        if dims.window != 0:
            raise ValueError("window: beams attend to all keys")
        super().__init__(dims, weights, n_requests * n_beams, num_pages, max_positions, max_prompt_tokens, n_top=1, sm_budget=sm_budget)
        self.n_requests, self.n_beams, self.max_tokens, self.end_token, self.length_penalty = n_requests, n_beams, max_tokens, end_token, length_penalty
        d, n = self.device, self.n
        i32 = lambda *s, fill=0: torch.full(s, fill, dtype=torch.int32, device=d)  # noqa: E731
        self.q_len.zero_()
        self.shares, self.shared_len = i32(num_pages), i32(n_requests)
        self.group_begin = torch.arange(0, n + 1, n_beams, dtype=torch.int32, device=d)
        self.scores, self.done = torch.full((n_requests, n_beams), -math.inf, device=d), i32(n_requests, n_beams)
        self.length = i32(n)                              # tokens that a row's hypothesis has behind its prompt
        self.out_score, self.out_done = torch.empty_like(self.scores), i32(n_requests, n_beams)
        self.out_parent, self.out_token = i32(n_requests, n_beams), i32(n_requests, n_beams)
        self.copy_src, self.copy_dst, self.copy_len = i32(n), i32(n), i32(n)
        # parents and tokens step by step
        self.steps = torch.zeros(1, dtype=torch.int64, device=d)
        self.past_parent, self.past_token = i32(max_tokens, n, fill=-1), i32(max_tokens, n, fill=-1)
        self._itself = torch.arange(n, dtype=torch.int32, device=d)

    def _state(self):
        return (self.ctx_len, self.tables, self.free_list, self.free_count, self.shares, self.q_len, self.scores, self.done, self.length, self.last_token, self.steps,
                self.past_parent, self.past_token)

    def _attend(self, b, layer: int, max_q_len: int) -> None:
        if max_q_len > 1:
            return super()._attend(b, layer, max_q_len)
        ops.shared_attention(b["q"], self.pool, layer, self.tables, b["kv_len"], self.group_begin, self.shared_len, b["o"], self.workspace, self.status,
                             cap=self.dims.cap, sm_budget=self.budget)

    def _fork(self, parent) -> None:
        ops.fork_pages(parent, self.ctx_len, self.tables, self.shares, self.free_list, self.free_count, self.copy_src, self.copy_dst, self.copy_len, self.workspace,
                       self.status, sm_budget=self.budget)
        ops.copy_pages(self.pool, self.copy_src, self.copy_dst, self.status, length=self.copy_len, sm_budget=self.budget)

    def _select(self, logits, scores, done, first_row) -> None:
        """The best continuations of rows of logits, n_beams of each request; rows i of the tables continue first_row times the parents."""
        weight = None
        if self.length_penalty != 0 and done is not None:
            weight = (self.length.view_as(done) + 1 - done).float().pow(-self.length_penalty)
        ops.beam_select(logits, scores, self.out_score, self.out_parent, self.out_token, self.workspace, self.status, done=done, weight=weight, out_done=self.out_done,
                        end_token=self.end_token, sm_budget=self.budget)
        parent = torch.where(self.out_parent < 0, -1, self.out_parent * first_row).flatten()
        more = self.steps < self.max_tokens
        self._fork(torch.where((self.status == 0) & more, parent, self._itself))
        ok = (self.status == 0) & more
        of = parent.clamp(min=0).long()
        was_done = torch.zeros_like(parent) if done is None else self.done.flatten()[of]
        at = self.steps.clamp(max=self.max_tokens - 1)
        self.past_parent.index_copy_(0, at, torch.where(ok, parent, self.past_parent[at]))
        self.past_token.index_copy_(0, at, torch.where(ok, self.out_token.flatten(), self.past_token[at]))
        self.length.copy_(torch.where(ok, self.length[of] + 1 - was_done, self.length))
        self.last_token[:self.n].copy_(torch.where(ok, self.out_token.flatten().clamp(min=0), self.last_token[:self.n]))
        self.scores.copy_(torch.where(ok, self.out_score, self.scores))
        self.done.copy_(torch.where(ok, self.out_done, self.done))
        self.steps.add_(ok)
        self.q_len.copy_(ok & (self.steps < self.max_tokens) & (self.ctx_len > 0) & (self.done.flatten() == 0))

    def prefill(self, prompts: Sequence[Sequence[int]]) -> None:
        """Begins a run: all prompts as one chunk, each in the first row of its request, then the beams with its n_beams most likely tokens.  Prompts that do not fit leave a
        status and no beams.  What a run before has left is forgotten; all of its requests have to be finished, and its status, if it left one, put
        back to 0."""
        b, lens, n = self._prompt_buffers, [len(p) for p in prompts], self.n_requests
        assert len(lens) == n and min(lens) >= 1 and sum(lens) <= b["tokens"].numel()
        if bool((self.ctx_len != 0).any()):
            raise RuntimeError("requests of a run before still hold tokens: finish them first")
        if int(self.status) != 0:
            raise B.HsError(int(self.status), "a run before")
        for t in (self.steps, self.length, self.done, self.q_len):
            t.zero_()
        self.scores.fill_(-math.inf)
        for t in (self.past_parent, self.past_token):
            t.fill_(-1)
        lengths = torch.tensor(lens, dtype=torch.int32, device=self.device)
        q_len = torch.zeros_like(self.q_len)
        q_len[::self.n_beams] = lengths
        ops.step_tables(self.ctx_len, q_len, self.free_list, self.free_count, self.tables, b["kv_len"], b["begin"], b["seq"], b["pos"], b["slot"], self.free_count,
                        self.workspace, self.status, sm_budget=self.budget)
        flat = [t for p in prompts for t in p]
        b["tokens"].zero_()
        b["tokens"][:len(flat)] = torch.tensor(flat, dtype=torch.int32, device=self.device)
        self._layers(b, max(max(lens), 2))
        self.ctx_len.copy_(b["kv_len"])
        self.shared_len.copy_(lengths)
        b["rows"][:n].copy_((b["begin"][1::self.n_beams] - 1).clamp(min=0))
        self._head(b, n)
        self._select(b["logits"][:n], torch.zeros(n, 1, device=self.device), None, self.n_beams)

    def _decode(self) -> None:
        b = self._decode_buffers
        ops.step_tables(self.ctx_len, self.q_len, self.free_list, self.free_count, self.tables, b["kv_len"], b["begin"], b["seq"], b["pos"], b["slot"],
                        self.free_count, self.workspace, self.status, sm_budget=self.budget)
        self.ctx_len.copy_(b["kv_len"])
        # Rows of a step are those that go on, one behind the other; here every row keeps its place, and those that do not go on have no keys and store none.
        first, on = b["begin"][:-1].clamp(max=self.n - 1).long(), b["begin"][1:] > b["begin"][:-1]
        b["pos"].copy_(torch.where(on, b["pos"][first], 0))
        b["slot"].copy_(torch.where(on, b["slot"][first], -1))
        b["kv_len"].mul_(on)
        b["tokens"].copy_(self.last_token[:self.n])
        self._layers(b, 1)
        self._head(b, self.n)
        self._select(b["logits"], self.scores, self.done, 1)

    def finish(self, done: torch.Tensor) -> None:
        """Ends the requests with done != 0 (int32 [n_requests], on the device): their rows' pages go back, and they take no further part."""
        over = (done != 0).repeat_interleave(self.n_beams)
        self._fork(torch.where(over, -1, self._itself))
        self.q_len.mul_(~over)
        self.scores.masked_fill_((done != 0)[:, None], -math.inf)

    def shrink(self, n_keep: int) -> None:
        """Makes the pool n_keep pages large: pages behind move below, and the memory of the rest is given back.  Raises HsError, and changes nothing, where there is no
        room or a block table names a page that is not a row's to have.  The next step is captured anew.  Both pools exist until the smaller one is filled: a layer's pages follow
        one another, so that the upper end is no end of the memory."""
        num_pages = self.shares.numel()
        if not 1 <= n_keep <= num_pages:
            raise ValueError(f"n_keep: 1 .. {num_pages} are possible")
        if n_keep == num_pages:
            return
        src, dst = (torch.empty(num_pages - n_keep, dtype=torch.int32, device=self.device) for _ in range(2))
        status, (tables, shares, free_list) = torch.zeros_like(self.status), (t.clone() for t in (self.tables, self.shares, self.free_list))
        ops.compact_pages(n_keep, self.ctx_len, tables, shares, free_list, self.free_count, src, dst, self.workspace, status, sm_budget=self.budget)
        if int(status) != 0:
            raise B.HsError(int(status), "compact_pages")
        pool = self.pool.new_empty(*self.pool.shape[:2], n_keep, *self.pool.shape[3:])
        for i in range(0, num_pages - n_keep, COPIES):    # (to pages that are free: nothing has changed until the tables do)
            ops.copy_pages(self.pool, src[i:i + COPIES], dst[i:i + COPIES], status, sm_budget=self.budget)
        pool.copy_(self.pool[:, :, :n_keep])
        self.graph = None
        self.pool, self.shares, self.free_list = pool, shares[:n_keep].clone(), free_list[num_pages - n_keep:].clone()
        self.tables.copy_(tables)
        self.free_count.sub_(num_pages - n_keep)

    def hypotheses(self):
        """For every request its hypotheses, best first, as (log probability, tokens behind the prompt); requests that were ended have none."""
        steps, scores = int(self.steps), self.scores.flatten().tolist()
        parent, token = self.past_parent[:steps].tolist(), self.past_token[:steps].tolist()
        found = []
        for r in range(self.n_requests):
            found.append([])
            for row in range(r * self.n_beams, (r + 1) * self.n_beams):
                if scores[row] == -math.inf:
                    continue
                tokens, i = [], row
                for t in range(steps - 1, -1, -1):
                    tokens.append(token[t][i])
                    i = parent[t][i]
                tokens.reverse()
                if self.end_token in tokens:
                    tokens = tokens[:tokens.index(self.end_token) + 1]
                found[-1].append((scores[row], tokens))
        return found


def main(argv: List[str] = None) -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--beams", type=int, default=0, help="hypotheses of a request; 0: greedy tokens")
    a = ap.parse_args(argv)
    dims = LoopDims()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, dims.vocab, (int(torch.randint(16, 200, (1,), generator=g)),), generator=g).tolist() for _ in range(a.requests)]
    most = max(len(p) for p in prompts) + a.tokens
    pages = sum(-(-(len(p) + a.tokens) // ops.PAGE) for p in prompts) + 1
    if a.beams:                                            # (a beam has pages of its own at most for what it has generated, and a copy while its parent is still there)
        pages += a.requests * a.beams * (-(-a.tokens // ops.PAGE) + 2)
        loop = BeamLoop(dims, make_weights(dims), a.requests, a.beams, pages, most, sum(len(p) for p in prompts), a.tokens)
    else:
        loop = DeviceLoop(dims, make_weights(dims), a.requests, pages, most, sum(len(p) for p in prompts))
    loop.prefill(prompts)
    loop.step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.tokens - 2):
        loop.step()
    end.record()
    torch.cuda.synchronize()
    if int(loop.status) != 0:
        raise SystemExit(f"status {B.status_str(int(loop.status))}")
    us = begin.elapsed_time(end) * 1000 / max(a.tokens - 2, 1)
    if a.beams:
        score, tokens = loop.hypotheses()[0][0]
        print(f"{a.requests} requests of {a.beams} beams, {dims.n_layers} layers: {us:.1f} us a step; request 0: log probability {score:.3f}, tokens {tokens[:8]} ...")
    else:
        print(f"{a.requests} requests, {dims.n_layers} layers: {us:.1f} us a step, {a.requests / us * 1e6:.0f} tokens/s; request 0: token {int(loop.last_token[0])}, "
              f"log probability {float(loop.logprob[0]):.3f}, alternatives {loop.top_ids[0].tolist()}")
    loop.finish(torch.ones(a.requests, dtype=torch.int32, device=loop.device))
    print(f"{int(loop.free_count)} of {loop.pool.shape[2]} pages free again")
    loop.close()


if __name__ == "__main__":
    main()
