"""A decoding loop that stays on the device: lengths, page tables, positions, sampled tokens and their log probabilities are device
tensors, and a decode step is one CUDA graph, captured once and replayed while requests grow, end and give their pages back.

The model is a small attention-only decoder (RMSNorm, attention with capped scores, output projection; a final norm and the vocabulary), enough
to run the operators of device_ops.py as they belong together:

    step_tables -> embedding -> [QKV product -> rope_cache -> paged_attention -> output product] per layer -> head -> token_logprobs

    python -m paper_2608_01785_b200.device_loop [--requests N] [--tokens N]
"""
from __future__ import annotations

import argparse
from dataclasses import dataclass
from typing import List, Sequence

import torch

from . import binding as B
from . import device_ops as ops

HEAD_ROWS = 128                       # rows that one hs_head_step samples from


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
            ops.paged_attention(b["q"], self.pool, l, self.tables, b["kv_len"], b["o"], self.workspace, self.status, tok_begin=b["begin"], max_q_len=max_q_len,
                                cap=d.cap, window=d.window, sm_budget=self.budget)
            B.hs_op_gemm_bf16(b["o"].data_ptr(), w["w_o"].data_ptr(), x.data_ptr(), x.data_ptr(), t, d.d_model, hq * dh, budget, self.status.data_ptr(), self._stream())

    def _sample(self, b, owner) -> None:
        """Greedy tokens of the rows b["rows"] of the residual stream, their log probabilities and alternatives, to the requests `owner`."""
        for i in range(0, self.n, HEAD_ROWS):
            B.hs_head_step(self.head, b["x"].data_ptr(), b["rows"][i:].data_ptr(), min(HEAD_ROWS, self.n - i), b["logits"][i:].data_ptr(), b["sampled"][i:].data_ptr(),
                           self._budget(), self._stream())
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

    def step(self) -> None:
        """One token for every request whose q_len is 1, as a replay of the captured step (the first call captures it)."""
        if self.graph is None:
            # the first run of everything outside a capture, on state that is put back
            kept = [t.clone() for t in (self.ctx_len, self.tables, self.free_count, self.last_token, self.logprob, self.top_ids)]
            side = torch.cuda.Stream(self.device)
            side.wait_stream(torch.cuda.current_stream(self.device))
            with torch.cuda.stream(side):
                self._decode()
            torch.cuda.current_stream(self.device).wait_stream(side)
            for t, k in zip((self.ctx_len, self.tables, self.free_count, self.last_token, self.logprob, self.top_ids), kept):
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


def main(argv: List[str] = None) -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--tokens", type=int, default=64)
    a = ap.parse_args(argv)
    dims = LoopDims()
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, dims.vocab, (int(torch.randint(16, 200, (1,), generator=g)),), generator=g).tolist() for _ in range(a.requests)]
    most = max(len(p) for p in prompts) + a.tokens
    loop = DeviceLoop(dims, make_weights(dims), a.requests, sum(-(-(len(p) + a.tokens) // ops.PAGE) for p in prompts) + 1, most, sum(len(p) for p in prompts))
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
    print(f"{a.requests} requests, {dims.n_layers} layers: {us:.1f} us a step, {a.requests / us * 1e6:.0f} tokens/s; request 0: token {int(loop.last_token[0])}, "
          f"log probability {float(loop.logprob[0]):.3f}, alternatives {loop.top_ids[0].tolist()}")
    loop.finish(torch.ones(a.requests, dtype=torch.int32, device=loop.device))
    print(f"{int(loop.free_count)} of {loop.pool.shape[2]} pages free again")
    loop.close()


if __name__ == "__main__":
    main()
