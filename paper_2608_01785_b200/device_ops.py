"""Operators of a decoding loop whose lengths, positions and page tables stay on the device, on torch tensors.

Each function checks its tensors' types, shapes and layout, and makes one call of the C ABI (include/horizonserve_device.h and, for
requests that continue one prompt in several ways, include/horizonserve_beams.h have the definitions) on the current stream of the tensors' device.  Nothing here allocates device memory or synchronises: outputs,
the workspace (`workspace()`) and the status word are the caller's.  There is no other implementation behind them.
"""
from __future__ import annotations

import ctypes as C
import importlib
from typing import Optional

import torch

from . import binding as B

WORKSPACE_BYTES = 32 << 20
MAX_SEQS = 4096
MAX_ALTERNATIVES = 32
MAX_BEAMS = 32
MAX_SHARED_SEQS = 2048
PAGE = 16
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = range(4)
EXPORTS = ("hs_op_step_tables", "hs_op_release_pages", "hs_op_rope_table", "hs_op_rope_cache", "hs_op_paged_attention", "hs_op_token_logprobs")
BEAM_EXPORTS = ("hs_op_beam_select", "hs_op_fork_pages", "hs_op_copy_pages", "hs_op_compact_pages", "hs_op_shared_attention")

_binding = None


def _load():
    """The compiled checks and calls (csrc/device_binding.cpp), bound to the library's entry points."""
    global _binding
    lib = B.lib()
    try:
        binding = importlib.import_module("._device_binding", __package__)
    except ImportError as e:
        raise RuntimeError("_device_binding.so is missing or does not fit this torch: build it with `python -m paper_2608_01785_b200.build`") from e
    binding.bind(*(C.cast(getattr(lib, name), C.c_void_p).value for name in EXPORTS + BEAM_EXPORTS))
    _binding = binding
    return binding


def workspace(device="cuda") -> torch.Tensor:
    """Scratch of the operators, zeroed once; one per stream that may run beside another."""
    return torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device=device)


def sm_count(device_index: int) -> int:
    return torch.cuda.get_device_properties(device_index).multi_processor_count


def step_tables(ctx_len, q_len, free_list, free_count, block_tables, kv_len, tok_begin, tok_seq, tok_pos, tok_slot, free_count_out, workspace, status,
                sm_budget: Optional[int] = None) -> None:
    """Allocates the pages of a step and writes its metadata (hs_op_step_tables).  All int32; block_tables [n_seqs, max_pages_per_seq] is extended
    in place, kv_len may be ctx_len, free_count_out may be free_count; the per-token tensors' length is the step's capacity."""
    st = (_binding or _load()).step_tables(ctx_len, q_len, free_list, free_count, block_tables, kv_len, tok_begin, tok_seq, tok_pos, tok_slot, free_count_out,
                                           workspace, status, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_step_tables")


def release_pages(done, ctx_len, block_tables, free_list, free_count, workspace, status, sm_budget: Optional[int] = None) -> None:
    """Gives the pages of the requests with done != 0 back to the stack (hs_op_release_pages).  Rows that share pages are ended by fork_pages."""
    st = (_binding or _load()).release_pages(done, ctx_len, block_tables, free_list, free_count, workspace, status, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_release_pages")


def rope_table(table, base: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0, trained_positions: int = 0, turns_slow: float = 1.0,
               turns_fast: float = 32.0, magnitude: float = 1.0, sm_budget: Optional[int] = None) -> None:
    """Fills table, fp32 [max_position, rotary_dim / 2, 2], with cos and sin (hs_op_rope_table)."""
    st = (_binding or _load()).rope_table(table, base, scaling, factor, trained_positions, turns_slow, turns_fast, magnitude, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_rope_table")


def rope_cache(q, k, v, tok_pos, tok_slot, table, q_out, kv_pool, layer: int, status, interleaved: bool = False, sm_budget: Optional[int] = None) -> None:
    """Rotates q and k by their tokens' positions and writes q to q_out, k and v to their slots of the cache (hs_op_rope_cache).
    q, k, v: [tokens, heads, head_dim] of one type, rows of any stride; the table's width says how much of a head rotates."""
    st = (_binding or _load()).rope_cache(q, k, v, tok_pos, tok_slot, table, q_out, kv_pool, layer, status, interleaved, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_rope_cache")


def paged_attention(q, kv_pool, layer: int, block_tables, kv_len, o, workspace, status, lse=None, tok_begin=None, max_q_len: int = 1, prefix_len=None,
                    slopes=None, scale: Optional[float] = None, cap: float = 0.0, window: int = 0, sm_budget: Optional[int] = None) -> None:
    """Attention of a step's tokens over the paged cache (hs_op_paged_attention).  q, o: [tokens, query heads, head_dim] in the cache's
    type; lse: fp32 [tokens, query heads]; max_q_len 1 is decoding, one row per sequence.  scale: head_dim^-1/2 if it is not given."""
    st = (_binding or _load()).paged_attention(q, kv_pool, layer, block_tables, kv_len, o, workspace, status, lse, tok_begin, max_q_len, prefix_len, slopes,
                                               scale, cap, window, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_paged_attention")


def token_logprobs(logits, targets, logprob, workspace, status, entropy=None, rank=None, top_ids=None, top_logprobs=None, scale: float = 1.0,
                   sm_budget: Optional[int] = None) -> None:
    """Log probability and rank of each row's target, its entropy and its top alternatives (hs_op_token_logprobs).  logits: [rows, vocab] in
    fp32, bf16 or fp16, rows of any stride; top_ids, top_logprobs: [rows, n_top]."""
    st = (_binding or _load()).token_logprobs(logits, targets, logprob, workspace, status, entropy, rank, top_ids, top_logprobs, scale, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_token_logprobs")


def beam_select(logits, scores, out_score, out_parent, out_token, workspace, status, done=None, weight=None, out_done=None, lse=None, end_token: int = -1,
                scale: float = 1.0, sm_budget: Optional[int] = None) -> None:
    """The best continuations of every request over its beams and the vocabulary (hs_op_beam_select).  logits: [requests * beams, vocab] in fp32, bf16
    or fp16, rows of any stride; scores, done, weight: [requests, beams]; out_*: [requests, continuations]; lse: [requests * beams]."""
    st = (_binding or _load()).beam_select(logits, scores, out_score, out_parent, out_token, workspace, status, done, weight, out_done, lse, end_token, scale,
                                           sm_budget)
    if st:
        raise B.HsError(st, "hs_op_beam_select")


def fork_pages(parent, ctx_len, block_tables, shares, free_list, free_count, copy_src, copy_dst, copy_len, workspace, status,
               sm_budget: Optional[int] = None) -> None:
    """Rows of the block tables continue the rows `parent`, or end (-1), and share their pages (hs_op_fork_pages).  All int32; ctx_len, block_tables, shares,
    free_list and free_count are changed in place; copy_*: [rows], what copy_pages then has to copy."""
    st = (_binding or _load()).fork_pages(parent, ctx_len, block_tables, shares, free_list, free_count, copy_src, copy_dst, copy_len, workspace, status, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_fork_pages")


def copy_pages(kv_pool, src, dst, status, length=None, sm_budget: Optional[int] = None) -> None:
    """Copies keys and values of the pages src to the pages dst in every layer (hs_op_copy_pages); their first `length` tokens if it is given."""
    st = (_binding or _load()).copy_pages(kv_pool, src, dst, status, length, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_copy_pages")


def compact_pages(n_keep: int, ctx_len, block_tables, shares, free_list, free_count, copy_src, copy_dst, workspace, status, sm_budget: Optional[int] = None) -> None:
    """Moves pages below n_keep, so that the pool's upper end is free (hs_op_compact_pages); copy_pages then has to copy copy_src to copy_dst."""
    st = (_binding or _load()).compact_pages(n_keep, ctx_len, block_tables, shares, free_list, free_count, copy_src, copy_dst, workspace, status, sm_budget)
    if st:
        raise B.HsError(st, "hs_op_compact_pages")


def shared_attention(q, kv_pool, layer: int, block_tables, kv_len, group_begin, shared_len, o, workspace, status, lse=None, slopes=None,
                     scale: Optional[float] = None, cap: float = 0.0, sm_budget: Optional[int] = None) -> None:
    """Attention of one new token per sequence over the paged cache, the keys that a group of sequences shares read once (hs_op_shared_attention).
    q, o: [sequences, query heads, head_dim] in the cache's type; group_begin: [groups + 1]; shared_len: [groups]; lse: fp32 [sequences, query heads]."""
    st = (_binding or _load()).shared_attention(q, kv_pool, layer, block_tables, kv_len, group_begin, shared_len, o, workspace, status, lse, slopes, scale, cap,
                                                sm_budget)
    if st:
        raise B.HsError(st, "hs_op_shared_attention")
