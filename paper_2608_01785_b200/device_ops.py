"""Operators of a decoding loop whose lengths, positions and page tables stay on the device, on torch tensors.

Each function checks its tensors' types, shapes and layout, and makes one call of the C ABI (include/horizonserve_device.h has
the definitions) on the current stream of the tensors' device.  Nothing here allocates device memory or synchronises: outputs,
the workspace (`workspace()`) and the status word are the caller's.  There is no other implementation behind them.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from . import binding as B

WORKSPACE_BYTES = 32 << 20
MAX_SEQS = 4096
MAX_ALTERNATIVES = 32
PAGE = 16
TYPE_F32, TYPE_BF16, TYPE_F16 = range(3)
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = range(4)
EXPORTS = ("hs_op_step_tables", "hs_op_release_pages", "hs_op_rope_table", "hs_op_rope_cache", "hs_op_paged_attention", "hs_op_token_logprobs")

_TYPES = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}
_I, _L, _P, _F, _D = C.c_int32, C.c_int64, C.c_void_p, C.c_float, C.c_double


def _struct(name, fields):
    return type(name, (C.Structure,), {"_fields_": [(f, t) for t, names in fields for f in names.split()]})


hs_step_tables_t = _struct("hs_step_tables_t", [
    (_I, "n_seqs max_pages_per_seq num_pages max_tokens"),
    (_P, "ctx_len q_len free_list free_count block_tables kv_len tok_begin tok_seq tok_pos tok_slot free_count_out workspace status")])
hs_release_pages_t = _struct("hs_release_pages_t", [
    (_I, "n_seqs max_pages_per_seq num_pages"), (_P, "done ctx_len block_tables free_list free_count workspace status")])
hs_rope_table_t = _struct("hs_rope_table_t", [
    (_I, "max_position rotary_dim scaling trained_positions"), (_D, "base factor turns_slow turns_fast magnitude"), (_P, "table")])
hs_rope_cache_t = _struct("hs_rope_cache_t", [
    (_I, "n_tokens n_q_heads n_kv_heads head_dim rotary_dim interleaved src_type cache_type"), (_P, "q k v"), (_L, "q_stride k_stride v_stride"),
    (_P, "tok_pos tok_slot table"), (_I, "max_position n_layers layer num_pages"), (_P, "q_out"), (_L, "q_out_stride"), (_P, "kv_pool status")])
hs_paged_attention_t = _struct("hs_paged_attention_t", [
    (_I, "n_seqs n_tokens max_q_len n_q_heads n_kv_heads head_dim type n_layers layer num_pages max_pages_per_seq"), (_P, "q"), (_L, "q_stride"),
    (_P, "kv_pool block_tables kv_len tok_begin prefix_len slopes"), (_F, "scale cap"), (_I, "window"), (_P, "o"), (_L, "o_stride"),
    (_P, "lse workspace status")])
hs_token_logprobs_t = _struct("hs_token_logprobs_t", [
    (_I, "n_rows vocab type n_top"), (_P, "logits"), (_L, "row_stride"), (_P, "targets"), (_F, "scale"),
    (_P, "logprob entropy rank top_ids top_logprobs workspace status")])

_fns = None
_sms = {}


def _functions():
    global _fns
    if _fns is None:
        lib = B.lib()
        _fns = {}
        for name in EXPORTS:
            fn = getattr(lib, name)
            fn.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
            fn.restype = C.c_int
            _fns[name] = fn
    return _fns


def workspace(device="cuda") -> torch.Tensor:
    """Scratch of the operators, zeroed once; one per stream that may run beside another."""
    return torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device=device)


def sm_count(device: torch.device) -> int:
    i = device.index if device.index is not None else torch.cuda.current_device()
    if i not in _sms:
        _sms[i] = torch.cuda.get_device_properties(i).multi_processor_count
    return _sms[i]


def _call(name: str, args, device: torch.device, sm_budget: Optional[int]) -> None:
    fn = _functions()[name]
    budget = sm_count(device) if sm_budget is None else sm_budget
    if device.index is not None and device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            st = fn(C.addressof(args), budget, torch.cuda.current_stream().cuda_stream)
    else:
        st = fn(C.addressof(args), budget, torch.cuda.current_stream().cuda_stream)
    if st != B.HS_OK:
        raise B.HsError(st, name)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _vec(t: Optional[torch.Tensor], n: Optional[int], dtype, device, what: str) -> int:
    """Address of a contiguous tensor of `dtype` with n elements (any number if None); 0 for None."""
    if t is None:
        return 0
    if t.dtype != dtype or t.device != device or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{what}: a contiguous {dtype} tensor of {'any number of' if n is None else n} elements on {device} is wanted")
    return t.data_ptr()


def _scratch(workspace: torch.Tensor, status: torch.Tensor, device):
    _need(workspace.device == device and workspace.is_contiguous() and workspace.numel() * workspace.element_size() >= WORKSPACE_BYTES,
          f"workspace: {WORKSPACE_BYTES} contiguous bytes on {device} are wanted")
    return workspace.data_ptr(), _vec(status, 1, torch.int32, device, "status")


def _rows(t: torch.Tensor, heads: int, dim: int, device, what: str):
    """(address, elements between rows) of [rows, heads, dim] whose rows are contiguous."""
    _need(t.dim() == 3 and t.shape[1] == heads and t.shape[2] == dim and t.device == device and (t.stride(2) == 1 or dim == 1)
          and (t.stride(1) == dim or heads == 1), f"{what}: a [rows, {heads}, {dim}] tensor with contiguous rows on {device} is wanted")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else heads * dim


def _pool(kv_pool: torch.Tensor, layer: int):
    _need(kv_pool.dim() == 6 and kv_pool.shape[1] == 2 and kv_pool.shape[4] == PAGE and kv_pool.is_contiguous(),
          f"kv_pool: a contiguous [layers, 2, pages, kv heads, {PAGE}, head_dim] tensor is wanted")
    _need(0 <= layer < kv_pool.shape[0], "layer is outside the pool")
    return kv_pool.shape[0], kv_pool.shape[2], kv_pool.shape[3], kv_pool.shape[5]


def step_tables(ctx_len, q_len, free_list, free_count, block_tables, kv_len, tok_begin, tok_seq, tok_pos, tok_slot, free_count_out, workspace, status,
                sm_budget: Optional[int] = None) -> None:
    """Allocates the pages of a step and writes its metadata (hs_op_step_tables).  All int32; block_tables [n_seqs, max_pages_per_seq] is extended
    in place, kv_len may be ctx_len, free_count_out may be free_count; the per-token tensors' length is the step's capacity."""
    d, i32, n = ctx_len.device, torch.int32, ctx_len.numel()
    _need(block_tables.dim() == 2 and block_tables.shape[0] == n, "block_tables: one row per request is wanted")
    cap = tok_seq.numel()
    ws, st = _scratch(workspace, status, d)
    a = hs_step_tables_t(n, block_tables.shape[1], free_list.numel(), cap, _vec(ctx_len, n, i32, d, "ctx_len"), _vec(q_len, n, i32, d, "q_len"),
                         _vec(free_list, None, i32, d, "free_list"), _vec(free_count, 1, i32, d, "free_count"), _vec(block_tables, None, i32, d, "block_tables"),
                         _vec(kv_len, n, i32, d, "kv_len"), _vec(tok_begin, n + 1, i32, d, "tok_begin"), _vec(tok_seq, cap, i32, d, "tok_seq"),
                         _vec(tok_pos, cap, i32, d, "tok_pos"), _vec(tok_slot, cap, i32, d, "tok_slot"), _vec(free_count_out, 1, i32, d, "free_count_out"), ws, st)
    _call("hs_op_step_tables", a, d, sm_budget)


def release_pages(done, ctx_len, block_tables, free_list, free_count, workspace, status, sm_budget: Optional[int] = None) -> None:
    """Gives the pages of the requests with done != 0 back to the stack (hs_op_release_pages)."""
    d, i32, n = ctx_len.device, torch.int32, ctx_len.numel()
    _need(block_tables.dim() == 2 and block_tables.shape[0] == n, "block_tables: one row per request is wanted")
    ws, st = _scratch(workspace, status, d)
    a = hs_release_pages_t(n, block_tables.shape[1], free_list.numel(), _vec(done, n, i32, d, "done"), _vec(ctx_len, n, i32, d, "ctx_len"),
                           _vec(block_tables, None, i32, d, "block_tables"), _vec(free_list, None, i32, d, "free_list"), _vec(free_count, 1, i32, d, "free_count"),
                           ws, st)
    _call("hs_op_release_pages", a, d, sm_budget)


def rope_table(table, base: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0, trained_positions: int = 0, turns_slow: float = 1.0,
               turns_fast: float = 32.0, magnitude: float = 1.0, sm_budget: Optional[int] = None) -> None:
    """Fills table, fp32 [max_position, rotary_dim / 2, 2], with cos and sin (hs_op_rope_table)."""
    _need(table.dim() == 3 and table.shape[2] == 2, "table: [positions, pairs, 2] is wanted")
    a = hs_rope_table_t(table.shape[0], 2 * table.shape[1], scaling, trained_positions, base, factor, turns_slow, turns_fast, magnitude,
                        _vec(table, None, torch.float32, table.device, "table"))
    _call("hs_op_rope_table", a, table.device, sm_budget)


def rope_cache(q, k, v, tok_pos, tok_slot, table, q_out, kv_pool, layer: int, status, interleaved: bool = False, sm_budget: Optional[int] = None) -> None:
    """Rotates q and k by their tokens' positions and writes q to q_out, k and v to their slots of the cache (hs_op_rope_cache).
    q, k, v: [tokens, heads, head_dim] of one type, rows of any stride; the table's width says how much of a head rotates."""
    layers, pages, hkv, dim = _pool(kv_pool, layer)
    d, n, hq = q.device, q.shape[0], q.shape[1]
    _need(q.dtype in _TYPES and k.dtype == q.dtype and v.dtype == q.dtype, "q, k, v: one of fp32, bf16, fp16 is wanted")
    _need(q_out.dtype == kv_pool.dtype and kv_pool.dtype in (torch.bfloat16, torch.float16), "q_out and kv_pool: both bf16 or both fp16 are wanted")
    _need(k.shape[0] == n and v.shape[0] == n and q_out.shape[0] == n and kv_pool.device == d, "q, k, v, q_out: as many rows each, on the pool's device")
    _need(table.dim() == 3 and table.shape[2] == 2, "table: [positions, pairs, 2] is wanted")
    qp, qs = _rows(q, hq, dim, d, "q")
    kp, ks = _rows(k, hkv, dim, d, "k")
    vp, vs = _rows(v, hkv, dim, d, "v")
    op, os_ = _rows(q_out, hq, dim, d, "q_out")
    a = hs_rope_cache_t(n, hq, hkv, dim, 2 * table.shape[1], int(interleaved), _TYPES[q.dtype], _TYPES[kv_pool.dtype], qp, kp, vp, qs, ks, vs,
                        _vec(tok_pos, n, torch.int32, d, "tok_pos"), _vec(tok_slot, n, torch.int32, d, "tok_slot"),
                        _vec(table, None, torch.float32, d, "table"), table.shape[0], layers, layer, pages, op, os_, kv_pool.data_ptr(),
                        _vec(status, 1, torch.int32, d, "status"))
    _call("hs_op_rope_cache", a, d, sm_budget)


def paged_attention(q, kv_pool, layer: int, block_tables, kv_len, o, workspace, status, lse=None, tok_begin=None, max_q_len: int = 1, prefix_len=None,
                    slopes=None, scale: Optional[float] = None, cap: float = 0.0, window: int = 0, sm_budget: Optional[int] = None) -> None:
    """Attention of a step's tokens over the paged cache (hs_op_paged_attention).  q, o: [tokens, query heads, head_dim] in the cache's
    type; lse: fp32 [tokens, query heads]; max_q_len 1 is decoding, one row per sequence."""
    layers, pages, hkv, dim = _pool(kv_pool, layer)
    d, t, hq, n = q.device, q.shape[0], q.shape[1], kv_len.numel()
    _need(q.dtype == kv_pool.dtype and o.dtype == q.dtype and q.dtype in (torch.bfloat16, torch.float16), "q, o and kv_pool: all bf16 or all fp16 are wanted")
    _need(o.shape[0] == t and kv_pool.device == d, "o: as many rows as q, on the pool's device")
    _need(block_tables.dim() == 2 and block_tables.shape[0] == n, "block_tables: one row per sequence is wanted")
    qp, qs = _rows(q, hq, dim, d, "q")
    op, os_ = _rows(o, hq, dim, d, "o")
    ws, st = _scratch(workspace, status, d)
    i32 = torch.int32
    a = hs_paged_attention_t(n, t, max_q_len, hq, hkv, dim, _TYPES[q.dtype], layers, layer, pages, block_tables.shape[1], qp, qs, kv_pool.data_ptr(),
                             _vec(block_tables, None, i32, d, "block_tables"), _vec(kv_len, n, i32, d, "kv_len"), _vec(tok_begin, n + 1, i32, d, "tok_begin"),
                             _vec(prefix_len, n, i32, d, "prefix_len"), _vec(slopes, hq, torch.float32, d, "slopes"),
                             dim ** -0.5 if scale is None else scale, cap, window, op, os_, _vec(lse, t * hq, torch.float32, d, "lse"), ws, st)
    _call("hs_op_paged_attention", a, d, sm_budget)


def token_logprobs(logits, targets, logprob, workspace, status, entropy=None, rank=None, top_ids=None, top_logprobs=None, scale: float = 1.0,
                   sm_budget: Optional[int] = None) -> None:
    """Log probability and rank of each row's target, its entropy and its top alternatives (hs_op_token_logprobs).  logits: [rows, vocab] in
    fp32, bf16 or fp16, rows of any stride; top_ids, top_logprobs: [rows, n_top]."""
    _need(logits.dim() == 2 and logits.dtype in _TYPES and (logits.stride(1) == 1 or logits.shape[1] == 1), "logits: [rows, vocab] with contiguous rows is wanted")
    _need((top_ids is None) == (top_logprobs is None), "top_ids and top_logprobs belong together")
    d, (n, v), f32 = logits.device, logits.shape, torch.float32
    n_top = 0
    if top_ids is not None:
        _need(top_ids.dim() == 2 and top_ids.shape[0] == n, "top_ids: [rows, alternatives] is wanted")
        n_top = top_ids.shape[1]
    ws, st = _scratch(workspace, status, d)
    a = hs_token_logprobs_t(n, v, _TYPES[logits.dtype], n_top, logits.data_ptr(), logits.stride(0) if n > 1 else v,
                            _vec(targets, n, torch.int32, d, "targets"), scale, _vec(logprob, n, f32, d, "logprob"), _vec(entropy, n, f32, d, "entropy"),
                            _vec(rank, n, torch.int32, d, "rank"), _vec(top_ids, n * n_top, torch.int32, d, "top_ids"),
                            _vec(top_logprobs, n * n_top, f32, d, "top_logprobs"), ws, st)
    _call("hs_op_token_logprobs", a, d, sm_budget)
