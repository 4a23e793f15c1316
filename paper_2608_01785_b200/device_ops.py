"""Operators of a decoding loop whose lengths, positions and page tables stay on the device, on torch tensors.

Each function checks its tensors' types, shapes and layout, and makes one call of the C ABI (include/horizonserve_device.h has
the definitions) on the current stream of the tensors' device.  Nothing here allocates device memory or synchronises: outputs,
the workspace (`workspace()`) and the status word are the caller's.  There is no other implementation behind them.
"""
from __future__ import annotations

import ctypes as C
import struct
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
_I32, _F32 = torch.int32, torch.float32

# The description structs of the C ABI, packed with their native alignment ("i" int32, "q" int64, "P" pointer, "f", "d").
_STEP_TABLES = struct.Struct("@4i13P")
_RELEASE_PAGES = struct.Struct("@3i7P")
_ROPE_TABLE = struct.Struct("@4i5dP")
_ROPE_CACHE = struct.Struct("@8i3P3q3P4iPq2P")
_PAGED_ATTENTION = struct.Struct("@11iPq6P2fiPq3P")
_TOKEN_LOGPROBS = struct.Struct("@4iPqPf7P")

_fns = None
_sms = {}


def _functions():
    global _fns
    if _fns is None:
        lib = B.lib()
        fns = {}
        for name in EXPORTS:
            fns[name] = getattr(lib, name)
            fns[name].argtypes = [C.c_char_p, C.c_int32, C.c_void_p]
            fns[name].restype = C.c_int
        _fns = fns
    return _fns


def workspace(device="cuda") -> torch.Tensor:
    """Scratch of the operators, zeroed once; one per stream that may run beside another."""
    return torch.zeros(WORKSPACE_BYTES, dtype=torch.uint8, device=device)


def sm_count(device_index: int) -> int:
    if device_index not in _sms:
        _sms[device_index] = torch.cuda.get_device_properties(device_index).multi_processor_count
    return _sms[device_index]


def _call(name: str, args: bytes, d: int, sm_budget: Optional[int]) -> None:
    """One call on the current stream of device d.  (The checks of every argument run in front of every call: what they cost is part of a small
    operator's time, so they are plain comparisons, and a message is made only where one fails.)"""
    fn = (_fns or _functions())[name]
    if d < 0:
        raise ValueError("the operators work on CUDA tensors")
    budget = (_sms.get(d) or sm_count(d)) if sm_budget is None else sm_budget
    if d == torch._C._cuda_getDevice():
        st = fn(args, budget, torch._C._cuda_getCurrentRawStream(d))
    else:
        with torch.cuda.device(d):
            st = fn(args, budget, torch._C._cuda_getCurrentRawStream(d))
    if st != B.HS_OK:
        raise B.HsError(st, name)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _vec(t: Optional[torch.Tensor], n: int, dtype, d: int, what: str) -> int:
    """Address of a contiguous tensor of `dtype` with n elements (any number if -1) on device d; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != d or not t.is_contiguous() or (t.numel() != n and n >= 0):
        raise ValueError(f"{what}: a contiguous {dtype} tensor of {'any number of' if n < 0 else n} elements on device {d} is wanted")
    return t.data_ptr()


def _scratch(workspace: torch.Tensor, d: int) -> int:
    if workspace.get_device() != d or not workspace.is_contiguous() or workspace.nbytes < WORKSPACE_BYTES:
        raise ValueError(f"workspace: {WORKSPACE_BYTES} contiguous bytes on device {d} are wanted")
    return workspace.data_ptr()


def _rows(t: torch.Tensor, rows: int, heads: int, dim: int, d: int, what: str):
    """(address, elements between rows) of [rows, heads, dim] whose rows are contiguous."""
    shape = t.shape
    if len(shape) == 3 and shape[0] == rows and shape[1] == heads and shape[2] == dim and t.get_device() == d:
        s0, s1, s2 = t.stride()
        if (s2 == 1 or dim == 1) and (s1 == dim or heads == 1):
            return t.data_ptr(), s0 if rows > 1 else heads * dim
    raise ValueError(f"{what}: a [{rows}, {heads}, {dim}] tensor with contiguous rows on device {d} is wanted")


def _pool(kv_pool: torch.Tensor, layer: int):
    shape = kv_pool.shape
    if len(shape) != 6 or shape[1] != 2 or shape[4] != PAGE or not kv_pool.is_contiguous():
        raise ValueError(f"kv_pool: a contiguous [layers, 2, pages, kv heads, {PAGE}, head_dim] tensor is wanted")
    if not 0 <= layer < shape[0]:
        raise ValueError("layer is outside the pool")
    return shape[0], shape[2], shape[3], shape[5]


def _table_rows(t: torch.Tensor, n: int, d: int):
    """(address, row length) of the block tables of n requests."""
    shape = t.shape
    if len(shape) != 2 or shape[0] != n:
        raise ValueError("block_tables: one row per request is wanted")
    return _vec(t, -1, _I32, d, "block_tables"), shape[1]


def step_tables(ctx_len, q_len, free_list, free_count, block_tables, kv_len, tok_begin, tok_seq, tok_pos, tok_slot, free_count_out, workspace, status,
                sm_budget: Optional[int] = None) -> None:
    """Allocates the pages of a step and writes its metadata (hs_op_step_tables).  All int32; block_tables [n_seqs, max_pages_per_seq] is extended
    in place, kv_len may be ctx_len, free_count_out may be free_count; the per-token tensors' length is the step's capacity."""
    d, n, cap = ctx_len.get_device(), ctx_len.numel(), tok_seq.numel()
    tables, width = _table_rows(block_tables, n, d)
    _call("hs_op_step_tables", _STEP_TABLES.pack(
        n, width, free_list.numel(), cap, _vec(ctx_len, n, _I32, d, "ctx_len"), _vec(q_len, n, _I32, d, "q_len"),
        _vec(free_list, -1, _I32, d, "free_list"), _vec(free_count, 1, _I32, d, "free_count"), tables, _vec(kv_len, n, _I32, d, "kv_len"),
        _vec(tok_begin, n + 1, _I32, d, "tok_begin"), _vec(tok_seq, cap, _I32, d, "tok_seq"), _vec(tok_pos, cap, _I32, d, "tok_pos"),
        _vec(tok_slot, cap, _I32, d, "tok_slot"), _vec(free_count_out, 1, _I32, d, "free_count_out"), _scratch(workspace, d),
        _vec(status, 1, _I32, d, "status")), d, sm_budget)


def release_pages(done, ctx_len, block_tables, free_list, free_count, workspace, status, sm_budget: Optional[int] = None) -> None:
    """Gives the pages of the requests with done != 0 back to the stack (hs_op_release_pages)."""
    d, n = ctx_len.get_device(), ctx_len.numel()
    tables, width = _table_rows(block_tables, n, d)
    _call("hs_op_release_pages", _RELEASE_PAGES.pack(
        n, width, free_list.numel(), _vec(done, n, _I32, d, "done"), _vec(ctx_len, n, _I32, d, "ctx_len"), tables, _vec(free_list, -1, _I32, d, "free_list"),
        _vec(free_count, 1, _I32, d, "free_count"), _scratch(workspace, d), _vec(status, 1, _I32, d, "status")), d, sm_budget)


def rope_table(table, base: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0, trained_positions: int = 0, turns_slow: float = 1.0,
               turns_fast: float = 32.0, magnitude: float = 1.0, sm_budget: Optional[int] = None) -> None:
    """Fills table, fp32 [max_position, rotary_dim / 2, 2], with cos and sin (hs_op_rope_table)."""
    _need(table.dim() == 3 and table.shape[2] == 2, "table: [positions, pairs, 2] is wanted")
    d = table.get_device()
    _call("hs_op_rope_table", _ROPE_TABLE.pack(table.shape[0], 2 * table.shape[1], scaling, trained_positions, base, factor, turns_slow, turns_fast,
                                               magnitude, _vec(table, -1, _F32, d, "table")), d, sm_budget)


def rope_cache(q, k, v, tok_pos, tok_slot, table, q_out, kv_pool, layer: int, status, interleaved: bool = False, sm_budget: Optional[int] = None) -> None:
    """Rotates q and k by their tokens' positions and writes q to q_out, k and v to their slots of the cache (hs_op_rope_cache).
    q, k, v: [tokens, heads, head_dim] of one type, rows of any stride; the table's width says how much of a head rotates."""
    layers, pages, hkv, dim = _pool(kv_pool, layer)
    d, (n, hq, _), (positions, pairs, two) = kv_pool.get_device(), q.shape, table.shape
    src, dst = _TYPES.get(q.dtype), _TYPES.get(kv_pool.dtype)
    if src is None or k.dtype is not q.dtype or v.dtype is not q.dtype:
        raise ValueError("q, k, v: one of fp32, bf16, fp16 is wanted")
    if not dst or q_out.dtype is not kv_pool.dtype:
        raise ValueError("q_out and kv_pool: both bf16 or both fp16 are wanted")
    if two != 2:
        raise ValueError("table: [positions, pairs, 2] is wanted")
    qp, qs = _rows(q, n, hq, dim, d, "q")
    kp, ks = _rows(k, n, hkv, dim, d, "k")
    vp, vs = _rows(v, n, hkv, dim, d, "v")
    op, os_ = _rows(q_out, n, hq, dim, d, "q_out")
    _call("hs_op_rope_cache", _ROPE_CACHE.pack(
        n, hq, hkv, dim, 2 * pairs, 1 if interleaved else 0, src, dst, qp, kp, vp, qs, ks, vs, _vec(tok_pos, n, _I32, d, "tok_pos"),
        _vec(tok_slot, n, _I32, d, "tok_slot"), _vec(table, -1, _F32, d, "table"), positions, layers, layer, pages, op, os_, kv_pool.data_ptr(),
        _vec(status, 1, _I32, d, "status")), d, sm_budget)


def paged_attention(q, kv_pool, layer: int, block_tables, kv_len, o, workspace, status, lse=None, tok_begin=None, max_q_len: int = 1, prefix_len=None,
                    slopes=None, scale: Optional[float] = None, cap: float = 0.0, window: int = 0, sm_budget: Optional[int] = None) -> None:
    """Attention of a step's tokens over the paged cache (hs_op_paged_attention).  q, o: [tokens, query heads, head_dim] in the cache's
    type; lse: fp32 [tokens, query heads]; max_q_len 1 is decoding, one row per sequence."""
    layers, pages, hkv, dim = _pool(kv_pool, layer)
    d, n, (t, hq, _) = kv_pool.get_device(), kv_len.numel(), q.shape
    kind = _TYPES.get(kv_pool.dtype)
    if not kind or q.dtype is not kv_pool.dtype or o.dtype is not kv_pool.dtype:
        raise ValueError("q, o and kv_pool: all bf16 or all fp16 are wanted")
    qp, qs = _rows(q, t, hq, dim, d, "q")
    op, os_ = _rows(o, t, hq, dim, d, "o")
    tables, width = _table_rows(block_tables, n, d)
    _call("hs_op_paged_attention", _PAGED_ATTENTION.pack(
        n, t, max_q_len, hq, hkv, dim, kind, layers, layer, pages, width, qp, qs, kv_pool.data_ptr(), tables, _vec(kv_len, n, _I32, d, "kv_len"),
        _vec(tok_begin, n + 1, _I32, d, "tok_begin"), _vec(prefix_len, n, _I32, d, "prefix_len"), _vec(slopes, hq, _F32, d, "slopes"),
        dim ** -0.5 if scale is None else scale, cap, window, op, os_, _vec(lse, t * hq, _F32, d, "lse"), _scratch(workspace, d),
        _vec(status, 1, _I32, d, "status")), d, sm_budget)


def token_logprobs(logits, targets, logprob, workspace, status, entropy=None, rank=None, top_ids=None, top_logprobs=None, scale: float = 1.0,
                   sm_budget: Optional[int] = None) -> None:
    """Log probability and rank of each row's target, its entropy and its top alternatives (hs_op_token_logprobs).  logits: [rows, vocab] in
    fp32, bf16 or fp16, rows of any stride; top_ids, top_logprobs: [rows, n_top]."""
    d, (n, v), (s0, s1), kind = logits.get_device(), logits.shape, logits.stride(), _TYPES.get(logits.dtype)
    if kind is None or (s1 != 1 and v != 1):
        raise ValueError("logits: [rows, vocab] in fp32, bf16 or fp16 with contiguous rows is wanted")
    n_top = 0
    if top_ids is not None:
        if top_logprobs is None or top_ids.dim() != 2 or top_ids.shape[0] != n:
            raise ValueError("top_ids and top_logprobs: [rows, alternatives] each are wanted")
        n_top = top_ids.shape[1]
    elif top_logprobs is not None:
        raise ValueError("top_ids and top_logprobs belong together")
    _call("hs_op_token_logprobs", _TOKEN_LOGPROBS.pack(
        n, v, kind, n_top, logits.data_ptr(), s0 if n > 1 else v, _vec(targets, n, _I32, d, "targets"), scale, _vec(logprob, n, _F32, d, "logprob"),
        _vec(entropy, n, _F32, d, "entropy"), _vec(rank, n, _I32, d, "rank"), _vec(top_ids, n * n_top, _I32, d, "top_ids"),
        _vec(top_logprobs, n * n_top, _F32, d, "top_logprobs"), _scratch(workspace, d), _vec(status, 1, _I32, d, "status")), d, sm_budget)
