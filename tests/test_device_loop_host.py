"""The device-resident loop's host side on the CPU: its tensors live here, the calls that would go to a GPU are recorded."""
import ctypes as C

import pytest
import torch

from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_ops as ops
from paper_2608_01785_b200.device_loop import DeviceLoop, LoopDims, make_weights

DIMS = LoopDims(n_layers=1, d_model=64, n_q_heads=1, n_kv_heads=1, head_dim=64, vocab=64)


class Head:
    """Stands for hs_head_*: remembers the rows of x that each call reads, refuses more rows than it was made for, and samples 7."""

    def __init__(self, monkeypatch):
        self.rows, self.max_rows = [], None
        monkeypatch.setattr(B, "make_head_config", self.config)
        monkeypatch.setattr(B, "hs_head_workspace_bytes", lambda cfg: 256)
        monkeypatch.setattr(B, "hs_head_create", lambda *a: 1)
        monkeypatch.setattr(B, "hs_head_destroy", lambda h: None)
        monkeypatch.setattr(B, "hs_head_step", self.step)

    def config(self, d_model, vocab, eps, max_rows, device):
        assert 1 <= max_rows <= 128
        self.max_rows = max_rows

    def step(self, head, y, rows, n, logits, tokens, budget, stream=0):
        if not 1 <= n <= self.max_rows:
            raise B.HsError(B.HS_ERR_INVALID_ARG, "hs_head_step")
        self.rows.append([list((C.c_int32 * n).from_address(rows)), (y, logits, tokens)])
        (C.c_int32 * n).from_address(tokens)[:] = [7] * n


@pytest.fixture()
def head(monkeypatch):
    h = Head(monkeypatch)
    monkeypatch.setattr(ops, "rope_table", lambda *a, **k: None)
    monkeypatch.setattr(ops, "token_logprobs", lambda *a, **k: None)
    monkeypatch.setattr(DeviceLoop, "_layers", lambda *a: None)
    monkeypatch.setattr(DeviceLoop, "_stream", lambda *a: 0)
    monkeypatch.setattr(DeviceLoop, "_budget", lambda *a: 1)
    return h


def tables(monkeypatch, begin, status):
    """hs_op_step_tables as its header has it: a step that is refused has no tokens and leaves the lengths as they are."""
    def step_tables(ctx, q, free_list, free_count, block_tables, kv_len, tok_begin, tok_seq, tok_pos, tok_slot, free_out, ws, st, sm_budget=None):
        tok_begin.copy_(torch.tensor(begin, dtype=torch.int32))
        kv_len.copy_(ctx if status else ctx + q)
        for t in (tok_seq, tok_pos, tok_slot):
            t.fill_(-1)
        st.fill_(status)
    monkeypatch.setattr(ops, "step_tables", step_tables)


@pytest.mark.parametrize("status", [B.HS_ERR_OUT_OF_PAGES, B.HS_ERR_INVALID_ARG])
def test_a_refused_prefill_reads_no_row_outside_its_buffers_and_samples_for_nobody(head, monkeypatch, status):
    tables(monkeypatch, [0, 0, 0, 0], status)
    loop = DeviceLoop(DIMS, make_weights(DIMS, device="cpu"), 3, 4, 64, 40)
    loop.last_token[:3] = torch.tensor([1, 2, 3])
    loop.prefill([[5] * 10, [6] * 20, [8]])
    assert [r for rows, _ in head.rows for r in rows if not 0 <= r < 40] == []
    assert loop.last_token[:3].tolist() == [1, 2, 3] and loop.ctx_len.tolist() == [0, 0, 0] and int(loop.status) == status
    loop.close()


def test_a_prefill_samples_from_the_last_rows(head, monkeypatch):
    tables(monkeypatch, [0, 10, 30, 31], 0)
    loop = DeviceLoop(DIMS, make_weights(DIMS, device="cpu"), 3, 4, 64, 40)
    loop.prefill([[5] * 10, [6] * 20, [8]])
    assert [r for rows, _ in head.rows for r in rows] == [9, 29, 30]
    assert loop.last_token[:3].tolist() == [7, 7, 7] and loop.ctx_len.tolist() == [10, 20, 1]
    loop.close()


@pytest.mark.parametrize("n", [128, 129, 300])
def test_any_number_of_requests_is_sampled_in_slices_of_the_heads_rows(head, monkeypatch, n):
    tables(monkeypatch, list(range(n + 1)), 0)
    loop = DeviceLoop(DIMS, make_weights(DIMS, device="cpu"), n, n, 16, n)
    loop.prefill([[5]] * n)
    assert [r for rows, _ in head.rows for r in rows] == list(range(n)) and loop.last_token[:n].tolist() == [7] * n
    y, logits, tokens = (loop._prompt_buffers[k].data_ptr() for k in ("x", "logits", "sampled"))
    at = 0
    for rows, pointers in head.rows:
        assert pointers == (y, logits + 4 * DIMS.vocab * at, tokens + 4 * at)
        at += len(rows)
    loop.close()


@pytest.mark.parametrize("n", [0, -1, 4097])
def test_a_number_of_requests_that_no_call_takes_is_refused_at_once(head, n):
    with pytest.raises(ValueError, match="n_requests"):
        DeviceLoop(DIMS, make_weights(DIMS, device="cpu"), n, 8, 16, 8)
