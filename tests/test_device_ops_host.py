"""CPU-only checks of the device-resident operators: the header, the library and the packed structs agree, wrong arguments are refused on the host
before any GPU is asked for, and the plain definitions of the GPU tests agree with the framework's host-side page allocator."""
import ctypes as C
import os
import re
import struct
import subprocess

import numpy as np
import pytest
import torch

import device_ref as ref
from oracle.paging import PageAllocator, plan_tokens
from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "horizonserve_device.h")
# The description structs as packed words ("i" int32, "q" int64, "P" pointer, "f", "d"), in the order of ops.EXPORTS.
STRUCTS = {name: struct.Struct(fmt) for name, fmt in {
    "hs_step_tables_t": "@4i13P", "hs_release_pages_t": "@3i7P", "hs_rope_table_t": "@4i5dP", "hs_rope_cache_t": "@8i3P3q3P4iPq2P",
    "hs_paged_attention_t": "@11iPq6P2fiPq3P", "hs_token_logprobs_t": "@4iPqPf7P"}.items()}


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def fields(name):
    """Member names of a struct of the header, in order."""
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text()).group(1)
    return [re.findall(r"\w+", part)[-1] for line in body.split(";") if line.strip() for part in line.split(",")]


def offsets(fmt):
    """Byte offset of every member of a struct format."""
    codes = [c for n, c in re.findall(r"(\d*)([a-zA-Z])", fmt[1:]) for _ in range(int(n or 1))]
    out = []
    for i, c in enumerate(codes):
        before = struct.calcsize("@" + "".join(codes[:i]) + "0" + c)
        out.append((before, struct.calcsize("@" + c)))
    return out


def test_every_declared_operator_is_exported_and_bound():
    names = re.findall(r"\b(hs_op_[a-z0-9_]+)\s*\(", text())
    assert sorted(names) == sorted(ops.EXPORTS) and len(names) == len(set(names)) == 6
    for n in names:
        assert hasattr(B.lib(), n), n


@pytest.mark.parametrize("compiler", ["gcc", "g++"])
def test_packed_structs_are_the_headers(tmp_path, compiler):
    lines = []
    for name, packed in STRUCTS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu %zu\\n", offsetof({name}, {f}), sizeof((({name} *)0)->{f}));' for f in fields(name)]
    src = tmp_path / ("m.c" if compiler == "gcc" else "m.cpp")
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"horizonserve_device.h\"\nint main(void) {\n" + "\n".join(lines)
                   + '\nprintf("%u %d %d\\n", HS_DEVICE_WORKSPACE_BYTES, HS_DEVICE_MAX_SEQS, HS_MAX_ALTERNATIVES);\nreturn 0;\n}\n')
    exe = str(tmp_path / "m")
    subprocess.run([compiler, "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines()
    want = []
    for name, packed in STRUCTS.items():
        of = offsets(packed.format)
        assert len(of) == len(fields(name)), name
        want.append(str(packed.size))
        want += [f"{o} {s}" for o, s in of]
    want.append(f"{ops.WORKSPACE_BYTES} {ops.MAX_SEQS} {ops.MAX_ALTERNATIVES}")
    assert got == want


P = 1 << 20        # an address that is aligned for everything; no call below gets as far as using it
GOOD = {
    "hs_step_tables_t": dict(n_seqs=4, max_pages_per_seq=8, num_pages=32, max_tokens=64),
    "hs_release_pages_t": dict(n_seqs=4, max_pages_per_seq=8, num_pages=32),
    "hs_rope_table_t": dict(max_position=64, rotary_dim=64, scaling=3, trained_positions=32, base=1e4, factor=2.0, turns_slow=1.0, turns_fast=32.0, magnitude=1.0),
    "hs_rope_cache_t": dict(n_tokens=4, n_q_heads=4, n_kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, src_type=0, cache_type=1, q_stride=256, k_stride=128,
                            v_stride=128, max_position=64, n_layers=2, layer=1, num_pages=32, q_out_stride=256),
    "hs_paged_attention_t": dict(n_seqs=4, n_tokens=4, max_q_len=1, n_q_heads=4, n_kv_heads=2, head_dim=64, type=1, n_layers=2, layer=1, num_pages=32,
                                 max_pages_per_seq=8, q_stride=256, scale=0.125, cap=0.0, window=0, o_stride=256),
    "hs_token_logprobs_t": dict(n_rows=4, vocab=100, type=0, n_top=5, row_stride=100, scale=1.0),
}
INF, NAN = float("inf"), float("nan")
INVALID, SHAPE = B.HS_ERR_INVALID_ARG, B.HS_ERR_UNSUPPORTED_SHAPE
REFUSED = {
    "hs_step_tables_t": [(dict(n_seqs=0), INVALID), (dict(max_tokens=0), INVALID), (dict(num_pages=0), INVALID), (dict(n_seqs=4097), SHAPE),
                         (dict(n_seqs=4096, max_pages_per_seq=32769), SHAPE), (dict(ctx_len=0), INVALID), (dict(tok_slot=0), INVALID),
                         (dict(workspace=P + 16), INVALID), (dict(workspace=0), INVALID), (dict(status=0), INVALID)],
    "hs_release_pages_t": [(dict(n_seqs=0), INVALID), (dict(done=0), INVALID), (dict(n_seqs=4097), SHAPE), (dict(workspace=P + 16), INVALID)],
    "hs_rope_table_t": [(dict(rotary_dim=8), SHAPE), (dict(rotary_dim=72), SHAPE), (dict(rotary_dim=272), SHAPE), (dict(max_position=0), INVALID),
                        (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID), (dict(base=0.0), INVALID), (dict(base=NAN), INVALID), (dict(factor=-1.0), INVALID),
                        (dict(turns_slow=32.0), INVALID), (dict(trained_positions=0), INVALID), (dict(magnitude=NAN), INVALID), (dict(table=P + 8), INVALID)],
    "hs_rope_cache_t": [(dict(n_tokens=0), INVALID), (dict(head_dim=24), SHAPE), (dict(head_dim=272), SHAPE), (dict(rotary_dim=80), SHAPE), (dict(rotary_dim=24), SHAPE),
                        (dict(q_stride=255), INVALID), (dict(q_stride=258), INVALID), (dict(k_stride=64), INVALID), (dict(q_out_stride=260), INVALID),
                        (dict(cache_type=0), INVALID), (dict(src_type=3), INVALID), (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(q=P + 8), INVALID),
                        (dict(q_out=P + 8), INVALID), (dict(kv_pool=P + 128), INVALID), (dict(max_position=0), INVALID)],
    "hs_paged_attention_t": [(dict(head_dim=96), SHAPE), (dict(n_kv_heads=3), SHAPE), (dict(n_q_heads=2048, q_stride=1 << 18, o_stride=1 << 18), SHAPE),
                             (dict(cap=-1.0), INVALID), (dict(cap=NAN), INVALID), (dict(cap=INF), INVALID), (dict(scale=INF), INVALID), (dict(scale=NAN), INVALID), (dict(window=-1), INVALID),
                             (dict(max_q_len=0), INVALID), (dict(tok_begin=0, max_q_len=2), INVALID), (dict(tok_begin=0, n_tokens=3), INVALID),
                             (dict(q_stride=252), INVALID), (dict(o_stride=260), INVALID), (dict(q=P + 8), INVALID), (dict(kv_pool=P + 64), INVALID),
                             (dict(type=0), INVALID), (dict(layer=2), INVALID), (dict(workspace=P + 64), INVALID), (dict(n_seqs=4097, n_tokens=4097), SHAPE),
                             (dict(n_seqs=4096, n_tokens=4096, max_pages_per_seq=32768, n_q_heads=16, q_stride=1024, o_stride=1024), SHAPE),
                             (dict(num_pages=1 << 25, n_layers=64), SHAPE)],
    "hs_token_logprobs_t": [(dict(n_rows=0), INVALID), (dict(vocab=0), INVALID), (dict(row_stride=99), INVALID), (dict(n_top=33), SHAPE), (dict(n_top=101), SHAPE),
                            (dict(n_top=-1), INVALID), (dict(top_ids=0), INVALID), (dict(scale=0.0), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID),
                            (dict(type=3), INVALID), (dict(logits=P + 2), INVALID), (dict(vocab=1 << 30, row_stride=1 << 30), SHAPE)],
}


@pytest.mark.parametrize("name", list(REFUSED))
def test_wrong_arguments_are_refused_before_a_device_is_needed(name):
    fn = C.CDLL(B.LIB_PATH)[ops.EXPORTS[list(STRUCTS).index(name)]]
    fn.argtypes, fn.restype = [C.c_char_p, C.c_int32, C.c_void_p], C.c_int
    assert fn(None, 8, None) == INVALID
    for change, want in REFUSED[name]:
        values = {f: P for f in fields(name)} | GOOD[name] | change
        assert set(change) <= set(fields(name))
        assert fn(STRUCTS[name].pack(*(values[f] for f in fields(name))), 8, None) == want, change


def test_python_refuses_tensors_of_the_wrong_kind():
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    ws, st = torch.zeros(ops.WORKSPACE_BYTES, dtype=torch.uint8), i32(1)
    good = dict(ctx_len=i32(3), q_len=i32(3), free_list=i32(9), free_count=i32(1), block_tables=torch.zeros(3, 4, dtype=torch.int32), kv_len=i32(3), tok_begin=i32(4),
                tok_seq=i32(7), tok_pos=i32(7), tok_slot=i32(7), free_count_out=i32(1), workspace=ws, status=st)
    for name, bad in [("q_len", i32(2)), ("tok_begin", i32(3)), ("tok_pos", i32(6)), ("kv_len", torch.zeros(3, dtype=torch.int64)), ("block_tables", i32(12)),
                      ("block_tables", torch.zeros(4, 3, dtype=torch.int32).T), ("workspace", ws[1:]), ("status", i32(2)), ("tok_slot", i32(14)[::2])]:
        with pytest.raises(ValueError, match=name):
            ops.step_tables(**(good | {name: bad}))
    with pytest.raises(ValueError, match="CUDA"):
        ops.step_tables(**good)

    pool = torch.zeros(2, 2, 5, 2, 16, 64, dtype=torch.bfloat16)
    rows = lambda h, dt=torch.bfloat16: torch.zeros(3, h, 64, dtype=dt)  # noqa: E731
    rope = dict(q=rows(4), k=rows(2), v=rows(2), tok_pos=i32(3), tok_slot=i32(3), table=torch.zeros(8, 32, 2), q_out=rows(4), kv_pool=pool, layer=0, status=st)
    for change in [dict(q=rows(4, torch.float64)), dict(k=rows(2, torch.float32)), dict(k=rows(3)), dict(q_out=rows(4, torch.float16)), dict(layer=2), dict(layer=-1),
                   dict(table=torch.zeros(8, 32, 3)), dict(q=torch.zeros(3, 64, 4, dtype=torch.bfloat16).transpose(1, 2)), dict(kv_pool=pool[:, :, :, :, :8]),
                   dict(kv_pool=pool[:, :, ::2]), dict(tok_slot=i32(4)), {}]:
        with pytest.raises(ValueError):
            ops.rope_cache(**(rope | change))

    att = dict(q=rows(4), kv_pool=pool, layer=0, block_tables=torch.zeros(3, 4, dtype=torch.int32), kv_len=i32(3), o=rows(4), workspace=ws, status=st)
    for change in [dict(q=rows(4, torch.float16)), dict(o=rows(4, torch.float32)), dict(o=rows(2)), dict(block_tables=torch.zeros(2, 4, dtype=torch.int32)),
                   dict(lse=torch.zeros(3, 3)), dict(tok_begin=i32(3)), dict(prefix_len=i32(2)), dict(slopes=torch.zeros(3)), {}]:
        with pytest.raises(ValueError):
            ops.paged_attention(**(att | change))

    lp = dict(logits=torch.zeros(3, 10), targets=i32(3), logprob=torch.zeros(3), workspace=ws, status=st)
    for change in [dict(logits=torch.zeros(3, 10, dtype=torch.float64)), dict(logits=torch.zeros(10, 3).T), dict(targets=torch.zeros(3, dtype=torch.int64)),
                   dict(top_ids=torch.zeros(3, 2, dtype=torch.int32)), dict(top_logprobs=torch.zeros(3, 2)),
                   dict(top_ids=torch.zeros(2, 2, dtype=torch.int32), top_logprobs=torch.zeros(3, 2)), dict(entropy=torch.zeros(4)), {}]:
        with pytest.raises(ValueError):
            ops.token_logprobs(**(lp | change))


def test_the_plain_tables_are_the_host_allocators():
    """Random steps and releases: the definition that the GPU tests use pops, pushes and numbers as the host's allocator does."""
    g = np.random.default_rng(3)
    n, num_pages, width, cap = 6, 40, 12, 64
    host = PageAllocator(num_pages, 16)
    ctx, tables = [0] * n, np.full((n, width), -1, dtype=np.int32)
    free_list, count = list(range(num_pages - 1, -1, -1)), num_pages
    refused = 0
    for _ in range(200):
        q = [int(x) for x in g.integers(0, 11, n)]
        q = [min(m, width * 16 - c) for m, c in zip(q, ctx)]
        status, out = ref.step_tables(ctx, q, free_list, count, tables, num_pages, cap)
        if status == "OUT_OF_PAGES":
            refused += 1
            need = sum(-(-(c + m) // 16) - -(-c // 16) for c, m in zip(ctx, q))
            assert need > len(host.free)
            done = [int(x) for x in g.integers(0, 2, n)]
            done[int(g.integers(0, n))] = 1
            for s in range(n):
                if done[s] and s in host.owned:
                    host.release(s)
            ctx, tables, free_list, count = ref.release_pages(done, ctx, tables, free_list, count)
        else:
            assert status is None
            grown = [host.alloc(s, c + m) for s, (c, m) in enumerate(zip(ctx, q))]
            seq, pos, slot = plan_tokens(q, ctx, out["block_tables"], 16)
            total = sum(q)
            assert list(seq) == out["tok_seq"][:total] and list(pos) == out["tok_pos"][:total] and list(slot) == out["tok_slot"][:total]
            ctx, tables, count = out["kv_len"], out["block_tables"], out["free_count"]
            assert [list(t[:len(p)]) for t, p in zip(tables, grown)] == grown
        assert free_list[:count] == host.free
    assert refused > 3
