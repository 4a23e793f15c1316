"""CPU-only checks of the operators of horizonserve_beams.h: the header, the library and the packed structs agree, wrong arguments are refused on the
host before any GPU is asked for, and the plain definitions of the GPU tests keep their own invariants."""
import ctypes as C
import os
import re
import struct
import subprocess
from collections import Counter

import numpy as np
import pytest
import torch

import beam_ref as ref
from paper_2608_01785_b200 import binding as B
from paper_2608_01785_b200 import device_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "horizonserve_beams.h")
# The description structs as packed words ("i" int32, "q" int64, "P" pointer, "f"), in the order of ops.BEAM_EXPORTS.
STRUCTS = {name: struct.Struct(fmt) for name, fmt in {
    "hs_beam_select_t": "@6iPq3Pf7P", "hs_fork_pages_t": "@3i11P", "hs_copy_pages_t": "@6i5P", "hs_compact_pages_t": "@5i9P",
    "hs_shared_attention_t": "@10iPq6P2fPq3P"}.items()}


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def fields(name):
    """Member names of a struct of the header, in order."""
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text()).group(1)
    return [re.findall(r"\w+", part)[-1] for line in body.split(";") if line.strip() for part in line.split(",")]


def offsets(fmt):
    """Byte offset of every member of a struct format."""
    codes = [c for n, c in re.findall(r"(\d*)([a-zA-Z])", fmt[1:]) for _ in range(int(n or 1))]
    return [(struct.calcsize("@" + "".join(codes[:i]) + "0" + c), struct.calcsize("@" + c)) for i, c in enumerate(codes)]


def test_every_declared_operator_is_exported_and_bound():
    names = re.findall(r"\b(hs_op_[a-z0-9_]+)\s*\(", text())
    assert sorted(names) == sorted(ops.BEAM_EXPORTS) and len(names) == len(set(names)) == len(STRUCTS)
    for n in names:
        assert hasattr(B.lib(), n), n


@pytest.mark.parametrize("compiler", ["gcc", "g++"])
def test_packed_structs_are_the_headers(tmp_path, compiler):
    lines = []
    for name in STRUCTS:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu %zu\\n", offsetof({name}, {f}), sizeof((({name} *)0)->{f}));' for f in fields(name)]
    src = tmp_path / ("m.c" if compiler == "gcc" else "m.cpp")
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"horizonserve_beams.h\"\nint main(void) {\n" + "\n".join(lines)
                   + '\nprintf("%d\\n", HS_MAX_BEAMS);\nreturn 0;\n}\n')
    exe = str(tmp_path / "m")
    subprocess.run([compiler, "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines()
    want = []
    for name, packed in STRUCTS.items():
        of = offsets(packed.format)
        assert len(of) == len(fields(name)), name
        want.append(str((packed.size + 7) // 8 * 8))
        want += [f"{o} {s}" for o, s in of]
    assert got == want + [str(ops.MAX_BEAMS)]


P = 1 << 20        # an address that is aligned for everything; no call below gets as far as using it
GOOD = {
    "hs_beam_select_t": dict(n_requests=3, n_beams=4, vocab=100, type=0, n_out=8, end_token=2, row_stride=100, scale=1.0),
    "hs_fork_pages_t": dict(n_rows=4, max_pages_per_seq=8, num_pages=32),
    "hs_copy_pages_t": dict(n_copies=4, type=1, n_layers=2, num_pages=32, n_kv_heads=2, head_dim=64),
    "hs_compact_pages_t": dict(n_rows=4, max_pages_per_seq=8, num_pages=32, n_keep=16, max_copies=16),
    "hs_shared_attention_t": dict(n_seqs=4, n_groups=2, n_q_heads=4, n_kv_heads=2, head_dim=64, type=1, n_layers=2, layer=1, num_pages=32, max_pages_per_seq=8,
                                  q_stride=256, scale=0.125, cap=0.0, o_stride=256),
}
INF, NAN = float("inf"), float("nan")
INVALID, SHAPE = B.HS_ERR_INVALID_ARG, B.HS_ERR_UNSUPPORTED_SHAPE
REFUSED = {
    "hs_beam_select_t": [(dict(n_requests=0), INVALID), (dict(n_beams=0), INVALID), (dict(vocab=0), INVALID), (dict(n_out=0), INVALID), (dict(row_stride=99), INVALID),
                         (dict(n_beams=33), SHAPE), (dict(n_out=33), SHAPE), (dict(n_requests=4097), SHAPE), (dict(n_requests=4096, n_beams=17), SHAPE),
                         (dict(vocab=1 << 30, row_stride=1 << 30), SHAPE), (dict(type=3), INVALID), (dict(logits=P + 2), INVALID), (dict(logits=P + 1, type=1), INVALID),
                         (dict(scale=0.0), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(scores=0), INVALID), (dict(out_score=0), INVALID),
                         (dict(out_parent=0), INVALID), (dict(out_token=0), INVALID), (dict(workspace=P + 64), INVALID), (dict(status=0), INVALID)],
    "hs_fork_pages_t": [(dict(n_rows=0), INVALID), (dict(max_pages_per_seq=0), INVALID), (dict(num_pages=0), INVALID), (dict(parent=0), INVALID), (dict(shares=0), INVALID),
                        (dict(copy_len=0), INVALID), (dict(workspace=P + 64), INVALID), (dict(n_rows=4097), SHAPE), (dict(n_rows=4096, max_pages_per_seq=32769), SHAPE),
                        (dict(num_pages=(1 << 24) + 1), SHAPE)],
    "hs_copy_pages_t": [(dict(n_copies=0), INVALID), (dict(type=0), INVALID), (dict(src=0), INVALID), (dict(kv_pool=P + 128), INVALID), (dict(n_layers=0), INVALID),
                        (dict(head_dim=260), SHAPE), (dict(head_dim=12), SHAPE), (dict(n_copies=(1 << 21) + 1), SHAPE), (dict(n_copies=1 << 21, n_layers=256), SHAPE),
                        (dict(num_pages=1 << 27), SHAPE)],
    "hs_compact_pages_t": [(dict(n_rows=0), INVALID), (dict(n_keep=-1), INVALID), (dict(n_keep=33), INVALID), (dict(max_copies=-1), INVALID), (dict(copy_src=0), INVALID),
                           (dict(free_count=0), INVALID), (dict(workspace=P + 64), INVALID), (dict(n_rows=4097), SHAPE), (dict(num_pages=(1 << 21) + 1), SHAPE)],
    "hs_shared_attention_t": [(dict(n_groups=0), INVALID), (dict(n_groups=5), INVALID), (dict(n_seqs=0), INVALID), (dict(head_dim=96), SHAPE), (dict(n_kv_heads=3), SHAPE),
                              (dict(n_q_heads=2048, q_stride=1 << 18, o_stride=1 << 18), SHAPE), (dict(cap=-1.0), INVALID), (dict(cap=NAN), INVALID), (dict(cap=INF), INVALID),
                              (dict(scale=INF), INVALID), (dict(scale=NAN), INVALID), (dict(q_stride=252), INVALID), (dict(o_stride=260), INVALID), (dict(q=P + 8), INVALID),
                              (dict(kv_pool=P + 64), INVALID), (dict(type=0), INVALID), (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(workspace=P + 64), INVALID),
                              (dict(group_begin=0), INVALID), (dict(shared_len=0), INVALID), (dict(n_seqs=2049), SHAPE), (dict(n_seqs=2048, max_pages_per_seq=32769), SHAPE),
                              (dict(n_seqs=2048, max_pages_per_seq=32768, n_q_heads=16, q_stride=1024, o_stride=1024), SHAPE),
                              (dict(num_pages=1 << 25, n_layers=64), SHAPE)],
}


@pytest.mark.parametrize("name", list(REFUSED))
def test_wrong_arguments_are_refused_before_a_device_is_needed(name):
    fn = C.CDLL(B.LIB_PATH)[ops.BEAM_EXPORTS[list(STRUCTS).index(name)]]
    fn.argtypes, fn.restype = [C.c_char_p, C.c_int32, C.c_void_p], C.c_int
    assert fn(None, 8, None) == INVALID
    for change, want in REFUSED[name]:
        values = {f: P for f in fields(name)} | GOOD[name] | change
        assert set(change) <= set(fields(name))
        assert fn(STRUCTS[name].pack(*(values[f] for f in fields(name))), 8, None) == want, change


def test_python_refuses_tensors_of_the_wrong_kind():
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    f32 = lambda *n: torch.zeros(*n)  # noqa: E731
    ws, st = torch.zeros(ops.WORKSPACE_BYTES, dtype=torch.uint8), i32(1)
    calls = {
        ops.beam_select: (dict(logits=f32(6, 50), scores=f32(3, 2), out_score=f32(3, 4), out_parent=i32(3, 4), out_token=i32(3, 4), workspace=ws, status=st),
                          [dict(logits=f32(6, 50).double()), dict(logits=f32(50, 6).T), dict(scores=f32(6)), dict(scores=f32(2, 2)), dict(scores=f32(3, 2).double()),
                           dict(out_score=f32(2, 4)), dict(out_parent=i32(3, 5)), dict(out_token=f32(3, 4)), dict(done=i32(3, 3)), dict(weight=f32(5)), dict(out_done=i32(3, 2)),
                           dict(lse=f32(3)), dict(workspace=ws[1:]), dict(end_token=1 << 31)]),
        ops.fork_pages: (dict(parent=i32(4), ctx_len=i32(4), block_tables=i32(4, 3), shares=i32(9), free_list=i32(9), free_count=i32(1), copy_src=i32(4), copy_dst=i32(4),
                              copy_len=i32(4), workspace=ws, status=st),
                         [dict(ctx_len=i32(3)), dict(block_tables=i32(3, 4)), dict(shares=i32(8)), dict(free_count=i32(2)), dict(copy_src=i32(3)), dict(copy_len=f32(4)),
                          dict(parent=i32(8)[::2])]),
        ops.copy_pages: (dict(kv_pool=torch.zeros(2, 2, 5, 2, 16, 64, dtype=torch.bfloat16), src=i32(3), dst=i32(3), status=st),
                         [dict(kv_pool=f32(2, 2, 5, 2, 16, 64)), dict(kv_pool=torch.zeros(0, 2, 5, 2, 16, 64, dtype=torch.bfloat16)), dict(dst=i32(2)), dict(length=i32(2)),
                          dict(src=f32(3)), dict(kv_pool=torch.zeros(2, 2, 10, 2, 16, 64, dtype=torch.bfloat16)[:, :, ::2])]),
        ops.compact_pages: (dict(n_keep=4, ctx_len=i32(2), block_tables=i32(2, 3), shares=i32(9), free_list=i32(9), free_count=i32(1), copy_src=i32(5), copy_dst=i32(5),
                                 workspace=ws, status=st),
                            [dict(shares=i32(8)), dict(copy_dst=i32(4)), dict(block_tables=i32(3, 3)), dict(n_keep="4"), dict(free_count=f32(1))]),
        ops.shared_attention: (dict(q=torch.zeros(4, 4, 64, dtype=torch.float16), kv_pool=torch.zeros(2, 2, 5, 2, 16, 64, dtype=torch.float16), layer=1, block_tables=i32(4, 3),
                                    kv_len=i32(4), group_begin=i32(3), shared_len=i32(2), o=torch.zeros(4, 4, 64, dtype=torch.float16), workspace=ws, status=st),
                               [dict(q=torch.zeros(4, 4, 64, dtype=torch.bfloat16)), dict(q=torch.zeros(4, 256, dtype=torch.float16)), dict(o=torch.zeros(4, 2, 64, dtype=torch.float16)),
                                dict(kv_len=i32(3)), dict(group_begin=i32(2)), dict(layer=2), dict(lse=f32(4, 3)), dict(slopes=f32(2)), dict(block_tables=i32(3, 3))]),
    }
    for fn, (good, changes) in calls.items():
        for change in changes:
            with pytest.raises((ValueError, TypeError)):
                fn(**(good | change))
        with pytest.raises(ValueError, match="CUDA"):
            fn(**good)


def test_the_plain_fork_keeps_its_books():
    """Random forks, growth and ends: a page is held by as many rows as its count says, and every page is either held or free, once."""
    rng = np.random.default_rng(4)
    n, width, num_pages = 6, 6, 60
    ctx, tables, shares = [0] * n, np.full((n, width), -1, dtype=np.int32), [0] * num_pages
    free, count = list(rng.permutation(num_pages)), num_pages
    ends = refused = 0
    for step in range(300):
        for i in range(n):                               # rows grow as hs_op_step_tables lets them
            more = int(rng.integers(0, 9))
            if ctx[i] + more > width * 16:
                continue
            need = ref.pages(ctx[i] + more) - ref.pages(ctx[i])
            if need > count:
                continue
            for p in range(need):
                count -= 1
                tables[i, ref.pages(ctx[i]) + p] = free[count]
            ctx[i] += more
        parent = [int(x) for x in rng.integers(-1, n, n)] if step % 3 else [int(x) for x in rng.permutation(n)]
        status, out = ref.fork(parent, ctx, tables, shares, free, count, num_pages)
        if status is not None:
            assert status == "OUT_OF_PAGES"
            refused += 1
            continue
        want = [ctx[p] if p >= 0 else 0 for p in parent]
        assert out["ctx_len"] == want
        for i, p in enumerate(parent):
            if p >= 0:
                whole = ctx[p] // 16
                assert (out["block_tables"][i, :whole] == tables[p, :whole]).all()
                if out["copy_src"][i] >= 0:
                    assert out["copy_src"][i] == tables[p, whole] and out["copy_dst"][i] == out["block_tables"][i, whole] and out["copy_len"][i] == ctx[p] % 16
        ends += parent.count(-1)
        ctx, tables, shares, free, count = out["ctx_len"], out["block_tables"], out["shares"], out["free_list"], out["free_count"]
        held = Counter(int(tables[i, c]) for i in range(n) for c in range(ref.pages(ctx[i])))
        assert all((tables[i, ref.pages(ctx[i]):] == -1).all() for i in range(n))
        assert set(held) | set(free[:count]) == set(range(num_pages)) and len(held) + count == num_pages and len(set(free[:count])) == count
        assert all(shares[p] == held[p] - 1 for p in held) and all(shares[p] == 0 for p in free[:count])
        tails = [int(tables[i, ctx[i] // 16]) for i in range(n) if ctx[i] % 16]
        assert len(set(tails)) == len(tails) and all(held[p] == 1 for p in tails)
    assert ends > 50 and refused < 250


def test_the_plain_compaction_keeps_what_rows_hold():
    rng = np.random.default_rng(5)
    for _ in range(50):
        ctx, tables, shares, free, num_pages = ref.shared_rows(rng, 3, 4, [int(x) for x in rng.integers(0, 90, 3)], 30)
        pad = free + [0] * (num_pages - len(free))
        keep = num_pages - int(rng.integers(0, 30))
        status, out = ref.compact(keep, ctx, tables, shares, pad, len(free), num_pages, num_pages)
        assert status is None
        to = {a: b for a, b in zip(out["copy_src"], out["copy_dst"]) if a >= 0}
        assert all(int(b) == to.get(int(a), int(a)) for a, b in zip(tables.ravel(), out["block_tables"].ravel()))
        held = {int(x) for x in out["block_tables"].ravel() if x >= 0}
        assert all(p < keep for p in held) and held | set(out["free_list"][:len(free)]) == set(range(num_pages))
        assert out["free_list"][:num_pages - keep] == list(range(num_pages - 1, keep - 1, -1))
        assert out["free_list"][:len(free)] == sorted(out["free_list"][:len(free)], reverse=True)
