"""The operators of horizonserve_beams.h at the ends of their arguments: offsets past 32 bits, the largest pools, the most rows, two calls that share a stream and
a workspace."""
import numpy as np
import pytest
import torch

from paper_2608_01785_b200 import device_ops as ops
from tests import beam_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(values):
    return torch.tensor(np.asarray(values, dtype=np.int32), device=DEV)


@pytest.fixture(scope="module")
def ws():
    return ops.workspace(DEV)


@pytest.fixture()
def status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def test_a_cache_of_more_than_four_gigabytes(ws, status):
    """The last pages of the last layer give what the same pages of a small cache give, bit for bit."""
    rng, layers, pages, hkv, dim = np.random.default_rng(1), 4, 20000, 8, 128
    big = torch.empty(layers, 2, pages, hkv, 16, dim, dtype=torch.bfloat16, device=DEV)
    assert big.numel() * 2 > 1 << 32
    tables, used = ref.grouped_tables(rng, [(100, [5, 40]), (33, [1, 20, 3])], 12)
    small = torch.randn(1, 2, used, hkv, 16, dim, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).bfloat16()
    first = pages - used
    big[-1, :, first:] = small[0]
    kv, q = i32([105, 140, 34, 53, 36]), torch.randn(5, 16, dim, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16()
    out = []
    for pool, offset in ((small, 0), (big, first)):
        o = torch.empty_like(q)
        ops.shared_attention(q, pool, pool.shape[0] - 1, i32(np.where(tables >= 0, tables + offset, -1)), kv, i32([0, 2, 5]), i32([100, 33]), o, ws, status)
        out.append(o)
    assert torch.equal(*out) and int(status) == 0
    # copies among them
    big[:, :, first:] = small
    src, dst = list(range(0, used - 1, 2)), list(range(1, used, 2))
    n = min(len(src), len(dst))
    ops.copy_pages(big, i32([first + p for p in src[:n]]), i32([first + p for p in dst[:n]]), status)
    want = small[0].clone()
    want[:, dst[:n]] = small[0][:, src[:n]]
    for layer in range(layers):
        assert torch.equal(big[layer, :, first:], want)
    assert int(status) == 0


def test_logits_whose_rows_are_far_apart(ws, status):
    rows, vocab, stride = 6, 30001, 450_000_001
    x = torch.randn(rows, vocab, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).bfloat16()
    far = torch.empty(stride * (rows - 1) + vocab, dtype=torch.bfloat16, device=DEV)
    view = far.as_strided((rows, vocab), (stride, 1))
    view.copy_(x)
    out = []
    for logits in (x, view):
        s = torch.zeros(2, 3, device=DEV)
        o = [torch.empty(2, 8, device=DEV), *(torch.empty(2, 8, dtype=torch.int32, device=DEV) for _ in range(2))]
        lse = torch.empty(rows, device=DEV)
        ops.beam_select(logits, s, *o, ws, status, lse=lse)
        out.append([*o, lse])
    for a, b in zip(*out):                                # (rows begin at other places of a tile: sums are rounded elsewhere)
        assert torch.equal(a, b) if a.dtype == torch.int32 else float((a - b).abs().max()) <= 1e-5
    assert int(status) == 0


@pytest.mark.parametrize("n,beams", [(1, 8), (512, 8), (128, 32)])
def test_rows_of_the_largest_pool_fork_as_those_of_a_small_one(n, beams, ws, status):
    rng = np.random.default_rng(n)
    ctx, tables, shares, free, num = ref.shared_rows(rng, n, beams, [int(x) for x in rng.integers(0, 90, n)], n * beams + 9)
    parent = [int(r * beams + rng.integers(0, beams)) if rng.random() < 0.95 else -1 for r in range(n) for _ in range(beams)]
    most, out = 1 << 24, []
    for pages in (num, most):
        at = pages - num
        t = [i32(parent), i32(ctx), i32(np.where(tables >= 0, tables + at, -1)), torch.zeros(pages, dtype=torch.int32, device=DEV),
             torch.full((pages,), -5, dtype=torch.int32, device=DEV), i32([len(free)]), *(torch.empty(n * beams, dtype=torch.int32, device=DEV) for _ in range(3))]
        t[3][at:] = i32(shares)
        t[4][:len(free)] = i32(free) + at
        ops.fork_pages(*t, ws, status)
        count = int(t[5])
        back = lambda x: torch.where(x >= 0, x - at, x)  # noqa: E731
        assert int(t[3][:at].abs().sum()) == 0 and bool((t[4][num:] == -5).all())
        out.append([t[1], back(t[2]), t[3][at:], back(t[4][:count]), t[5], back(t[6]), back(t[7]), t[8]])
    for a, b in zip(*out):
        assert torch.equal(a, b)
    assert int(status) == 0 and not bool(ws[-(2 << 20):].any()) and not bool(ws[:64 << 10].any())


@pytest.mark.parametrize("pages", [1 << 21, (1 << 21) - 37])
def test_the_largest_pool_that_is_compacted(pages, ws, status):
    rng, rows, width = np.random.default_rng(pages), 4096, 300
    name = rng.permutation(pages)
    ctx = rng.integers(0, width * 16 + 1, rows)
    owned = -(-ctx // 16)
    tables = np.full((rows, width), -1, dtype=np.int64)
    mine = np.arange(width)[None] < owned[:, None]
    tables[mine] = name[:int(owned.sum())]
    used = np.zeros(pages, dtype=bool)
    used[tables[mine]] = True
    free, keep = rng.permutation(np.nonzero(~used)[0]), int(pages * 0.7)
    shares = np.where(used, rng.integers(0, 5, pages), 0)
    src, dst = np.nonzero(used[keep:])[0] + keep, np.nonzero(~used[:keep])[0]
    moves = len(src)
    assert 0 < moves < len(dst)
    to = np.arange(pages)
    to[src] = dst[:moves]
    t = [i32(ctx), i32(tables), i32(shares), i32(np.concatenate([free, np.full(pages - len(free), -5)])), i32([len(free)]),
         *(torch.empty(pages - keep, dtype=torch.int32, device=DEV) for _ in range(2))]
    ops.compact_pages(keep, *t, ws, status)
    got = [x.cpu().numpy() for x in t]
    assert int(status) == 0
    assert np.array_equal(got[5], np.concatenate([src, np.full(pages - keep - moves, -1)])) and np.array_equal(got[6][:moves], dst[:moves])
    assert np.array_equal(got[1], np.where(mine, to[tables.clip(0)], -1))
    want = shares.copy()
    want[dst[:moves]], want[src] = shares[src], 0
    assert np.array_equal(got[2], want)
    rest = np.concatenate([dst[moves:], np.arange(keep, pages)])[::-1]
    assert np.array_equal(got[3][:len(rest)], rest) and bool((got[3][len(rest):] == -5).all()) and int(got[4][0]) == len(rest)
    assert not bool(ws[-(2 << 20):].any())


def test_calls_behind_one_another_share_a_workspace(ws, status):
    """Selections of different shapes, attention, forks and compactions on one stream without a pause give what each gives by itself."""
    g = torch.Generator(device=DEV).manual_seed(5)
    shapes = [(64, 8, 20000, 8), (1, 32, 152064, 32), (4096, 1, 33, 2), (3, 5, 7001, 5)]
    xs = [torch.randn(n * b, v, generator=g, device=DEV) for n, b, v, _ in shapes]

    def select(i):
        n, b, _, k = shapes[i]
        o = [torch.empty(n, k, device=DEV), *(torch.empty(n, k, dtype=torch.int32, device=DEV) for _ in range(2))]
        ops.beam_select(xs[i], torch.zeros(n, b, device=DEV), *o, ws, status)
        return o

    alone = []
    for i in range(4):
        alone.append(select(i))
        torch.cuda.synchronize()
    for _ in range(3):
        together = [select(i) for i in (0, 1, 2, 3, 2, 1, 0)]
        for got, i in zip(together, (0, 1, 2, 3, 2, 1, 0)):
            assert all(torch.equal(a, b) for a, b in zip(got, alone[i]))
    assert int(status) == 0


@pytest.mark.parametrize("groups,hq,hkv,dim,cap", [([(4000, [30] * 36)], 28, 4, 128, 0.0), ([(900, [5, 60, 17, 1]), (2000, [64] * 9), (16, [300, 40])] * 3, 16, 4, 64, 30.0),
                                                    ([(8000, [40, 1])], 4, 1, 128, 0.0), ([(1500 + 61 * g, [9 + g] * 8) for g in range(12)], 14, 2, 128, 50.0)])
def test_shared_attention_of_cut_tiles_time_after_time(groups, hq, hkv, dim, cap, ws, status):
    """Tiles cut between many shares, which one block or a few take one behind the other: every call leaves the bits and the control words of the first."""
    rng, g = np.random.default_rng(6), torch.Generator(device=DEV).manual_seed(6)
    kv = [s + n for s, own in groups for n in own]
    tables, pages = ref.grouped_tables(rng, groups, max(map(ref.pages, kv)) + 1)
    q = torch.randn(len(kv), hq, dim, generator=g, device=DEV).bfloat16()
    pool = torch.randn(1, 2, pages, hkv, 16, dim, generator=g, device=DEV).bfloat16()
    arguments = [pool, 0, i32(tables), i32(kv), i32(np.cumsum([0] + [len(own) for _, own in groups])), i32([s for s, _ in groups])]

    def call(budget):
        o, lse = torch.full_like(q, 77.0), torch.full((len(kv), hq), 55.0, device=DEV)
        ops.shared_attention(q, *arguments, o, ws, status, lse=lse, cap=cap, sm_budget=budget)
        return torch.cat([o.view(torch.int16).flatten().int(), lse.view(torch.int32).flatten()])

    first = call(None)
    for budget in (1, 2, 5, 9, 37, 74, 147):
        wrong = torch.zeros(1, dtype=torch.int64, device=DEV)
        for _ in range(200):
            wrong += (call(budget) != first).sum() + (ws[:64 << 10] != 0).sum()
        assert int(wrong) == 0, f"budget {budget}"
    assert int(status) == 0


def test_all_operators_behind_one_another_share_a_workspace(ws, status):
    """Attention of cut tiles, forks that free pages, compactions by three launches, selections of cut rows, copies: in mixed order on one stream and workspace, without a
    pause and at several budgets, each gives what it gives by itself."""
    rng, g = np.random.default_rng(7), torch.Generator(device=DEV).manual_seed(7)

    def selection(n, b, vocab, k):
        x = torch.randn(n * b, vocab, generator=g, device=DEV).bfloat16()

        def call(budget):
            out = [torch.empty(n, k, device=DEV), *(torch.empty(n, k, dtype=torch.int32, device=DEV) for _ in range(2))]
            ops.beam_select(x, torch.zeros(n, b, device=DEV), *out, ws, status, sm_budget=budget)
            return out
        return call

    def attention(groups, hq, hkv, dim):
        kv = [s + n for s, own in groups for n in own]
        tables, pages = ref.grouped_tables(rng, groups, max(map(ref.pages, kv)) + 1)
        q = torch.randn(len(kv), hq, dim, generator=g, device=DEV).bfloat16()
        pool = torch.randn(1, 2, pages, hkv, 16, dim, generator=g, device=DEV).bfloat16()
        rest = [i32(tables), i32(kv), i32(np.cumsum([0] + [len(own) for _, own in groups])), i32([s for s, _ in groups])]

        def call(budget):
            o, lse = torch.empty_like(q), torch.empty(len(kv), hq, device=DEV)
            ops.shared_attention(q, pool, 0, *rest, o, ws, status, lse=lse, sm_budget=budget)
            return [o, lse]
        return call

    def fork(n, beams, most):
        ctx, tables, shares, free, num = ref.shared_rows(rng, n, beams, [int(x) for x in rng.integers(20, most, n)], n * beams + 9)
        parent = [-1 if rng.random() < 0.3 else i // beams * beams + int(rng.integers(beams)) for i in range(n * beams)]
        given = [i32(x) for x in (parent, ctx, tables, shares, free + [0] * (num - len(free)), [len(free)])]

        def call(budget):
            out = [t.clone() for t in given] + [torch.empty(n * beams, dtype=torch.int32, device=DEV) for _ in range(3)]
            ops.fork_pages(*out, ws, status, sm_budget=budget)
            return out
        return call

    def compaction(spare):
        ctx, tables, shares, free, num = ref.shared_rows(rng, 20, 4, [int(x) for x in rng.integers(0, 700, 20)], spare)
        given = [i32(x) for x in (ctx, tables, shares, free + [0] * (num - len(free)), [len(free)])]

        def call(budget):
            out = [t.clone() for t in given] + [torch.empty(spare // 2, dtype=torch.int32, device=DEV) for _ in range(2)]
            ops.compact_pages(num - spare // 2, *out, ws, status, sm_budget=budget)
            return out
        return call

    def copies():
        pool, order = torch.randn(2, 2, 101, 2, 16, 64, generator=g, device=DEV).bfloat16(), rng.permutation(101)
        src, dst = i32(order[:50]), i32(order[50:100])

        def call(budget):
            out = pool.clone()
            ops.copy_pages(out, src, dst, status, sm_budget=budget)
            return [out]
        return call

    calls = [selection(64, 8, 20000, 8), selection(1, 32, 152064, 32), selection(3, 5, 7001, 5), attention([(3000, [30] * 20)], 28, 4, 128),
             attention([(900, [5, 60]), (40, [300, 1, 7])] * 4, 16, 4, 64), fork(40, 8, 300), fork(3, 2, 60), compaction(30000), compaction(9000), compaction(60), copies()]
    alone = []
    for call in calls:
        alone.append([t.clone() for t in call(None)])
        torch.cuda.synchronize()
    for budget in (None, 1, 20):
        order = np.concatenate([rng.permutation(len(calls)) for _ in range(6)])
        together = [(i, calls[i](budget)) for i in order]
        for i, got in together:
            assert all(torch.equal(a, b) for a, b in zip(got, alone[i])), (budget, i)
    assert int(status) == 0 and not bool(ws[:64 << 10].any()) and not bool(ws[-(2 << 20):].any())
