"""Windows and drafted trees on the paged cache where the ways of computing them meet their
limits: many rows, split and shared-out caches, offsets past 32 bits, captured calls."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import DT, FMT, TORCH, Pool, attention_errors, dev, i32, offsets, rnd
from test_gpu_paged_loop import BIG, LAYOUT, Append, _tree_case, _tree_look, _window_look, _workspace, tree, window

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]


MANY_ROWS = [
    # lens, rows, group, heads, page: many rows of few sequences, whose caches are cut; ragged
    # ones; more sequences than are shared out; lengths and rows around tiles and blocks
    ([9000, 100, 5000, 0], [40, 70, 33, 5], 4, 1, 64),
    ([17000], [70], 1, 2, 32),
    ([5000, 4900, 16], [130, 7, 16], 1, 1, 16),
    ([64, 65, 63, 128, 129, 16, 15, 1], [33, 32, 31, 64, 65, 16, 15, 1], 4, 2, 16),
    ([20] * 290, [20] * 290, 4, 1, 32),
    ([333, 4097], [128, 129], 1, 2, 256),
    ([2049, 700, 4200], [300, 500, 257], 1, 1, 128),
    ([900], [25], 16, 1, 64),
    # enough blocks of 128 rows to go by them: caches cut in equal parts, shared out, ragged, blocks of
    # more than 64 rows
    ([1700], [70], 1, 128, 32),
    ([3300, 100, 1000], [66, 70, 5], 1, 43, 64),
    ([64, 65, 63, 128, 129, 16, 15, 1], [33, 32, 31, 64, 65, 16, 15, 1], 4, 6, 16),
    ([1049, 700], [300, 257], 1, 22, 16),
]


@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", MANY_ROWS, ids=lambda c: f"n{max(c[0])}r{sum(c[1])}g{c[2]}h{c[3]}b{len(c[0])}")
def test_many_rows(case, fmt, dh):
    say(f"paged masks, many rows {case[0][:4]} {case[1][:4]} {fmt} {dh}")
    lens, rows, group, H, page = case
    rng = np.random.default_rng(dh + len(lens))
    pool = Pool(fmt, lens, H, dh, page, seed=1)
    total = sum(rows)
    q = rnd(2 * rng.standard_normal((total, H * group * dh)), "bf16")
    d = dev(q, torch.bfloat16)
    t = np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)])
    size = max(2, max(lens) // 3)
    got = window(pool, d, rows, group, "bf16", t, size, 70).double().cpu().numpy()
    assert attention_errors(pool, got, q, rows, group, "bf16", _window_look(pool, rows, t, size, 70)) <= 1
    words = 3
    ctx, mask = _tree_case(lens, rows, words, rng)
    got = tree(pool, d, rows, group, "bf16", ctx, mask).double().cpu().numpy()
    assert attention_errors(pool, got, q, rows, group, "bf16", _tree_look(pool, rows, ctx, mask)) <= 1


@pytest.mark.parametrize("rows,group", [(1, 1), (20, 1), (100, 1), (40, 4)])
def test_rows_in_any_order(rows, group):
    """Rows that stand anywhere see what they see in order."""
    say(f"paged window, order of rows {rows} {group}")
    rng = np.random.default_rng(rows)
    pool = Pool("e4m3", [4000, 1000], 1, 128, 64, seed=1)
    q = rnd(rng.standard_normal((2 * rows, group * 128)), "bf16")
    t = np.concatenate([rng.integers(0, n, rows) for n in (4000, 1000)])
    got = window(pool, dev(q, torch.bfloat16), [rows] * 2, group, "bf16", t, 200, 9).double().cpu().numpy()
    assert attention_errors(pool, got, q, [rows] * 2, group, "bf16", _window_look(pool, [rows] * 2, t, 200, 9)) <= 1


@pytest.mark.parametrize("rows", [3, 130])
def test_equal_rows_need_no_offsets(rows):
    say(f"paged masks without offsets {rows}")
    rng = np.random.default_rng(1)
    pool = Pool("int8", [700, 50], 2, 64, 16, seed=1)
    q = dev(rnd(rng.standard_normal((2 * rows, 128)), "bf16"), torch.bfloat16)
    t = np.arange(2 * rows)
    assert torch.equal(window(pool, q, [rows] * 2, 1, "bf16", t, 33, 2), window(pool, q, [rows] * 2, 1, "bf16", t, 33, 2, off=None))
    mask = rng.integers(0, 2 ** 32, (2 * rows, 2), dtype=np.uint32)
    assert torch.equal(tree(pool, q, [rows] * 2, 1, "bf16", [600, 3], mask), tree(pool, q, [rows] * 2, 1, "bf16", [600, 3], mask, off=None))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows,H", [(2, 1), (100, 1), (100, 64)])
def test_queries_that_are_not_finite_stay_among_themselves(fmt, rows, H):
    say(f"paged masks, NaN queries {fmt} {rows} {H}")
    rng = np.random.default_rng(1)
    pool = Pool(fmt, [300], H, 64, 16, seed=1)
    q = rnd(rng.standard_normal((rows, H * 128)), "bf16")
    q[1, 3], q[0, 70] = np.nan, np.inf
    t = np.full(rows, 250)
    for got in (window(pool, dev(q, torch.bfloat16), [rows], 2, "bf16", t, 100, 3),
                tree(pool, dev(q, torch.bfloat16), [rows], 2, "bf16", [200], np.full((rows, 1), 5, np.uint32))):
        g = got.double().cpu().numpy().reshape(rows, 2 * H, 64)
        bad = np.zeros((rows, 2 * H), bool)
        bad[1, 0] = bad[0, 1] = True
        assert np.isnan(g[bad]).all() and np.isfinite(g[~bad]).all()


def test_lengths_are_cut():
    """len_max below a length, and lengths past the page table, for few and many rows."""
    say("paged masks, cut lengths")
    rng = np.random.default_rng(4)
    for rows, H in ((4, 1), (90, 1), (90, 64)):
        pool = Pool("bf16", [200, 90], H, 64, 16, seed=1, width_extra=0)
        q = rnd(rng.standard_normal((2 * rows, H * 64)), "bf16")
        d = dev(q, torch.bfloat16)
        t = np.arange(2 * rows) % rows + 50
        mask = rng.integers(0, 2 ** 32, (2 * rows, 7), dtype=np.uint32)
        for lens, len_max, seen in (([200, 90], 100, [100, 90]), ([BIG, 90], 208, [208, 90])):
            pool.lens = [200, 90]
            pool.dlens = i32(lens)
            if seen[0] == 208:  # the last page's slots behind token 199
                pool.dk.nan_to_num_(0.5)
                pool.dv.nan_to_num_(0.5)
            got = (window(pool, d, [rows] * 2, 1, "bf16", t, 60, 5, len_max=len_max), tree(pool, d, [rows] * 2, 1, "bf16", [10, 80], mask, len_max=len_max))
            pool.lens = seen
            for g, look in zip(got, (_window_look(pool, [rows] * 2, t, 60, 5), _tree_look(pool, [rows] * 2, [10, 80], mask))):
                assert attention_errors(pool, g.double().cpu().numpy(), q, [rows] * 2, 1, "bf16", look) <= 1


@pytest.mark.parametrize("fmt,dh,rows,H", [("e4m3", 128, 80, 8), ("bf16", 80, 80, 32), ("int8", 64, 3, 1), ("bf16", 128, 70, 1)])
def test_captured_calls_replay(fmt, dh, rows, H):
    """Both attentions captured, with split caches and their joins, replayed on new queries and
    lengths with eager calls between."""
    say(f"paged masks captured {fmt} {dh} {rows} {H}")
    lens = [9000, 40]
    pool = Pool(fmt, lens, H, dh, 64, seed=1)
    group, total, len_max = 2, 2 * rows, 9000
    heads = group * H
    D = heads * dh
    n1 = binding.paged_attention_window_workspace_bytes(pool.cache, 2, total, rows, heads, len_max, 6000, 4)
    n2 = binding.paged_attention_tree_workspace_bytes(pool.cache, 2, total, rows, heads, len_max)
    assert n1 and n2
    q, o1, o2 = (torch.zeros(total, D, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    off, t, ctx = i32(offsets([rows, rows])), i32(np.zeros(total)), i32([0, 0])
    mask = torch.zeros(total, 3, dtype=torch.int32, device="cuda")
    dl = i32(lens)

    def run(ws, o1, o2, stream):
        binding.paged_attention_window(pool.cache, 0, pool.dtable, pool.width, dl, len_max, 2, q, D, t, off, total, rows, heads,
                                       DT["bf16"], 6000, 4, o1, ws[0], n1, stream=stream)
        binding.paged_attention_tree(pool.cache, 0, pool.dtable, pool.width, dl, len_max, 2, q, D, off, total, rows, heads, DT["bf16"],
                                     ctx, mask, 3, o2, ws[1], n2, stream=stream)

    ws, we = [[_workspace(n) for n in (n1, n2)] for _ in range(2)]
    e1, e2 = torch.zeros_like(o1), torch.zeros_like(o2)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run(ws, o1, o2, side)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            run(ws, o1, o2, torch.cuda.current_stream())
    for i in range(4):
        rng = np.random.default_rng(i)
        n = [[9000, 40], [8999, 0], [500, 33], [7000, 1]][i]
        q.copy_(dev(rnd(rng.standard_normal((total, D)), "bf16"), torch.bfloat16))
        t.copy_(i32(np.concatenate([np.arange(rows) + max(0, x - rows) for x in n])))
        ctx.copy_(i32([max(0, x - 80) for x in n]))
        mask.copy_(i32(rng.integers(-2 ** 31, 2 ** 31, (total, 3))))
        dl.copy_(i32(n))
        for x in (o1, o2, e1, e2):
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        run(we, e1, e2, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(e1, o1) and torch.equal(e2, o2) and e1.isfinite().all() and e2.isfinite().all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,H", [(64, 64), (80, 64), (128, 16)])
def test_masked_places_count_nothing_in_many_rows(dh, H, fmt):
    """Infinities and NaN in masked keys and values, in tiles that rows see a part of, by blocks
    of many rows; an infinite value that some rows see reaches its channel there alone."""
    say(f"paged masked infinities, many rows {fmt} {dh}")
    rng = np.random.default_rng(3)
    n, rows = 400, 150
    pool = Pool(fmt, [n], H, dh, 16, seed=4)
    bad = [3, 150, 151, 249, n - 1]
    for j, x in zip(bad, (np.nan, np.inf, -np.inf, np.nan, np.inf)):
        page, slot = pool.table[0][j // 16], j % 16
        for d, e in ((pool.dk, pool.dke), (pool.dv, pool.dve)):
            if fmt == "bf16":
                d[0, page, 1, slot, 5:9] = x
            else:
                d[0, page, 1, slot] = 0x7F if fmt == "e4m3" else 0
                e[0, page, 1, slot] = 255
    group = 2 if dh == 128 else 1
    q = rnd(rng.standard_normal((rows, H * group * dh)), "bf16")
    t = np.array([250 + 20 + 119 * i // rows for i in range(rows)])
    t = np.where(t == n - 1, n - 2, t)
    got = window(pool, dev(q, torch.bfloat16), [rows], group, "bf16", t, 20, 3).double().cpu().numpy()
    assert np.isfinite(got).all()
    assert attention_errors(pool, got, q, [rows], group, "bf16", _window_look(pool, [rows], t, 20, 3)) <= 1
    mask = rng.integers(0, 2 ** 32, (rows, 13), dtype=np.uint32)
    for j in bad:
        mask[:, (j - 3) // 32] &= ~np.uint32(1 << ((j - 3) % 32))
    got = tree(pool, dev(q, torch.bfloat16), [rows], group, "bf16", [3], mask).double().cpu().numpy()
    assert np.isfinite(got).all()
    assert attention_errors(pool, got, q, [rows], group, "bf16", _tree_look(pool, [rows], [3], mask)) <= 1
    if fmt != "bf16":
        return
    pool = Pool(fmt, [n], H, dh, 16, seed=4)
    page, slot = pool.table[0][100 // 16], 100 % 16
    pool.dv[0, page, 0, slot, 9] = float("inf")
    t = np.array([100 + (i % 2) * 60 for i in range(rows)])
    o = window(pool, dev(q, torch.bfloat16), [rows], group, "bf16", t, 30, 0).double().cpu().numpy().reshape(rows, H, group, dh)
    want = np.zeros(o.shape, bool)
    want[::2, 0, :, 9] = True
    assert np.array_equal(np.isinf(o), want) and not np.isnan(o).any()


@pytest.mark.parametrize("dh,H", [(64, 64), (128, 16)])
def test_layout_of_many_rows(dh, H):
    """Rows of no sequence are left alone, pages that no row sees may be gone, by blocks of many rows."""
    say(f"paged masks, layout of many rows {dh}")
    rng = np.random.default_rng(2)
    lens, rows, before, extra = [300, 20, 600], [70, 1, 140], 2, 3
    total = sum(rows)
    pool = Pool("bf16", lens, H, dh, 32, seed=7)
    q = rnd(rng.standard_normal((total, H * dh)), "bf16")
    buf = torch.full((before + total + extra, H * dh + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[before:before + total, 8:8 + H * dh] = dev(q, torch.bfloat16)
    off = i32(offsets(rows) + before)
    t = np.concatenate([[BIG] * before] + [n - 1 - np.arange(r) for n, r in zip(lens, rows)] + [[5] * extra])
    mask = rng.integers(0, 2 ** 32, (before + total + extra, 2), dtype=np.uint32)
    ctx = [max(0, n - r) for n, r in zip(lens, rows)]
    for kind in ("tree", "window"):
        o = torch.full((before + total + extra, H * dh), 7.0, dtype=torch.bfloat16, device="cuda")
        if kind == "window":
            seen, pool.table = pool.table, pool.table.copy()
            pool.table[2, 1:(600 - 140 - 77) // 32] = -1
            pool.dtable = i32(pool.table)
            window(pool, buf[:, 8:], rows, 1, "bf16", t, 77, 5, o=o, off=off, q_stride=H * dh + 24)
            pool.table = seen
            look = _window_look(pool, rows, t[before:before + total], 77, 5)
        else:
            tree(pool, buf[:, 8:], rows, 1, "bf16", ctx, mask, o=o, off=off, q_stride=H * dh + 24)
            look = _tree_look(pool, rows, ctx, mask[before:before + total])
        assert (o[:before] == 7).all() and (o[before + total:] == 7).all()
        got = o[before:before + total].double().cpu().numpy()
        assert attention_errors(pool, got, q, rows, 1, "bf16", look) <= 1


def test_rows_that_see_nothing_among_many():
    """Empty masks and windows in blocks of many rows, on cut caches and on others."""
    say("paged masks that leave nothing, many rows")
    pool = Pool("e4m3", [5000, 40, 0], 16, 128, 16, seed=2)
    rows = [130, 70, 66]
    q = dev(np.ones((266, 16 * 128)), torch.bfloat16)
    t = np.full(266, -1)
    mask = np.zeros((266, 3), np.uint32)
    assert (window(pool, q, rows, 1, "bf16", t, 900, 9) == 0).all() and (tree(pool, q, rows, 1, "bf16", [0, 0, 0], mask) == 0).all()
    t[5], mask[129, 2] = 7000, 1
    one = window(pool, q, rows, 1, "bf16", t, 900, 3).cpu(), tree(pool, q, rows, 1, "bf16", [0, 0, 0], mask).cpu()
    for o, i in zip(one, (5, 129)):
        assert (o[i] != 0).any() and (o[[j for j in range(266) if j != i]] == 0).all()


def test_repeated_calls_are_equal():
    """Sums do not depend on the order in which workgroups run."""
    say("paged masks repeated")
    rng = np.random.default_rng(1)
    for rows, H in (([2, 2, 2], 2), ([90, 70, 50], 2), ([90, 70, 50], 8)):
        pool = Pool("e4m3", [9000, 3000, 77], H, 128, 64, seed=1)
        q = dev(rnd(rng.standard_normal((sum(rows), H * 2 * 128)), "bf16"), torch.bfloat16)
        mask = rng.integers(0, 2 ** 32, (sum(rows), 2), dtype=np.uint32)
        t = rng.integers(0, 9000, sum(rows))
        one = tree(pool, q, rows, 2, "bf16", [8950, 2990, 0], mask), window(pool, q, rows, 2, "bf16", t, 4000, 4)
        for _ in range(3):
            assert torch.equal(one[0], tree(pool, q, rows, 2, "bf16", [8950, 2990, 0], mask))
            assert torch.equal(one[1], window(pool, q, rows, 2, "bf16", t, 4000, 4))


@pytest.mark.parametrize("rows", [5, 90])
def test_widest_masks(rows):
    """64 words: 2048 drafted tokens, some of them past the length, some past the last word."""
    say(f"paged tree, widest masks {rows}")
    rng = np.random.default_rng(3)
    pool = Pool("bf16", [2500, 1200], 1, 64, 16, seed=1)
    q = rnd(rng.standard_normal((2 * rows, 64)), "bf16")
    mask = rng.integers(0, 2 ** 32, (2 * rows, 64), dtype=np.uint32)
    got = tree(pool, dev(q, torch.bfloat16), [rows] * 2, 1, "bf16", [100, 333], mask).double().cpu().numpy()
    assert attention_errors(pool, got, q, [rows] * 2, 1, "bf16", _tree_look(pool, [rows] * 2, [100, 333], mask)) <= 1


@pytest.mark.parametrize("fmt", ["int8", "bf16"])
def test_pool_past_32_bits(fmt):
    """Pages whose byte and element offsets pass 2^32: appended to, and seen by few and many rows."""
    say(f"paged loop, pool past 32 bits {fmt}")
    H, dh, page, n_pages = 8, 128, 64, 70000  # 4.59e9 elements
    es = 1 if fmt == "int8" else 2
    k = torch.empty(n_pages, H, page, dh * es, dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    ke, ve = (torch.empty(n_pages, H, page, dtype=torch.uint8, device="cuda") for _ in range(2)) if es == 1 else (None, None)
    cache = binding.paged_cache(1, n_pages, H, page, dh, FMT[fmt], k, v, ke, ve)
    pool = Pool(fmt, [4 * page], H, dh, page, seed=1)  # (of the same sizes, for the rows and the checks)
    pool.cache, pool.width = cache, 4
    pool.table = np.array([[n_pages - 1, 3, n_pages - 2, 65536]], np.int32)
    pool.dtable = i32(pool.table)
    n = 4 * page
    a = Append(pool, [n], 1, "bf16", seed=3)
    rot = binding.rotary(dh, LAYOUT["halves"], [0])
    a.call(i32(np.arange(n)), rot, None)
    want = [a.x[:, (w + 1) * H:(w + 2) * H] for w in range(2)]
    if es == 1:
        want = [ref.value(*ref.quantise(x, fmt)) for x in want]
    for rows in (1, n):
        t = np.arange(n - rows, n)
        q = a.q_out[n - rows:]
        mask = np.full((rows, 8), 0x55555555, np.uint32)
        for got, look in ((window(pool, q, [rows], 1, "bf16", t, 100, 4, q_stride=a.q_out.stride(0)), ref.window(t, n, 100, 4)),
                          (tree(pool, q, [rows], 1, "bf16", [50], mask, q_stride=a.q_out.stride(0)), ref.tree(mask, n, 50))):
            qq = q[:, 2 * dh:3 * dh].double().cpu().numpy()
            o, m, dl = ref.attention(qq, want[0][:, 2], want[1][:, 2], look)
            allow = 2.0 ** -8 * (np.abs(o) + m) + m * (2 * (dh + 8) * dl[:, None] + n + 64) * 2.0 ** -24
            assert (np.abs(got.double().cpu().numpy().reshape(rows, H, dh)[:, 2] - o) <= allow).all()


@pytest.mark.parametrize("fmt,dtype,H,group,dh", [("int8", "bf16", 6, 2, 64), ("bf16", "f32", 5, 1, 128), ("e4m3", "bf16", 4, 8, 80)])
def test_large_appends_are_small_ones_together(fmt, dtype, H, group, dh):
    """A call whose rows are loaded past the caches against calls of a few rows."""
    say(f"paged append large {fmt} {dtype} {dh}")
    per = int(64e6 / (2 if dtype == "bf16" else 4) / (12 * H * (group + 2) * dh)) + 1
    lens = [per] * 12
    big, small = (Pool(fmt, lens, H, dh, 64, seed=2) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    D, E = H * group * dh, H * dh
    n = sum(lens)
    buf = torch.randn(n, D + 2 * E, generator=g, device="cuda").to(TORCH[dtype])
    assert buf.numel() * buf.element_size() >= 64e6
    rot = binding.rotary(dh, LAYOUT["neighbours"], [7, 9, 4])
    pos = i32(np.stack([np.arange(n) % 1000, np.arange(n) // 7, -np.arange(n)]))
    idx = i32(np.concatenate([np.random.default_rng(b).permutation(x) for b, x in enumerate(lens)]))
    outs = []
    for pool, cuts in ((big, [(0, 12)]), (small, [(b, b + 1) for b in range(12)])):
        out = torch.zeros(n, D, dtype=TORCH[dtype], device="cuda")
        for lo, hi in cuts:
            step = n if hi - lo == 12 else 100
            for r in range(lo * per, hi * per, step):
                m = min(step, hi * per - r)
                x = buf[r:r + m]
                p = pos[:, r:r + m].contiguous()
                binding.paged_append(pool.cache, 0, pool.dtable[lo:hi].contiguous(), pool.width, hi - lo, idx[r:r + m].contiguous(), None,
                                     m, rot, p, x, H * group, x[:, D:], x[:, D + E:], D + 2 * E, DT[dtype], out[r:r + m], D)
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(*outs)
    for x, y in ((big.dk, small.dk), (big.dv, small.dv), (big.dke, small.dke), (big.dve, small.dve)):
        assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))
