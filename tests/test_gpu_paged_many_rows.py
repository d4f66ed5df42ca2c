"""Windows and drafted trees by the kernel of many rows (csrc/paged_rows.h) on the GPU against
the float64 oracle: tokens in any order, calls without offsets, the widest masks, pools past
32 bits, and the tests of test_gpu_paged_loop_edges.py that are of either kernel, at sizes for this
one.  tests/test_paged_plan.py holds the sizes to that kernel."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import FMT, Pool, attention_errors, dev, i32, rnd
import test_gpu_paged_loop_edges as edges
from test_gpu_paged_loop import BIG, LAYOUT, Append, _tree_look, _window_look, tree, window

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]
DIMS = [64, 80, 128]
RAGGED = [300, 70, 0, 40, 129, 1, 128, 33]  # rows of 8 sequences: 24 blocks, most of them empty, for each key head
# lens, rows of each sequence, heads, group, page, window, sinks
ANY_ORDER = [
    ([700, 90, 5, 40, 300, 1, 513, 64], RAGGED, 24, 1, 16, 40, 9),
    ([1300, 64, 0, 65, 128, 700, 16, 33], RAGGED, 24, 1, 64, 500, 0),
    ([513, 1, 0, 600, 64, 100, 63, 90], [150, 33, 66, 0, 65, 64, 129, 1], 24, 2, 32, 1, 100),
    ([300, 2100, 17, 40, 90, 64, 128, 500], RAGGED, 24, 1, 128, BIG, 3),
]
EQUAL = dict(lens=[700, 50, 64, 0, 300, 129, 16, 400], rows=[130] * 8, heads=32, page=16)
WIDEST = dict(lens=[2500, 1200], rows=[140, 140], heads=64, page=16)
# format, channels, heads, query heads of each, page, pages
PAST = [("int8", 128, 16, 8, 64, 35000), ("bf16", 64, 64, 3, 16, 70000)]
PAST_ROWS = 384
CUT = dict(rows=[90, 90], heads=256)
NOTHING = dict(lens=[5000, 40, 0], rows=[130, 70, 66], heads=88)
# the tests of test_gpu_paged_loop_edges.py, with heads for blocks enough: their own arguments
MASKED = [(64, 256), (80, 256), (128, 128)]                    # dh, heads
LAYOUT_OF = [(64, 88), (80, 88), (128, 24)]                    # dh, heads
CAPTURED = [("e4m3", 64, 80, 40), ("bf16", 80, 80, 32), ("int8", 128, 80, 24), ("bf16", 128, 80, 8)]  # format, dh, rows, heads
QUERIES = (100, 256)                                           # rows, heads
MANY = [([3300, 100, 1000, 0, 64, 65, 17, 1], [300, 100, 70, 0, 64, 65, 17, 1], 1, 24, 64),
        ([64, 65, 63, 128, 129, 16, 15, 1], [33, 32, 31, 64, 65, 16, 15, 1], 4, 24, 16),
        ([590, 300], [300, 257], 1, 88, 16)]                  # as its MANY_ROWS
REPEATED = ([9000, 3000, 77], [90, 70, 50], 32)                # lens, rows, heads


def _sizes(look, fmt, dh, heads, lens, rows, group=1, window=1, sinks=0):
    return dict(dtype="bf16", fmt=fmt, dh=dh, seqs=len(rows), total=sum(rows), most=max(rows), heads=heads, group=group,
                len_max=max(lens), look=look, window=window, sinks=sinks)


def by_blocks():
    """Sizes of the calls below."""
    out = []

    def both(*args, **kw):
        out.append(_sizes("window", *args, **kw))
        out.append(_sizes("tree", *args, group=kw.get("group", 1)))
    for fmt in FORMATS:
        for dh in DIMS:
            out.extend(_sizes("window", fmt, dh, H, n, r, g, w, s) for n, r, H, g, _, w, s in ANY_ORDER)
            both(fmt, dh, EQUAL["heads"], EQUAL["lens"], EQUAL["rows"], window=33, sinks=2)
            out.append(_sizes("tree", fmt, dh, WIDEST["heads"], WIDEST["lens"], WIDEST["rows"]))
            both(fmt, dh, NOTHING["heads"], NOTHING["lens"], NOTHING["rows"], window=900, sinks=3)
            for n, r, g, H, _ in MANY:
                both(fmt, dh, H, n, r, group=g, window=max(2, max(n) // 3), sinks=70)
        for dh, H in MASKED:
            both(fmt, dh, H, [400], [150], group=2 if dh == 128 else 1, window=20, sinks=3)
        both(fmt, 64, QUERIES[1], [300], [QUERIES[0]], group=2, window=100, sinks=3)
    for len_max in (100, 208):
        both("bf16", 64, CUT["heads"], [len_max], CUT["rows"], window=60, sinks=5)
    for dh, H in LAYOUT_OF:
        both("bf16", dh, H, [300, 20, 600], [70, 1, 140], window=77, sinks=5)
    for fmt, dh, rows, H in CAPTURED:
        both(fmt, dh, H, [9000, 40], [rows] * 2, group=2, window=6000, sinks=4)
    both("e4m3", 128, REPEATED[2], REPEATED[0], REPEATED[1], group=2, window=4000, sinks=4)
    for fmt, dh, H, g, page, _ in PAST:
        both(fmt, dh, H, [PAST_ROWS], [PAST_ROWS], group=g, window=100, sinks=4)
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh", DIMS)
@pytest.mark.parametrize("case", ANY_ORDER, ids=lambda c: f"n{max(c[0])}w{c[5]}s{c[6]}")
def test_tokens_in_any_order(case, dh, fmt):
    """Rows before the first token, at any one, past the last and at the ends of int32."""
    say(f"paged window, many rows in any order {case} {fmt} {dh}")
    lens, rows, H, group, page, size, sinks = case
    rng = np.random.default_rng(dh + sum(rows))
    pool = Pool(fmt, lens, H, dh, page, seed=1)
    q = rnd(2 * rng.standard_normal((sum(rows), H * group * dh)), "bf16")
    t = np.concatenate([rng.integers(-9, n + 60, r) for n, r in zip(lens, rows)])
    t[[0, 40, 69]] = [BIG, -BIG - 1, BIG - 1]
    got = window(pool, dev(q, torch.bfloat16), rows, group, "bf16", t, size, sinks).double().cpu().numpy()
    assert attention_errors(pool, got, q, rows, group, "bf16", _window_look(pool, rows, t, size, sinks)) <= 1


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh", DIMS)
def test_equal_numbers_of_rows_need_no_offsets(dh, fmt):
    say(f"paged masks without offsets, many rows {fmt} {dh}")
    rng = np.random.default_rng(1)
    lens, rows, H = EQUAL["lens"], EQUAL["rows"], EQUAL["heads"]
    pool = Pool(fmt, lens, H, dh, EQUAL["page"], seed=1)
    q = rnd(rng.standard_normal((sum(rows), H * dh)), "bf16")
    d = dev(q, torch.bfloat16)
    t = np.concatenate([np.arange(r) + n - r for n, r in zip(lens, rows)])
    ctx, mask = [660, 3, 0, 0, 290, 129, 1, 380], rng.integers(0, 2 ** 32, (sum(rows), 2), dtype=np.uint32)
    for one, two, look in (
            (window(pool, d, rows, 1, "bf16", t, 33, 2), window(pool, d, rows, 1, "bf16", t, 33, 2, off=None), _window_look(pool, rows, t, 33, 2)),
            (tree(pool, d, rows, 1, "bf16", ctx, mask), tree(pool, d, rows, 1, "bf16", ctx, mask, off=None),
             _tree_look(pool, rows, ctx, mask))):
        assert torch.equal(one, two)
        assert attention_errors(pool, two.double().cpu().numpy(), q, rows, 1, "bf16", look) <= 1


@pytest.mark.parametrize("dh,fmt", zip(DIMS, FORMATS))
def test_widest_masks_of_many_rows(dh, fmt):
    """64 words: 2048 drafted tokens, some of them past the length, some past the last word."""
    say(f"paged tree, widest masks, many rows {fmt} {dh}")
    rng = np.random.default_rng(3)
    rows, H = WIDEST["rows"], WIDEST["heads"]
    pool = Pool(fmt, WIDEST["lens"], H, dh, WIDEST["page"], seed=1)
    q = rnd(rng.standard_normal((sum(rows), H * dh)), "bf16")
    mask = rng.integers(0, 2 ** 32, (sum(rows), 64), dtype=np.uint32)
    got = tree(pool, dev(q, torch.bfloat16), rows, 1, "bf16", [100, 333], mask).double().cpu().numpy()
    assert attention_errors(pool, got, q, rows, 1, "bf16", _tree_look(pool, rows, [100, 333], mask)) <= 1


@pytest.mark.parametrize("fmt,dh,H,group,page,n_pages", PAST)
def test_pool_past_32_bits_of_many_rows(fmt, dh, H, group, page, n_pages):
    """Pages whose byte and element offsets pass 2^32."""
    say(f"paged masks, pool past 32 bits, many rows {fmt} {dh}")
    es, n = 1 if fmt == "int8" else 2, PAST_ROWS
    assert n_pages * H * page * dh > 2 ** 32
    k = torch.empty(n_pages, H, page, dh * es, dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    ke, ve = (torch.empty(n_pages, H, page, dtype=torch.uint8, device="cuda") for _ in range(2)) if es == 1 else (None, None)
    pool = Pool(fmt, [n], H, dh, page, seed=1)  # (of the same sizes, for the rows)
    pool.cache, pool.width = binding.paged_cache(1, n_pages, H, page, dh, FMT[fmt], k, v, ke, ve), n // page
    ids = [n_pages - 1, 3, n_pages - 2, 5] + list(range(n_pages - 3, n_pages - 3 - n // page, -1))  # most past 2^32
    pool.table = np.array([ids[:n // page]], np.int32)
    pool.dtable = i32(pool.table)
    a = Append(pool, [n], group, "bf16", seed=3)
    a.call(i32(np.arange(n)), binding.rotary(dh, LAYOUT["halves"], [0]), None)
    want = [a.x[:, (w + group) * H:(w + group + 1) * H] for w in range(2)]
    if es == 1:
        want = [ref.value(*ref.quantise(x, fmt)) for x in want]
    t, mask = np.arange(n), np.full((n, 8), 0x55555555, np.uint32)
    for got, look in ((window(pool, a.q_out, [n], group, "bf16", t, 100, 4, q_stride=a.q_out.stride(0)), ref.window(t, n, 100, 4)),
                      (tree(pool, a.q_out, [n], group, "bf16", [50], mask, q_stride=a.q_out.stride(0)), ref.tree(mask, n, 50))):
        g = got.double().cpu().numpy().reshape(n, H * group, dh)
        for x in (0, H * group - 1):
            h = x // group
            q = a.q_out[:, x * dh:(x + 1) * dh].double().cpu().numpy()
            o, m, d = ref.attention(q, want[0][:, h], want[1][:, h], look)
            # (half a step of the output and of each weight, the logits' sums twice, the weighted sum)
            allow = 2.0 ** -8 * (np.abs(o) + m) + m * (2 * (dh + 8) * d[:, None] + n + 64) * 2.0 ** -24
            assert (np.abs(g[:, x] - o) <= allow).all()


# ------------------------------------------------------------------ what is tested of either kernel

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,H", MASKED)
def test_masked_places_count_nothing_by_blocks(dh, H, fmt):
    edges.test_masked_places_count_nothing_in_many_rows(dh, H, fmt)


@pytest.mark.parametrize("dh,H", LAYOUT_OF)
def test_layout_by_blocks(dh, H):
    edges.test_layout_of_many_rows(dh, H)


@pytest.mark.parametrize("fmt,dh,rows,H", CAPTURED)
def test_captured_calls_replay_by_blocks(fmt, dh, rows, H):
    edges.test_captured_calls_replay(fmt, dh, rows, H)


@pytest.mark.parametrize("fmt", FORMATS)
def test_queries_that_are_not_finite_by_blocks(fmt):
    edges.test_queries_that_are_not_finite_stay_among_themselves(fmt, *QUERIES)


@pytest.mark.parametrize("case,dh", [(i, dh) for i in range(len(MANY)) for dh in DIMS])
def test_many_rows_by_blocks(case, dh):
    edges.test_many_rows(MANY[case], FORMATS[(case + DIMS.index(dh)) % 3], dh)


@pytest.mark.parametrize("lens,len_max,seen", [([200, 90], 100, [100, 90]), ([BIG, 90], 208, [208, 90])])
def test_lengths_are_cut_by_blocks(lens, len_max, seen):
    """len_max below a length, and lengths past the page table."""
    say(f"paged masks, cut lengths by blocks {lens}")
    rng = np.random.default_rng(4)
    rows, H = CUT["rows"], CUT["heads"]
    pool = Pool("bf16", [200, 90], H, 64, 16, seed=1, width_extra=0)
    q = rnd(rng.standard_normal((sum(rows), H * 64)), "bf16")
    d = dev(q, torch.bfloat16)
    t = np.concatenate([np.arange(r) + 50 for r in rows])
    mask = rng.integers(0, 2 ** 32, (sum(rows), 7), dtype=np.uint32)
    pool.dlens = i32(lens)
    pool.dk.nan_to_num_(0.5)  # (the last page's slots behind token 199)
    pool.dv.nan_to_num_(0.5)
    got = window(pool, d, rows, 1, "bf16", t, 60, 5, len_max=len_max), tree(pool, d, rows, 1, "bf16", [10, 80], mask, len_max=len_max)
    pool.lens = seen
    for g, look in zip(got, (_window_look(pool, rows, t, 60, 5), _tree_look(pool, rows, [10, 80], mask))):
        assert attention_errors(pool, g.double().cpu().numpy(), q, rows, 1, "bf16", look) <= 1


@pytest.mark.parametrize("dh", DIMS)
@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_that_see_nothing_by_blocks(fmt, dh):
    """Empty masks and windows, whole blocks and single rows of them."""
    say(f"paged masks that leave nothing by blocks {fmt} {dh}")
    H, rows = NOTHING["heads"], NOTHING["rows"]
    n = sum(rows)
    pool = Pool(fmt, NOTHING["lens"], H, dh, 16, seed=2)
    q = torch.ones(n, H * dh, dtype=torch.bfloat16, device="cuda")
    t, mask = np.full(n, -1), np.zeros((n, 3), np.uint32)
    assert (window(pool, q, rows, 1, "bf16", t, 900, 3) == 0).all() and (tree(pool, q, rows, 1, "bf16", [0, 0, 0], mask) == 0).all()
    t[5], mask[129, 2] = 7000, 1
    one = window(pool, q, rows, 1, "bf16", t, 900, 3), tree(pool, q, rows, 1, "bf16", [0, 0, 0], mask)
    for o, i in zip(one, (5, 129)):
        assert (o[i] != 0).any() and (o[[j for j in range(n) if j != i]] == 0).all()


def test_repeated_calls_are_equal_by_blocks():
    say("paged masks repeated by blocks")
    rng = np.random.default_rng(1)
    lens, rows, H = REPEATED
    pool = Pool("e4m3", lens, H, 128, 64, seed=1)
    q = dev(rnd(rng.standard_normal((sum(rows), H * 2 * 128)), "bf16"), torch.bfloat16)
    mask = rng.integers(0, 2 ** 32, (sum(rows), 2), dtype=np.uint32)
    t = rng.integers(0, 9000, sum(rows))
    one = tree(pool, q, rows, 2, "bf16", [8950, 2990, 0], mask), window(pool, q, rows, 2, "bf16", t, 4000, 4)
    for _ in range(3):
        assert torch.equal(one[0], tree(pool, q, rows, 2, "bf16", [8950, 2990, 0], mask))
        assert torch.equal(one[1], window(pool, q, rows, 2, "bf16", t, 4000, 4))
