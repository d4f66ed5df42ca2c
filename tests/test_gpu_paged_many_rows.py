"""Windows and drafted trees by the kernel of many rows (csrc/paged_rows.h) on the GPU against
the float64 oracle: tokens in any order, calls without offsets, the widest masks, pools past
32 bits.  tests/test_paged_plan.py holds the sizes to that kernel."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import FMT, Pool, attention_errors, dev, i32, rnd
from test_gpu_paged_loop import BIG, LAYOUT, Append, _tree_look, _window_look, tree, window

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]
HEADS = [(64, 64), (80, 64), (128, 16)]  # channels, key heads: for blocks enough

# lens, rows of each sequence, group, page, window, sinks
ANY_ORDER = [
    ([700, 90], [150, 70], 1, 16, 40, 9),
    ([1300, 64], [130, 130], 1, 64, 500, 0),
    ([513, 1, 0], [70, 33, 66], 2, 32, 1, 100),
    ([300, 2100], [80, 200], 1, 128, BIG, 3),
]
EQUAL = dict(lens=[700, 50], rows=[130, 130], page=16)
WIDEST = dict(lens=[2500, 1200], rows=[140, 140], page=16)
PAST = [("int8", 128, 16, 64, 35000), ("bf16", 64, 64, 16, 70000)]  # format, channels, heads, page, pages
PAST_ROWS = 384


def _sizes(look, dh, heads, lens, rows, group=1, window=1, sinks=0):
    return dict(dtype="bf16", dh=dh, seqs=len(rows), total=sum(rows), most=max(rows), heads=heads, group=group, len_max=max(lens),
                look=look, window=window, sinks=sinks)


def by_blocks():
    """Sizes of the calls below."""
    out = []
    for dh, H in HEADS:
        out += [_sizes("window", dh, H, c[0], c[1], c[2], c[4], c[5]) for c in ANY_ORDER]
        out += [_sizes("window", dh, H, EQUAL["lens"], EQUAL["rows"], 1, 33, 2), _sizes("tree", dh, H, EQUAL["lens"], EQUAL["rows"]),
                _sizes("tree", dh, H, WIDEST["lens"], WIDEST["rows"])]
    for _, dh, H, page, _ in PAST:
        out += [_sizes("window", dh, H, [PAST_ROWS], [PAST_ROWS], 1, 100, 4), _sizes("tree", dh, H, [PAST_ROWS], [PAST_ROWS])]
    return out


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,H", HEADS)
@pytest.mark.parametrize("case", ANY_ORDER, ids=lambda c: f"n{max(c[0])}w{c[4]}s{c[5]}")
def test_tokens_in_any_order(case, dh, H, fmt):
    """Rows before the first token, at any one, past the last and at the ends of int32."""
    say(f"paged window, many rows in any order {case} {fmt} {dh}")
    lens, rows, group, page, size, sinks = case
    rng = np.random.default_rng(dh + sum(rows))
    pool = Pool(fmt, lens, H, dh, page, seed=1)
    q = rnd(2 * rng.standard_normal((sum(rows), H * group * dh)), "bf16")
    t = np.concatenate([rng.integers(-9, n + 60, r) for n, r in zip(lens, rows)])
    t[[0, 40, 69]] = [BIG, -BIG - 1, BIG - 1]
    got = window(pool, dev(q, torch.bfloat16), rows, group, "bf16", t, size, sinks).double().cpu().numpy()
    assert attention_errors(pool, got, q, rows, group, "bf16", _window_look(pool, rows, t, size, sinks)) <= 1


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,H", HEADS)
def test_equal_numbers_of_rows_need_no_offsets(dh, H, fmt):
    say(f"paged masks without offsets, many rows {fmt} {dh}")
    rng = np.random.default_rng(1)
    lens, rows = EQUAL["lens"], EQUAL["rows"]
    pool = Pool(fmt, lens, H, dh, EQUAL["page"], seed=1)
    q = rnd(rng.standard_normal((sum(rows), H * dh)), "bf16")
    d = dev(q, torch.bfloat16)
    t = np.concatenate([np.arange(r) + n - r for n, r in zip(lens, rows)])
    mask = rng.integers(0, 2 ** 32, (sum(rows), 2), dtype=np.uint32)
    for one, two, look in (
            (window(pool, d, rows, 1, "bf16", t, 33, 2), window(pool, d, rows, 1, "bf16", t, 33, 2, off=None), _window_look(pool, rows, t, 33, 2)),
            (tree(pool, d, rows, 1, "bf16", [660, 3], mask), tree(pool, d, rows, 1, "bf16", [660, 3], mask, off=None),
             _tree_look(pool, rows, [660, 3], mask))):
        assert torch.equal(one, two)
        assert attention_errors(pool, two.double().cpu().numpy(), q, rows, 1, "bf16", look) <= 1


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dh,H", HEADS)
def test_widest_masks_of_many_rows(dh, H, fmt):
    """64 words: 2048 drafted tokens, some of them past the length, some past the last word."""
    say(f"paged tree, widest masks, many rows {fmt} {dh}")
    rng = np.random.default_rng(3)
    rows = WIDEST["rows"]
    pool = Pool(fmt, WIDEST["lens"], H, dh, WIDEST["page"], seed=1)
    q = rnd(rng.standard_normal((sum(rows), H * dh)), "bf16")
    mask = rng.integers(0, 2 ** 32, (sum(rows), 64), dtype=np.uint32)
    got = tree(pool, dev(q, torch.bfloat16), rows, 1, "bf16", [100, 333], mask).double().cpu().numpy()
    assert attention_errors(pool, got, q, rows, 1, "bf16", _tree_look(pool, rows, [100, 333], mask)) <= 1


@pytest.mark.parametrize("fmt,dh,H,page,n_pages", PAST)
def test_pool_past_32_bits_of_many_rows(fmt, dh, H, page, n_pages):
    """Pages whose byte and element offsets pass 2^32."""
    say(f"paged masks, pool past 32 bits, many rows {fmt} {dh}")
    es, n = 1 if fmt == "int8" else 2, PAST_ROWS
    assert n_pages * H * page * dh > 2 ** 32
    k = torch.empty(n_pages, H, page, dh * es, dtype=torch.uint8, device="cuda")
    v = torch.empty_like(k)
    ke, ve = (torch.empty(n_pages, H, page, dtype=torch.uint8, device="cuda") for _ in range(2)) if es == 1 else (None, None)
    pool = Pool(fmt, [n], H, dh, page, seed=1)  # (of the same sizes, for the rows)
    pool.cache, pool.width = binding.paged_cache(1, n_pages, H, page, dh, FMT[fmt], k, v, ke, ve), n // page
    ids = [n_pages - 1, 3, n_pages - 2, 5] + list(range(n_pages - 3, n_pages - 3 - n // page, -1))
    pool.table = np.array([ids[:n // page]], np.int32)
    pool.dtable = i32(pool.table)
    a = Append(pool, [n], 1, "bf16", seed=3)
    a.call(i32(np.arange(n)), binding.rotary(dh, LAYOUT["halves"], [0]), None)
    want = [a.x[:, (w + 1) * H:(w + 2) * H] for w in range(2)]
    if es == 1:
        want = [ref.value(*ref.quantise(x, fmt)) for x in want]
    t, mask = np.arange(n), np.full((n, 8), 0x55555555, np.uint32)
    for got, look in ((window(pool, a.q_out, [n], 1, "bf16", t, 100, 4, q_stride=a.q_out.stride(0)), ref.window(t, n, 100, 4)),
                      (tree(pool, a.q_out, [n], 1, "bf16", [50], mask, q_stride=a.q_out.stride(0)), ref.tree(mask, n, 50))):
        g = got.double().cpu().numpy().reshape(n, H, dh)
        for h in (0, H - 1):
            q = a.q_out[:, h * dh:(h + 1) * dh].double().cpu().numpy()
            o, m, d = ref.attention(q, want[0][:, h], want[1][:, h], look)
            # (half a step of the output and of each weight, the logits' sums twice, the weighted sum)
            allow = 2.0 ** -8 * (np.abs(o) + m) + m * (2 * (dh + 8) * d[:, None] + n + 64) * 2.0 ** -24
            assert (np.abs(g[:, h] - o) <= allow).all()
