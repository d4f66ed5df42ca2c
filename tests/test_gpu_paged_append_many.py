"""Appends of many rows, four heads a lane group (csrc/k_paged_append.hip): halves and neighbours,
row offsets with empty sequences, in place, rows loaded past the caches or not.
tests/test_paged_plan.py holds the sizes to those ways."""
import numpy as np
import pytest
import torch

from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import DT, Pool, i32, offsets
from test_gpu_paged_loop import LAYOUT, Append

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]
HEADS, GROUP = 5, 2                          # the last lane group of a row takes one head, or two of the queries
ROWS = [700, 0, 3, 0, 0, 640, 1, 0, 400, 0]  # of each sequence
LARGE = [r * 16 for r in ROWS]               # past the caches
FEW = 100                                    # of a small call, a head a lane group


def plans():
    """(dtype, dh, rows, query heads, key heads), heads of a lane group, rows past the caches"""
    out = []
    for dtype in ("bf16", "f32"):
        for dh in (64, 80, 128):
            out += [((dtype, dh, sum(ROWS), HEADS * g, HEADS), 4, False) for g in (GROUP, 3)]
            out += [((dtype, dh, FEW, HEADS * GROUP, HEADS), 1, False)]
        out += [((dtype, 64, sum(LARGE), HEADS * GROUP, HEADS), 4, True)]
    return out


def _same(one, two):
    for x, y in ((one.dk, two.dk), (one.dv, two.dv), (one.dke, two.dke), (one.dve, two.dve)):
        assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def _indexes(rows, seed):
    return np.concatenate([np.random.default_rng(seed + b).permutation(n) for b, n in enumerate(rows)]).astype(np.int32)


@pytest.mark.parametrize("layout,pairs,pos", [("halves", [0], False), ("neighbours", [0, 0], False), ("halves", [32], True),
                                              ("neighbours", [27], True)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_many_rows_without_a_turn_are_written(fmt, dtype, layout, pairs, pos):
    """No pairs, or every position 0: queries come back and the cache holds what
    marche_paged_write puts there, bit for bit."""
    say(f"paged append, many rows as write {fmt} {dtype} {layout} {pairs}")
    rot = binding.rotary(64, LAYOUT[layout], pairs)
    one, two = (Pool(fmt, ROWS, HEADS, 64, 16, seed=3) for _ in range(2))
    a = Append(one, ROWS, 3, dtype, seed=5, scale=10.0)
    idx = i32(_indexes(ROWS, 1))
    a.call(idx, rot, torch.zeros(rot.n_axes, a.n, dtype=torch.int32, device="cuda") if pos else None)
    q, k, v = a.cut()
    binding.paged_write(two.cache, 0, two.dtable, two.width, len(ROWS), idx, i32(a.off), a.n, k, v, a.stride, DT[dtype])
    torch.cuda.synchronize()
    assert torch.equal(a.q_out[:, :a.D], q[:, :a.D]) and (a.q_out[:, a.D:] == 7).all()
    _same(one, two)


def _against_small_calls(fmt, dtype, dh, layout, pairs, rows, in_place):
    """One call for all the rows against calls of FEW rows of a sequence each."""
    rot = binding.rotary(dh, LAYOUT[layout], pairs)
    big, small = (Pool(fmt, rows, HEADS, dh, 64, seed=2) for _ in range(2))
    a, b = (Append(p, rows, GROUP, dtype, seed=4) for p in (big, small))
    n, off = a.n, offsets(rows)
    pos = i32(np.stack([(np.arange(n) * (x + 3)) % 5000 - 70 * x for x in range(rot.n_axes)]))
    idx = i32(_indexes(rows, 7))
    a.call(idx, rot, pos, q_out=a.cut()[0] if in_place else None)
    q, k, v = b.cut()
    for s, r in enumerate(rows):
        for r0 in range(off[s], off[s + 1], FEW):
            m = min(FEW, off[s + 1] - r0)
            binding.paged_append(small.cache, 0, small.dtable[s:s + 1].contiguous(), small.width, 1, idx[r0:r0 + m].contiguous(), None, m,
                                 rot, pos[:, r0:r0 + m].contiguous(), q[r0:r0 + m], HEADS * GROUP, k[r0:r0 + m],
                                 v[r0:r0 + m], b.stride, DT[dtype], b.q_out[r0:r0 + m], b.q_out.stride(0))
    torch.cuda.synchronize()
    if in_place:
        assert torch.equal(a.cut()[0][:, :a.D], b.q_out[:, :b.D])
        assert torch.equal(a.buf[:, 8 + a.D:], b.buf[:, 8 + b.D:]) and a.buf[:, :8].isnan().all()
    else:
        assert torch.equal(a.q_out, b.q_out) and torch.equal(a.buf[:, 8:], b.buf[:, 8:])
    _same(big, small)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("layout,share", [("halves", [1.0]), ("halves", [0.25, 0.375, 0.125]), ("neighbours", [1.0]),
                                          ("neighbours", [0.1, 0.3, 0.2, 0.1])])
@pytest.mark.parametrize("fmt,dtype,dh", [("bf16", "bf16", 64), ("e4m3", "f32", 80), ("int8", "bf16", 128), ("int8", "f32", 64),
                                          ("bf16", "f32", 128), ("e4m3", "bf16", 80)])
def test_many_rows_are_small_calls_together(fmt, dtype, dh, layout, share, in_place):
    say(f"paged append, many rows {fmt} {dtype} {dh} {layout} {share} {in_place}")
    pairs = [int(s * dh // 2) for s in share]
    if layout == "halves":
        pairs[0] -= sum(pairs) % 4
    _against_small_calls(fmt, dtype, dh, layout, pairs, ROWS, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("layout", ["halves", "neighbours"])
@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("bf16", "f32")])
def test_rows_past_the_caches_with_offsets(fmt, dtype, layout, in_place):
    say(f"paged append, rows past the caches {fmt} {dtype} {layout} {in_place}")
    _against_small_calls(fmt, dtype, 64, layout, [8, 12, 8], LARGE, in_place)
