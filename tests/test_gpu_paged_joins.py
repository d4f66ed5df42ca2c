"""The join of split caches' parts for windows and drafted trees, by lane groups (csrc/k_paged.hip,
paged_rows_join_kernel): behind the kernels of few and of many rows, for both types of rows, one
(row, head) pair a group and four in turn, from sequence to sequence.  tests/test_paged_plan.py
holds the sizes to those ways."""
import numpy as np
import pytest
import torch

from gpu_util import say
from paged_util import TORCH, Pool, attention_errors, dev, i32, offsets, rnd
from test_gpu_paged_loop import BIG, _tree_look, _window_look, tree, window

pytestmark = pytest.mark.gpu


def _spread(n, most, step):
    """Ragged numbers up to `most`, 0 among them."""
    return [most if i == n // 2 else (i * step) % (most + 1) for i in range(n)]


# look, dtype, head_dim, heads, group, format, lens, rows, rows before and behind the sequences',
# window, sinks; then what the plan has to be: many-row kernel, turns of the join
CASES = [
    ("tree", "f32", 64, 16, 1, "bf16", _spread(16, 4200, 1300), _spread(16, 33, 13), 0, 3, 0, 0, False, 1),
    ("tree", "bf16", 64, 16, 1, "int8", _spread(16, 4200, 1300), _spread(16, 33, 13), 0, 3, 0, 0, False, 1),
    ("tree", "f32", 128, 1, 64, "e4m3", _spread(20, 4300, 700), _spread(20, 12, 5), 150, 300, 0, 0, False, 4),
    ("tree", "bf16", 128, 4, 16, "e4m3", [5000] + [19] * 128 + [700], [4] * 130, 2, 0, 0, 0, False, 4),
    ("tree", "bf16", 80, 4, 16, "bf16", [4500] + [40] * 134, [4, 0, 3] * 45, 50, 200, 0, 0, False, 4),
    ("tree", "bf16", 128, 4, 16, "bf16", [2000, 30, 1500, 700, 0, 64], [100, 100, 99, 100, 14, 99], 1, 3, 0, 0, True, 4),
    ("tree", "bf16", 64, 4, 16, "int8", [2000, 30, 1500, 700, 0, 64], [100, 100, 99, 100, 14, 99], 200, 320, 0, 0, True, 4),
    ("window", "f32", 64, 4, 8, "int8", [4000, 500, 0, 3333], [33, 32, 31, 33], 5, 20, 3000, 4, False, 1),
    ("window", "bf16", 64, 4, 8, "e4m3", [4000, 500, 0, 3333], [8, 7, 1, 8], 50, 70, 3000, 4, False, 1),
    ("window", "f32", 80, 4, 16, "bf16", [4000, 500, 0, 3333], [9, 8, 5, 9], 300, 200, 3000, 70, False, 4),
    ("window", "bf16", 128, 4, 16, "int8", [4000, 500, 0, 3333], [4, 4, 3, 1], 100, 410, 3000, 0, False, 4),
    ("window", "bf16", 128, 1, 64, "bf16", [2000], [520], 0, 0, 1500, 4, True, 4),
    ("window", "bf16", 80, 8, 16, "e4m3", [4000, 130, 2000], [130, 129, 41], 0, 0, 3000, 40, True, 4),
]


def _name(c):
    return f"{c[0]}-{c[1]}-{c[2]}-{c[5]}-{'many' if c[12] else 'few'}{c[13]}"


def plans():
    """(sizes, what their plan has to be) of the calls below."""
    return [(dict(dtype=dtype, fmt=fmt, dh=dh, seqs=len(rows), total=before + sum(rows) + extra, most=max(rows), heads=H, group=group,
                  len_max=max(lens), look=look, window=max(1, size), sinks=sinks), many, turns)
            for look, dtype, dh, H, group, fmt, lens, rows, before, extra, size, sinks, many, turns in CASES]


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_joins(case):
    say(f"paged joins {_name(case)}")
    look, dtype, dh, H, group, fmt, lens, rows, before, extra, size, sinks, _, _ = case
    rng = np.random.default_rng(dh + sum(rows))
    pool = Pool(fmt, lens, H, dh, 64, seed=1)
    n, total, D = sum(rows), before + sum(rows) + extra, H * group * dh
    q = rnd(2 * rng.standard_normal((total, D)), dtype)
    o = torch.full((total, D), 7.0, dtype=TORCH[dtype], device="cuda")
    off = i32(offsets(rows) + before)
    if look == "tree":
        ctx = np.array([max(0, x - r) if i % 3 else rng.integers(0, x + 1) for i, (x, r) in enumerate(zip(lens, rows))])
        mask = rng.integers(0, 2 ** 32, (total, 4), dtype=np.uint32)
        mask[::7] = 0
        ctx[0::5] = 0
        got = tree(pool, dev(q, TORCH[dtype]), rows, group, dtype, ctx, mask, o=o, off=off)
        sees = _tree_look(pool, rows, ctx, mask[before:before + n])
    else:
        t = np.concatenate([np.zeros(before, int)] + [np.arange(x - r, x) for x, r in zip(lens, rows)] + [np.zeros(extra, int)])
        t[before:before + n:9] = rng.integers(-3, 4100, len(t[before:before + n:9]))
        t[before + 1] = BIG
        got = window(pool, dev(q, TORCH[dtype]), rows, group, dtype, t, size, sinks, o=o, off=off)
        sees = _window_look(pool, rows, t[before:before + n], size, sinks)
    assert (got[:before] == 7).all() and (got[before + n:] == 7).all()
    got = got[before:before + n].double().cpu().numpy()
    assert attention_errors(pool, got, q[before:before + n], rows, group, dtype, sees) <= 1
