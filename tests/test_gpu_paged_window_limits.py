"""Windows of rows that stand far past their sequences' tokens, whole blocks of them, by the
kernels of few and of many rows."""
import numpy as np
import pytest
import torch

from gpu_util import say
from paged_util import TORCH, Pool, attention_errors, dev, rnd
from test_gpu_paged_loop import BIG, _window_look, window

pytestmark = pytest.mark.gpu


LENS = [300, 40, 1, 64]
WINDOWS = [(256, 4), (960, 64), (1, 1), (256, 0), (BIG - 300, 9), (BIG, 70)]
# format, dh, heads, rows of each sequence, type: many rows (tests/test_paged_plan.py) and few
MANY = [("bf16", 128, 24, 130, "bf16"), ("e4m3", 64, 64, 130, "bf16"), ("int8", 80, 64, 129, "bf16"), ("e4m3", 128, 64, 130, "bf16")]
FEW = [("bf16", 64, 2, 40, "bf16"), ("int8", 128, 2, 3, "f32")]


def by_blocks():
    return [dict(dtype=dtype, fmt=fmt, dh=dh, seqs=4, total=4 * rows, most=rows, heads=H, group=1, len_max=max(LENS), look="window",
                 window=size, sinks=sinks) for fmt, dh, H, rows, dtype in MANY for size, sinks in WINDOWS]


@pytest.mark.parametrize("size,sinks", WINDOWS)
@pytest.mark.parametrize("fmt,dh,H,rows,dtype", MANY + FEW)
def test_rows_far_past_the_tokens(fmt, dh, H, rows, dtype, size, sinks):
    """What they see is what their window and the sinks have of the sequence, nothing for some."""
    say(f"paged window, rows far past the tokens {fmt} {dh} {rows} {size} {sinks}")
    rng = np.random.default_rng(rows)
    n = 4 * rows
    pool = Pool(fmt, LENS, H, dh, 16, seed=1)
    q = rnd(rng.standard_normal((n, H * dh)), dtype)
    d = dev(q, TORCH[dtype])
    tokens = [np.full(n, BIG), np.repeat([BIG - size, 299 + size, BIG - 1, 0], rows).clip(0, BIG)]
    if H < 20:
        tokens += [BIG - rng.integers(0, 2000, n), np.full(n, BIG - 960 - 15)]
    for t in tokens:
        got = window(pool, d, [rows] * 4, 1, dtype, t, size, sinks).double().cpu().numpy()
        assert attention_errors(pool, got, q, [rows] * 4, 1, dtype, _window_look(pool, [rows] * 4, t, size, sinks)) <= 1
