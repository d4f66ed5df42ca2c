"""Windows of rows that stand far past their sequences' tokens, whole blocks of them, by the
kernels of few and of many rows."""
import numpy as np
import pytest
import torch

from gpu_util import say
from paged_util import TORCH, Pool, attention_errors, dev, rnd
from test_gpu_paged_loop import BIG, _window_look, window

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size,sinks", [(256, 4), (960, 64), (1, 1), (256, 0), (BIG - 300, 9), (BIG, 70)])
@pytest.mark.parametrize("fmt,dh,H,rows,dtype", [("bf16", 128, 16, 130, "bf16"), ("e4m3", 64, 64, 130, "bf16"), ("int8", 80, 64, 129, "bf16"),
                                                 ("bf16", 64, 2, 40, "bf16"), ("int8", 128, 2, 3, "f32")])
def test_rows_far_past_the_tokens(fmt, dh, H, rows, dtype, size, sinks):
    """What they see is what their window and the sinks have of the sequence, nothing for some."""
    say(f"paged window, rows far past the tokens {fmt} {dh} {rows} {size} {sinks}")
    rng = np.random.default_rng(rows)
    lens = [1000, 40]
    pool = Pool(fmt, lens, H, dh, 16, seed=1)
    q = rnd(rng.standard_normal((2 * rows, H * dh)), dtype)
    d = dev(q, TORCH[dtype])
    for t in (np.full(2 * rows, BIG), BIG - rng.integers(0, 2000, 2 * rows), np.full(2 * rows, BIG - 960 - 15),
              np.repeat([BIG - size, 999 + size], rows).clip(0, BIG)):
        got = window(pool, d, [rows] * 2, 1, dtype, t, size, sinks).double().cpu().numpy()
        assert attention_errors(pool, got, q, [rows] * 2, 1, dtype, _window_look(pool, [rows] * 2, t, size, sinks)) <= 1
