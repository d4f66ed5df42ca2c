"""Queries and keys turned by their positions, as closely as float32 products allow: sine and
cosine are the nearest float32 numbers, at near and at far positions."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import Pool, i32
from test_gpu_paged_loop import LAYOUT, Append, _table

pytestmark = pytest.mark.gpu


def _parts(x, pos, freq, axis, layout):
    """Of a rotation's pairs: |x cos| + |y sin|, |x cos| and the angle, for either channel."""
    size, first, t = np.zeros(x.shape), np.zeros(x.shape), np.zeros(x.shape)
    n = len(freq)
    for i in range(n):
        one, two = (i, i + n) if layout == "halves" else (2 * i, 2 * i + 1)
        a = pos[axis[i]] * freq[i]
        c, s = np.abs(np.cos(a))[:, None], np.abs(np.sin(a))[:, None]
        for u, v in ((one, two), (two, one)):
            first[..., u], size[..., u] = np.abs(x[..., u]) * c, np.abs(x[..., u]) * c + np.abs(x[..., v]) * s
            t[..., u] = np.abs(a)[:, None] * (np.abs(x[..., u]) + np.abs(x[..., v]))
    return size, first, t


@pytest.mark.parametrize("layout", ["halves", "neighbours"])
@pytest.mark.parametrize("rows,heads", [(90, 2), (900, 5)])
@pytest.mark.parametrize("far", [1 << 10, 1 << 20, 1 << 29])
def test_turned_rows_are_off_by_their_products_roundings(far, rows, heads, layout):
    say(f"paged append angles {far} {rows} {layout}")
    dh, rot = 128, binding.rotary(128, LAYOUT[layout], [64])
    pool = Pool("bf16", [rows], heads, dh, 64, seed=1)
    a = Append(pool, [rows], 6, "f32", seed=2)
    rng = np.random.default_rng(3)
    pos = rng.integers(-far, far, (1, rows)).astype(np.int32)
    a.call(i32(np.arange(rows)), rot, i32(pos))
    torch.cuda.synchronize()
    freq, axis = _table(rot)
    x = a.x[:, :6 * heads]
    want = ref.rotate(x, pos, freq, axis, layout)
    size, first, t = _parts(x, pos.astype(np.float64), freq, axis, layout)
    # sine and cosine rounded (half a step, 2^-24 of them, and the sums' terms left out, below 2^-32), the
    # 64-bit angle's factors and itself rounded and its reference's (4 * 2^-53 of it), one product rounded, the fused sum rounded
    allow = size * (2.0 ** -24 + 2.0 ** -32) + 4 * 2.0 ** -53 * t + first * 2.0 ** -24 * (1 + 2.0 ** -20)
    allow += (np.abs(want) + allow) * 2.0 ** -24 + 2.0 ** -149
    got = a.q_out[:, :a.D].double().cpu().numpy().reshape(want.shape)
    worst = (np.abs(got - want) / allow).max()
    assert worst <= 1, worst
