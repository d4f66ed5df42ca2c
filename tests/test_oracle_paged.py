"""The paged cache's oracle against independent statements of the same things
(CPU only)."""
import numpy as np
import pytest
import torch

from oracle import block
from oracle import paged as ref


def test_e4m3_rounding_is_torch_s():
    rng = np.random.default_rng(0)
    y = np.concatenate([rng.uniform(-448, 448, 4000), rng.uniform(-0.1, 0.1, 4000), [0.0, 448.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10],
                        np.exp2(rng.uniform(-12, 8, 4000))]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(ref.round_e4m3(y), want)


@pytest.mark.parametrize("fmt,limit", [("e4m3", 448.0), ("int8", 127.0)])
def test_exponents_are_the_least(fmt, limit):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3000, 8)) * np.exp2(rng.uniform(-90, 90, (3000, 1)))
    x[:8, 0] = limit * np.exp2(np.arange(8.0))
    x[:8, 1:] = 0
    x[8:16, 0] = np.nextafter(limit * np.exp2(np.arange(8.0)), np.inf)
    x[8:16, 1:] = 0
    q, code = ref.quantise(x, fmt)
    amax, e = np.abs(x).max(-1), code - 127.0
    assert (amax <= limit * np.exp2(e)).all()
    assert ((amax > limit * np.exp2(e - 1)) | (e == ref.LEAST)).all()
    assert (e[:8] == np.arange(8)).all() and (e[8:16] == np.arange(1, 9)).all()
    assert np.abs(q).max() <= limit
    # half a step of the format: int8 steps 2^e, e4m3 2^-4 of the value above its subnormals
    err = np.abs(ref.value(q, code) - x)
    step = np.exp2(e)[:, None] if fmt == "int8" else np.maximum(np.abs(x) * 2.0 ** -3, np.exp2(e)[:, None] * 2.0 ** -9)
    assert (err <= step / 2).all()


def test_small_zero_and_infinite_rows():
    q, code = ref.quantise(np.array([[0.0, 0.0], [2.0 ** -120, 0.0], [np.inf, 1.0], [np.nan, 1.0]]), "int8")
    assert code.tolist() == [16, 16, 255, 255] and (q == 0).all()
    assert np.isnan(ref.value(q, code)[2:]).all()
    q, code = ref.quantise(np.array([[np.inf, 1.0]]), "e4m3")
    assert np.isnan(q).all() and code.tolist() == [255]


def test_scores_bound_the_logits():
    """With exact bounds and queries the score is an upper bound of every
    logit of the page; quantising moves it by at most the two steps' parts."""
    rng = np.random.default_rng(2)
    k, q = rng.standard_normal((16, 1, 64)), rng.standard_normal((3, 64))
    b, code = ref.bounds(k)
    s = ref.scores(q, b, code)
    qq, qc = ref.quantise(q, "int8")
    slack = (np.abs(q).sum(1) * np.exp2(code[0] - 128.0) + np.abs(ref.value(b[0], np.array([code[0]] * 2))).max(0).sum() *
             np.exp2(qc - 128.0))
    assert s.shape == (1,)
    assert (k[:, 0] @ q.T).max() <= s[0] + slack.max()


def test_selection_order():
    assert ref.select(np.array([1.0, 3, 3, -np.inf, 2]), 3) == [1, 2, 4]
    assert ref.select(np.array([1.0, 1, 1]), 2) == [0, 1]
    assert ref.select(np.array([1.0]), 3) == [0, -1, -1]


def test_attention_is_the_block_s():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 64)), rng.standard_normal((40, 64)), rng.standard_normal((40, 64))
    o, _, _ = ref.attention(q, k, v)
    np.testing.assert_allclose(o, block.attention(q, k, v)[0], rtol=1e-12)
    look = rng.random((3, 40)) < 0.3
    look[1] = False
    o, a, _ = ref.attention(q, k, v, look)
    assert (o[1] == 0).all()
    np.testing.assert_allclose(o[0], block.attention(q[:1], k[look[0]], v[look[0]])[0][0], rtol=1e-12)
