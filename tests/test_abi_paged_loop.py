"""Positions, windows and drafted trees on the paged cache without a GPU: what the
calls refuse on the host before any HIP call, and the rotation's table (CPU only)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2506_12035_amd import binding

from test_abi_paged import FAKE, INVALID, OK, UNSUPPORTED, WORKSPACE, _cache, built_library  # noqa: F401

HALVES, NEIGHBOURS = binding.MARCHE_ROTARY_HALVES, binding.MARCHE_ROTARY_NEIGHBOURS
BIG = 2 ** 31 - 1


def _append(cache=None, **kw):
    a = dict(layer=1, table=FAKE, max_pages=5, n_seqs=2, idx=FAKE, off=FAKE, total=6, rot=None, pos=FAKE, q=FAKE,
             heads=8, k=FAKE, v=FAKE, stride=512, dtype=binding.MARCHE_BF16, q_out=FAKE + 4096, q_out_stride=512)
    a.update(kw)
    rot = a["rot"] or binding.rotary(64, HALVES, [32])
    return binding.lib().marche_paged_append(
        C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"], a["n_seqs"], a["idx"], a["off"], a["total"],
        None if rot == "none" else C.byref(rot), a["pos"], a["q"], a["heads"], a["k"], a["v"], a["stride"], a["dtype"],
        a["q_out"], a["q_out_stride"], None)


def _window(cache=None, **kw):
    a = dict(layer=0, table=FAKE, max_pages=5, lens=FAKE, len_max=320, n_seqs=2, q=FAKE, stride=512, idx=FAKE, off=FAKE,
             total=6, q_max=4, heads=8, dtype=binding.MARCHE_BF16, window=100, sinks=4, o=FAKE, ws=None, ws_bytes=0)
    a.update(kw)
    return binding.lib().marche_paged_attention_window(
        C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"], a["lens"], a["len_max"], a["n_seqs"], a["q"],
        a["stride"], a["idx"], a["off"], a["total"], a["q_max"], a["heads"], a["dtype"], a["window"], a["sinks"], a["o"],
        a["ws"], a["ws_bytes"], None)


def _tree(cache=None, **kw):
    a = dict(layer=0, table=FAKE, max_pages=5, lens=FAKE, len_max=320, n_seqs=2, q=FAKE, stride=512, off=FAKE, total=6,
             q_max=4, heads=8, dtype=binding.MARCHE_BF16, ctx=FAKE, mask=FAKE, words=1, o=FAKE, ws=None, ws_bytes=0)
    a.update(kw)
    return binding.lib().marche_paged_attention_tree(
        C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"], a["lens"], a["len_max"], a["n_seqs"], a["q"],
        a["stride"], a["off"], a["total"], a["q_max"], a["heads"], a["dtype"], a["ctx"], a["mask"], a["words"], a["o"],
        a["ws"], a["ws_bytes"], None)


CALLS = [_append, _window, _tree]


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__[1:])
@pytest.mark.parametrize("kw,status,word", [
    (dict(n_layers=0), INVALID, "n_layers"), (dict(n_heads=0), INVALID, "n_heads"),
    (dict(page_size=48), UNSUPPORTED, "page_size"), (dict(head_dim=96), UNSUPPORTED, "head_dim"),
    (dict(fmt=3), UNSUPPORTED, "format"), (dict(k=None), INVALID, "cache.k"), (dict(v_exp=None), INVALID, "v_exp"),
    (dict(k=FAKE + 8), INVALID, "aligned")])
def test_cache_is_checked(call, kw, status, word):
    assert call(_cache(**kw)) == status
    assert word in binding.last_error()


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__[1:])
def test_shared_arguments_are_checked(call):
    assert call(layer=-1) == INVALID and "layer" in binding.last_error()
    assert call(layer=2) == INVALID
    assert call(max_pages=0) == INVALID and "max_pages" in binding.last_error()
    assert call(n_seqs=-1) == INVALID
    assert call(n_seqs=0) == INVALID
    assert call(table=None) == INVALID and "NULL" in binding.last_error()
    assert call(dtype=2) == UNSUPPORTED and "dtype" in binding.last_error()
    assert call(total=-1) == INVALID
    assert call(off=None, total=5) == INVALID and "multiple" in binding.last_error()
    for stride in (511, 508, -512):
        assert call(stride=stride) == INVALID and "stride" in binding.last_error()
    assert call(heads=6) == INVALID and "n_q_heads" in binding.last_error()
    assert call(q=None) == INVALID and "NULL" in binding.last_error()
    assert call(q=FAKE + 8) == INVALID and "aligned" in binding.last_error()
    # nothing to do
    assert call(total=0, q_max=0) == OK
    assert call(total=0, q_max=0, n_seqs=0) == OK


def test_append_refusals():
    for name in ("idx", "k", "v", "q_out"):
        assert _append(**{name: None}) == INVALID and "NULL" in binding.last_error()
    for name in ("k", "v", "q_out"):
        assert _append(**{name: FAKE + 8}) == INVALID and "aligned" in binding.last_error()
    for stride in (504, 516, 511, -512):
        assert _append(q_out_stride=stride) == INVALID and "q_out_stride" in binding.last_error()
    # in place only row for row
    assert _append(q_out=FAKE, q_out_stride=520, stride=528) == INVALID and "q_out is q" in binding.last_error()
    # keys and values alone take neither queries nor a place for them
    assert _append(heads=0) == INVALID and "without query heads" in binding.last_error()
    assert _append(heads=0, q=None) == INVALID
    assert _append(heads=0, q=None, q_out=None, k=None) == INVALID and "NULL" in binding.last_error()
    assert _append(heads=-4) == INVALID
    assert _append(heads=0, q=None, q_out=None, stride=248) == INVALID and "stride" in binding.last_error()
    assert _append(rot="none") == INVALID and "rotary" in binding.last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(layout=2), "layout"), (dict(layout=-1), "layout"), (dict(n_pairs=-4), "n_pairs"), (dict(n_pairs=36), "n_pairs"),
    (dict(n_pairs=30), "n_pairs"), (dict(n_axes=0), "n_axes"), (dict(n_axes=5), "n_axes"), (dict(axis=(31, 1)), "axis[31]"),
    (dict(freq=(0, math.nan)), "freq[0]"), (dict(freq=(7, math.inf)), "freq[7]"), (dict(freq=(7, -65537.0)), "freq[7]")])
def test_rotation_is_checked(kw, word):
    rot = binding.rotary(64, HALVES, [32])
    for name, x in kw.items():
        if name in ("axis", "freq"):
            getattr(rot, name)[x[0]] = x[1]
        else:
            setattr(rot, name, x)
    assert _append(rot=rot) == INVALID and word in binding.last_error()


def test_rotation_past_its_pairs_is_not_looked_at():
    rot = binding.rotary(64, NEIGHBOURS, [3])
    rot.axis[3], rot.freq[3] = 9, math.nan
    assert _append(rot=rot, idx=None) == INVALID and "NULL" in binding.last_error()


@pytest.mark.parametrize("dh", [64, 80, 128])
def test_rotation_tables(dh):
    p = dh // 2
    r = binding.rotary(dh, HALVES, [p])
    np.testing.assert_allclose(r.freq[:p], 10000.0 ** (-np.arange(p) / p), rtol=1e-15)
    assert (r.n_pairs, r.n_axes, r.layout, set(r.axis)) == (p, 1, HALVES, {0})
    r = binding.rotary(dh, NEIGHBOURS, [3, 0, 7, 5], base=500.0)
    assert (r.n_pairs, r.n_axes, r.layout) == (15, 4, NEIGHBOURS) and list(r.axis[:15]) == [0] * 3 + [2] * 7 + [3] * 5
    np.testing.assert_allclose(r.freq[:15], 500.0 ** (-np.arange(15) / 15), rtol=1e-15)
    r = binding.rotary(dh, NEIGHBOURS, [3, 5], True, 500.0)
    np.testing.assert_allclose(r.freq[:8], [500.0 ** (-j / n) for n in (3, 5) for j in range(n)], rtol=1e-15)
    assert binding.rotary(dh, HALVES, [0]).n_pairs == 0


@pytest.mark.parametrize("args,status", [
    ((96, HALVES, [32]), UNSUPPORTED), ((64, HALVES, [33]), INVALID), ((64, HALVES, [20, 16]), INVALID),
    ((64, HALVES, [-4]), INVALID), ((64, HALVES, [30]), INVALID), ((64, 2, [32]), INVALID), ((64, HALVES, []), INVALID),
    ((64, HALVES, [4] * 5), INVALID), ((64, HALVES, [32], False, 0.0), INVALID), ((64, HALVES, [32], False, -2.0), INVALID),
    ((64, HALVES, [32], False, math.nan), INVALID), ((64, HALVES, [32], False, math.inf), INVALID),
    ((64, HALVES, [32], False, 1e-300), INVALID), ((64, NEIGHBOURS, [BIG, BIG]), INVALID)])
def test_rotary_refusals(args, status):
    with pytest.raises(binding.MarcheError) as e:
        binding.rotary(*args)
    assert e.value.status == status


@pytest.mark.parametrize("dh", [64, 80, 128])
def test_append_fills_the_largest_launch(dh):
    """Whole workgroups of the queries', the keys' and the values' heads: one of each a row."""
    c = _cache(n_heads=1, head_dim=dh)
    rot = binding.rotary(dh, HALVES, [4])
    call = dict(heads=1, rot=rot, stride=dh, q_out_stride=dh, k=FAKE + 8)
    most = (2 ** 28 - 64) // 3
    assert _append(c, total=most, **call) == INVALID and "aligned" in binding.last_error()
    for total in (most + 1, 2 ** 28, BIG):
        assert _append(c, total=total, **call) == UNSUPPORTED and "2^28" in binding.last_error()


@pytest.mark.parametrize("call", [_window, _tree], ids=lambda c: c.__name__[1:])
def test_attention_refusals(call):
    for name in ("lens", "o"):
        assert call(**{name: None}) == INVALID and "NULL" in binding.last_error()
    assert call(o=FAKE + 8) == INVALID and "aligned" in binding.last_error()
    assert call(len_max=-1) == INVALID and "len_max" in binding.last_error()
    assert call(len_max=321) == INVALID
    for q_max in (-1, 0, 7):
        assert call(q_max=q_max) == INVALID and "q_max" in binding.last_error()
    assert call(off=None, q_max=4) == INVALID
    big = _cache(n_heads=1)
    assert call(big, total=2 ** 30, q_max=1, heads=1, stride=64) == UNSUPPORTED


def test_window_refusals():
    assert _window(idx=None) == INVALID and "NULL" in binding.last_error()
    for w in (0, -1, -2 ** 31):
        assert _window(window=w) == INVALID and "window" in binding.last_error()
    assert _window(sinks=-1) == INVALID and "sinks" in binding.last_error()
    long = dict(max_pages=4096, len_max=4096 * 64, total=1, q_max=1, n_seqs=1, off=None)
    n = binding.paged_attention_window_workspace_bytes(_cache(), 1, 1, 1, 8, 4096 * 64, 10 ** 6, 4)
    assert n > 0
    assert _window(window=10 ** 6, **long) == WORKSPACE and "workspace" in binding.last_error()
    assert _window(window=10 ** 6, ws=FAKE, ws_bytes=n - 1, **long) == WORKSPACE
    assert _window(window=10 ** 6, ws=FAKE + 16, ws_bytes=n, **long) == INVALID and "256" in binding.last_error()
    for bad in (dict(window=0), dict(sinks=-1), dict(n_seqs=0), dict(q_total=0), dict(q_max=0), dict(q_max=2),
                dict(n_q_heads=6), dict(len_max=-1), dict(len_max=BIG)):
        a = dict(n_seqs=1, q_total=1, q_max=1, n_q_heads=8, len_max=4096 * 64, window=10 ** 6, sinks=4)
        assert binding.paged_attention_window_workspace_bytes(_cache(), **dict(a, **bad)) == 0
    # sizes at their ends
    for w, s in ((1, 0), (BIG, 0), (BIG, BIG), (1, BIG)):
        binding.paged_attention_window_workspace_bytes(_cache(), 1, 1, 1, 8, 2 ** 30, w, s)
        assert _window(window=w, sinks=s, q=None) == INVALID and "NULL" in binding.last_error()


def test_tree_refusals():
    for name in ("ctx", "mask"):
        assert _tree(**{name: None}) == INVALID and "NULL" in binding.last_error()
    for words in (0, -1, 65, BIG):
        assert _tree(words=words) == INVALID and "mask_words" in binding.last_error()
    long = dict(max_pages=4096, len_max=4096 * 64, total=1, q_max=1, n_seqs=1, off=None)
    n = binding.paged_attention_tree_workspace_bytes(_cache(), 1, 1, 1, 8, 4096 * 64)
    assert n > 0
    assert _tree(**long) == WORKSPACE and "workspace" in binding.last_error()
    assert _tree(ws=FAKE, ws_bytes=n - 1, **long) == WORKSPACE
    assert _tree(ws=FAKE + 16, ws_bytes=n, **long) == INVALID and "256" in binding.last_error()
    for bad in (dict(n_seqs=0), dict(q_total=0), dict(q_max=2), dict(n_q_heads=6), dict(len_max=-1)):
        a = dict(n_seqs=1, q_total=1, q_max=1, n_q_heads=8, len_max=4096 * 64)
        assert binding.paged_attention_tree_workspace_bytes(_cache(), **dict(a, **bad)) == 0


def test_join_of_padded_rows_is_bounded():
    """Rows of no sequence count for the join of split caches."""
    c = _cache(n_heads=1)
    call = dict(n_seqs=1, q_max=1, heads=1, stride=64, max_pages=64, len_max=4096)
    assert _tree(c, total=2 ** 24 - 1, **call) == WORKSPACE
    assert _tree(c, total=2 ** 24, ws=FAKE, ws_bytes=1 << 40, **call) == UNSUPPORTED and "too many" in binding.last_error()
    assert _window(c, total=2 ** 24 - 1, window=4096, **call) == WORKSPACE
    assert _window(c, total=2 ** 24, window=4096, ws=FAKE, ws_bytes=1 << 40, **call) == UNSUPPORTED
    assert binding.paged_attention_window_workspace_bytes(c, 1, 2 ** 24, 1, 1, 4096, 4096, 0) == 0
