"""The paged cache's calls without a GPU: sizes, and what they refuse on the
host before any HIP call (CPU only; no kernel is launched)."""
import ctypes as C
import os

import pytest

from paper_2506_12035_amd import binding, build

FAKE = 0x10000000  # never dereferenced: validation fails first, or there is nothing to do
OK, INVALID, UNSUPPORTED, WORKSPACE = (binding.MARCHE_OK, binding.MARCHE_ERR_INVALID_ARG,
                                       binding.MARCHE_ERR_UNSUPPORTED, binding.MARCHE_ERR_WORKSPACE)
INT8, BF16C = binding.MARCHE_CACHE_INT8, binding.MARCHE_CACHE_BF16


@pytest.fixture(scope="module", autouse=True)
def built_library():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def _cache(**kw):
    base = dict(n_layers=2, n_pages=10, n_heads=4, page_size=64, head_dim=64, fmt=INT8, k=FAKE, v=FAKE, k_exp=FAKE,
                v_exp=FAKE, bounds=FAKE, bounds_exp=FAKE)
    base.update(kw)
    return binding.paged_cache(**base)


def _write(cache=None, **kw):
    a = dict(layer=1, table=FAKE, max_pages=5, n_seqs=2, idx=FAKE, off=FAKE, total=6, k=FAKE, v=FAKE, stride=256,
             dtype=binding.MARCHE_BF16)
    a.update(kw)
    return binding.lib().marche_paged_write(C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"],
                                            a["n_seqs"], a["idx"], a["off"], a["total"], a["k"], a["v"], a["stride"],
                                            a["dtype"], None)


def _read(cache=None, **kw):
    a = dict(layer=0, table=FAKE, max_pages=5, lens=FAKE, n_seqs=2, n=100, k=FAKE, v=FAKE, dtype=binding.MARCHE_F32)
    a.update(kw)
    return binding.lib().marche_paged_read(C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"],
                                           a["lens"], a["n_seqs"], a["n"], a["k"], a["v"], a["dtype"], None)


def _bounds(cache=None, **kw):
    a = dict(layer=0, table=FAKE, max_pages=5, lens=FAKE, first=None, span=5, n_seqs=2)
    a.update(kw)
    return binding.lib().marche_paged_bounds(C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"],
                                             a["lens"], a["first"], a["span"], a["n_seqs"], None)


def _select(cache=None, **kw):
    a = dict(layer=0, table=FAKE, max_pages=5, lens=FAKE, n_seqs=2, q=FAKE, stride=512, off=FAKE, total=6, heads=8,
             dtype=binding.MARCHE_BF16, k=3, pages=FAKE)
    a.update(kw)
    return binding.lib().marche_paged_select(C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"],
                                             a["lens"], a["n_seqs"], a["q"], a["stride"], a["off"], a["total"],
                                             a["heads"], a["dtype"], a["k"], a["pages"], None)


def _attend(cache=None, **kw):
    a = dict(layer=0, table=FAKE, max_pages=5, lens=FAKE, len_max=320, n_seqs=2, q=FAKE, stride=512, off=FAKE,
             total=6, q_max=4, heads=8, dtype=binding.MARCHE_BF16, o=FAKE, pages=None, k=0, ws=None, ws_bytes=0)
    a.update(kw)
    return binding.lib().marche_paged_attention(C.byref(cache or _cache()), a["layer"], a["table"], a["max_pages"],
                                                a["lens"], a["len_max"], a["n_seqs"], a["q"], a["stride"], a["off"],
                                                a["total"], a["q_max"], a["heads"], a["dtype"], a["o"], a["pages"],
                                                a["k"], a["ws"], a["ws_bytes"], None)


CALLS = [_write, _read, _bounds, _select, _attend]


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__[1:])
@pytest.mark.parametrize("kw,status,word", [
    (dict(n_layers=0), INVALID, "n_layers"), (dict(n_pages=0), INVALID, "n_pages"), (dict(n_heads=0), INVALID, "n_heads"),
    (dict(page_size=48), UNSUPPORTED, "page_size"), (dict(page_size=8), UNSUPPORTED, "page_size"),
    (dict(page_size=512), UNSUPPORTED, "page_size"), (dict(page_size=-64), UNSUPPORTED, "page_size"),
    (dict(head_dim=96), UNSUPPORTED, "head_dim"), (dict(fmt=3), UNSUPPORTED, "format"), (dict(fmt=-1), UNSUPPORTED, "format"),
    (dict(n_pages=2147483647, n_heads=60000, page_size=256), UNSUPPORTED, "2^50"),
    (dict(k=None), INVALID, "cache.k"), (dict(v_exp=None), INVALID, "v_exp"), (dict(k=FAKE + 8), INVALID, "aligned"),
    (dict(k_exp=FAKE + 4), INVALID, "aligned"), (dict(bounds_exp=None), INVALID, "bounds"),
    (dict(bounds=FAKE + 8), INVALID, "aligned")])
def test_cache_is_checked(call, kw, status, word):
    assert call(_cache(**kw)) == status
    assert word in binding.last_error()


@pytest.mark.parametrize("call", CALLS, ids=lambda c: c.__name__[1:])
def test_shared_arguments_are_checked(call):
    assert call(layer=-1) == INVALID and "layer" in binding.last_error()
    assert call(layer=2) == INVALID
    assert call(max_pages=0) == INVALID and "max_pages" in binding.last_error()
    assert call(n_seqs=-1) == INVALID
    assert call(table=None) == INVALID and "NULL" in binding.last_error()


def test_write_refusals():
    assert _write(dtype=2) == UNSUPPORTED and "dtype" in binding.last_error()
    assert _write(total=-1) == INVALID
    assert _write(n_seqs=0) == INVALID
    assert _write(off=None, total=5) == INVALID and "multiple" in binding.last_error()
    assert _write(stride=255) == INVALID and "stride" in binding.last_error()
    assert _write(stride=260) == INVALID
    assert _write(stride=-512) == INVALID
    for name in ("idx", "k", "v"):
        assert _write(**{name: None}) == INVALID
    for name in ("k", "v"):
        assert _write(**{name: FAKE + 8}) == INVALID and "aligned" in binding.last_error()
    assert _write(total=1 << 29) == UNSUPPORTED  # 2^29 rows of 4 heads
    assert _write(total=1 << 26) == UNSUPPORTED and "2^28" in binding.last_error()
    assert _write(total=0) == OK
    assert _write(total=0, n_seqs=0) == OK
    # a bf16 cache has no exponents, a cache that is only written no bounds
    assert _write(_cache(fmt=BF16C, k_exp=None, v_exp=None, bounds=None, bounds_exp=None), total=0) == OK


def test_read_refusals():
    assert _read(dtype=7) == UNSUPPORTED
    assert _read(n=-1) == INVALID and "n_tokens" in binding.last_error()
    for name in ("lens", "k", "v"):
        assert _read(**{name: None}) == INVALID
    assert _read(k=FAKE + 2) == INVALID and "aligned" in binding.last_error()
    assert _read(n_seqs=1 << 16, n=1 << 24) == UNSUPPORTED
    assert _read(n_seqs=1 << 22, n=1) == UNSUPPORTED and "2^24" in binding.last_error()
    assert _read(n_seqs=2147483647, n=2147483647) == UNSUPPORTED
    assert _read(n=0) == OK and _read(n_seqs=0) == OK


def test_bounds_refusals():
    assert _bounds(_cache(bounds=None, bounds_exp=None)) == INVALID and "bounds" in binding.last_error()
    assert _bounds(span=-1) == INVALID and "span" in binding.last_error()
    assert _bounds(lens=None) == INVALID
    assert _bounds(n_seqs=1 << 25, max_pages=1 << 20, span=1 << 20) == UNSUPPORTED
    assert _bounds(n_seqs=1 << 24, span=1) == UNSUPPORTED and "2^26" in binding.last_error()
    assert _bounds(_cache(n_heads=65535, n_pages=4, page_size=16), n_seqs=2147483647, max_pages=2147483647,
                   span=2147483647) == UNSUPPORTED
    assert _bounds(span=0) == OK and _bounds(n_seqs=0) == OK


def test_select_refusals():
    assert _select(_cache(bounds=None, bounds_exp=None)) == INVALID and "bounds" in binding.last_error()
    assert _select(dtype=5) == UNSUPPORTED
    assert _select(heads=6) == INVALID and "n_q_heads" in binding.last_error()
    assert _select(heads=0) == INVALID
    assert _select(stride=504) == INVALID and "stride" in binding.last_error()
    assert _select(k=0) == INVALID and "n_select" in binding.last_error()
    assert _select(k=4097) == INVALID
    assert _select(max_pages=4097) == UNSUPPORTED and "max_pages" in binding.last_error()
    assert _select(off=None, total=5) == INVALID
    for name in ("lens", "q", "pages"):
        assert _select(**{name: None}) == INVALID
    assert _select(q=FAKE + 4) == INVALID
    assert _select(total=1 << 28) == UNSUPPORTED
    assert _select(total=1 << 27) == UNSUPPORTED and "2^30" in binding.last_error()
    assert _select(total=1 << 24, max_pages=4096) == UNSUPPORTED and "too many" in binding.last_error()
    assert _select(total=0) == OK


def test_attention_refusals():
    assert _attend(dtype=3) == UNSUPPORTED
    assert _attend(heads=2) == INVALID and "n_q_heads" in binding.last_error()
    assert _attend(stride=511) == INVALID
    assert _attend(len_max=321) == INVALID and "len_max" in binding.last_error()
    assert _attend(len_max=-1) == INVALID
    assert _attend(max_pages=1 << 26, len_max=2147483647) == UNSUPPORTED
    assert _attend(q_max=0) == INVALID and _attend(q_max=7) == INVALID
    assert _attend(off=None, q_max=4) == INVALID and "q_max" in binding.last_error()
    assert _attend(k=3) == INVALID and "n_select" in binding.last_error()
    assert _attend(pages=FAKE) == INVALID and _attend(pages=FAKE, k=5000) == INVALID
    assert _attend(pages=FAKE, k=2, max_pages=4097) == UNSUPPORTED
    for name in ("lens", "q", "o"):
        assert _attend(**{name: None}) == INVALID
    assert _attend(q=FAKE + 8) == INVALID and _attend(o=FAKE + 8) == INVALID
    assert _attend(ws=FAKE + 64, ws_bytes=1 << 30) == INVALID
    assert _attend(total=1 << 22, q_max=1 << 22, n_seqs=8192, heads=4, stride=256) == UNSUPPORTED and "too many" in binding.last_error()
    assert _attend(total=1 << 27) == UNSUPPORTED and "2^30" in binding.last_error()
    assert _attend(total=0, q_max=0) == OK


def test_attention_workspace():
    """Long caches with few rows are split: the workspace holds the parts, and
    a short one is refused before anything runs."""
    c = _cache()
    n = binding.paged_attention_workspace_bytes(c, 1, 1, 1, 8, 32768)
    assert n > 0 and n % 256 == 0
    call = dict(n_seqs=1, total=1, q_max=1, max_pages=512, len_max=32768)
    assert _attend(c, **call) == WORKSPACE and "workspace" in binding.last_error()
    assert _attend(c, ws=FAKE, ws_bytes=256, **call) == WORKSPACE
    assert binding.paged_attention_workspace_bytes(c, 64, 64 * 320, 320, 8, 320) == 0
    # sizes alone decide: a pool that is not there yet will do
    assert binding.paged_attention_workspace_bytes(_cache(k=None, v=None, k_exp=None, v_exp=None, bounds=None), 1, 1, 1,
                                                   8, 32768) == n
    for bad in (dict(n_seqs=-1), dict(n_seqs=0), dict(q_total=0), dict(q_max=0), dict(q_max=2), dict(n_q_heads=6), dict(len_max=-1),
                dict(len_max=2147483647), dict(n_select=-1), dict(n_select=4097), dict(q_total=1 << 27)):
        a = dict(n_seqs=1, q_total=1, q_max=1, n_q_heads=8, len_max=100, n_select=0)
        a.update(bad)
        assert binding.paged_attention_workspace_bytes(c, **a) == 0


def test_cache_in_one_buffer():
    up = lambda v: (v + 255) // 256 * 256  # noqa: E731
    args = (2, 5, 3, 16, 80)
    kv, ex, bd, be = up(2 * 5 * 3 * 16 * 80), up(2 * 5 * 3 * 16), up(2 * 5 * 3 * 160), up(2 * 5 * 3)
    assert binding.paged_cache_bytes(*args, INT8, True) == 2 * kv + 2 * ex + bd + be
    assert binding.paged_cache_bytes(*args, INT8, False) == 2 * kv + 2 * ex
    assert binding.paged_cache_bytes(*args, BF16C, False) == 2 * up(2 * 5 * 3 * 16 * 80 * 2)
    assert binding.paged_cache_bytes(2, 5, 3, 20, 80, INT8, True) == 0
    assert binding.paged_cache_bytes(2147483647, 2147483647, 65535, 256, 128, BF16C, True) == 0
    n = 2 * kv + 2 * ex + bd + be
    c = binding.paged_cache_init(*args, INT8, True, FAKE, n)
    assert [c.k, c.v, c.k_exp, c.v_exp, c.bounds, c.bounds_exp] == [
        FAKE + x for x in (0, kv, 2 * kv, 2 * kv + ex, 2 * kv + 2 * ex, 2 * kv + 2 * ex + bd)]
    assert (c.n_layers, c.n_pages, c.n_heads, c.page_size, c.head_dim, c.format) == (*args, INT8)
    c = binding.paged_cache_init(*args, BF16C, False, FAKE, 2 * up(2 * 5 * 3 * 16 * 80 * 2))
    assert c.k_exp is None and c.bounds is None and c.bounds_exp is None
    for bad in (dict(nbytes=n - 1), dict(buffer=None), dict(buffer=FAKE + 8)):
        a = dict(buffer=FAKE, nbytes=n)
        a.update(bad)
        with pytest.raises(binding.MarcheError):
            binding.paged_cache_init(*args, INT8, True, a["buffer"], a["nbytes"])
    with pytest.raises(binding.MarcheError, match="UNSUPPORTED"):
        binding.paged_cache_init(2, 5, 3, 16, 72, INT8, True, FAKE, n)
    assert binding.lib().marche_paged_cache_init(None, *args, INT8, 1, FAKE, n) == INVALID


def test_cache_handle_keeps_its_tensors_alive():
    import gc
    import weakref

    import torch

    t = [torch.ones(4) for _ in range(6)]
    probes = [weakref.ref(x) for x in t]
    c = binding.paged_cache(1, 1, 1, 16, 64, INT8, *t)
    del t
    gc.collect()
    assert all(r() is not None for r in probes)
    del c
    gc.collect()
    assert all(r() is None for r in probes)
