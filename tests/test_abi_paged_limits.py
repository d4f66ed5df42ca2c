"""The largest launches of the paged cache's calls (CPU only): what would need
2^32 threads is refused before any HIP call, and what just does not is judged by
its next argument."""
import pytest

from paper_2506_12035_amd import binding

from test_abi_paged import FAKE, INVALID, UNSUPPORTED, _attend, _bounds, _cache, _write, built_library  # noqa: F401


@pytest.mark.parametrize("dh,most", [(64, 2 ** 28 - 1), (80, 2 ** 28 - 16), (128, 2 ** 28 - 16)])
def test_write_fills_the_largest_launch(dh, most):
    """(row, head) pairs by whole workgroups of 32 (64 channels) or 16."""
    c = _cache(n_heads=1, head_dim=dh)
    for total, status in ((most, INVALID), (most + 1, UNSUPPORTED), (2 ** 28, UNSUPPORTED)):
        assert _write(c, total=total, stride=dh, k=FAKE + 8) == status
        assert ("aligned" if status == INVALID else "2^28") in binding.last_error()


def test_bounds_fill_the_largest_launch():
    """(page, head) pairs by whole workgroups of four."""
    c = _cache(n_heads=1)
    for n, status in ((2 ** 26 - 4, INVALID), (2 ** 26 - 3, UNSUPPORTED), (2 ** 26 - 1, UNSUPPORTED), (2 ** 26, UNSUPPORTED)):
        assert _bounds(c, n_seqs=n, span=1, lens=None) == status
        assert ("NULL" if status == INVALID else "2^26") in binding.last_error()


def test_attention_whose_join_is_too_large():
    """Rows of no sequence count for the join of split caches: one workgroup of
    256 threads for every row and query head."""
    c = _cache(n_heads=1)
    call = dict(n_seqs=1, q_max=1, heads=1, stride=64, max_pages=64, len_max=4096)
    n = binding.paged_attention_workspace_bytes(c, 1, 2 ** 24 - 1, 1, 1, 4096)
    assert n > 0
    assert _attend(c, total=2 ** 24 - 1, **call) == binding.MARCHE_ERR_WORKSPACE
    assert binding.paged_attention_workspace_bytes(c, 1, 2 ** 24, 1, 1, 4096) == 0
    assert _attend(c, total=2 ** 24, **call) == UNSUPPORTED and "too many" in binding.last_error()
    assert _attend(c, total=2 ** 24, ws=FAKE, ws_bytes=1 << 40, **call) == UNSUPPORTED
    # one key range needs no join
    call["len_max"] = 32
    assert binding.paged_attention_workspace_bytes(c, 1, 2 ** 24, 1, 1, 32) == 0
    assert _attend(c, total=2 ** 24, **dict(call, q=None)) == INVALID and "NULL" in binding.last_error()
