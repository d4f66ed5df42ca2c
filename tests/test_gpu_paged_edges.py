"""The paged key/value cache on the GPU at the ends of its types' ranges."""
import numpy as np
import pytest
import torch

from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import DT, Pool, attention, attention_errors, dev, i32, rnd

pytestmark = pytest.mark.gpu

F32_MAX = float(np.finfo(np.float32).max)


# ------------------------------------------------------------------ select

@pytest.mark.parametrize("n_pages", [8, 70])
def test_scores_below_the_range_rank_above_nan(n_pages):
    """Scores of finite queries and keys past float32's range on the negative
    side are numbers, and NaN ranks below every number."""
    say(f"paged select, scores below the range, {n_pages} pages")
    pool = Pool("int8", [16 * n_pages], 1, 64, 16, with_bounds=True, width_extra=0)
    pool.db[:] = -3
    pool.dbe[:] = 127 + 100
    pool.dbe[0, torch.from_numpy(pool.table[0, [0, 3]].astype(np.int64)).cuda()] = 255
    q = dev(np.full((1, 64), 2.0 ** 100), torch.bfloat16)
    numbers = [p for p in range(n_pages) if p not in (0, 3)]
    for k, want in ((2, numbers[:2]), (n_pages - 2, numbers), (n_pages - 1, [0] + numbers)):
        pages = torch.full((1, 1, k), -5, dtype=torch.int32, device="cuda")
        binding.paged_select(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 1, q, 64, None, 1, 1, DT["bf16"], k,
                             pages)
        assert pages[0, 0].tolist() == want


# ------------------------------------------------------------------ rows of no sequence

@pytest.mark.parametrize("validate", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_behind_the_last_sequence_need_not_be_there(monkeypatch, dtype, validate):
    """Totals of a larger batch over buffers that end with the last sequence's rows."""
    say(f"paged rows that are not there {dtype} {validate}")
    if validate:
        monkeypatch.setenv("MARCHE_VALIDATE", "1")
    pool = Pool("int8", [40, 0, 17], 2, 64, 16, seed=1, with_bounds=True)
    off, n, total = i32([1, 4, 4, 6]), 6, 1 << 20
    rng = np.random.default_rng(2)
    x = dev(rng.standard_normal((n, 128)), torch.bfloat16 if dtype == "bf16" else torch.float32)
    idx = i32([-1, 39, 0, 5, 16, 2])
    binding.paged_bounds(pool.cache, 0, pool.dtable, pool.width, pool.dlens, None, pool.width, 3)
    out = []
    for rows in (n, total):
        pages = torch.full((n, 2, 2), -5, dtype=torch.int32, device="cuda")
        o = torch.full((n, 128), 7.0, dtype=x.dtype, device="cuda")
        binding.paged_write(pool.cache, 0, pool.dtable, pool.width, 3, idx, off, rows, x, x, 128, DT[dtype])
        binding.paged_select(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 3, x, 128, off, rows, 2, DT[dtype], 2, pages)
        binding.paged_attention(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 40, 3, x, 128, off, rows, 3, 2,
                                DT[dtype], o, pages, 2)
        torch.cuda.synchronize()
        assert (pages[0] == -5).all() and (o[0] == 7).all() and not (o[1:] == 7).any()
        out.append((pages, o, pool.layer_of("k")[0], pool.layer_of("v")[0]))
        assert (pool.seq("k", 0)[39] != 0).any()
    for a, b in zip(*out):
        np.testing.assert_array_equal(np.asarray(torch.as_tensor(a).double().cpu()), np.asarray(torch.as_tensor(b).double().cpu()))


# ------------------------------------------------------------------ fp32 queries

@pytest.mark.parametrize("rows", [1, 20])
@pytest.mark.parametrize("dh", [64, 80, 128])
def test_largest_fp32_queries(dh, rows):
    """Finite queries above the largest bf16 over keys so small that the logits
    are ordinary: every part of a query is finite."""
    say(f"paged attention, largest fp32 queries {dh} {rows}")
    pool = Pool("bf16", [90], 1, dh, 16, seed=31)
    rng = np.random.default_rng(32)
    for p in pool.table[0, :6]:  # two channels' keys, normal bf16 numbers
        for d in {0, min(dh - 1, 70)}:
            pool.dk[0, int(p), 0, :, d] = dev(rng.uniform(0.25, 1, 16) * rng.choice([-1, 1], 16) * 2.0 ** -122,
                                              torch.bfloat16)
    q = rnd(rng.standard_normal((rows, dh)), "f32")
    q[:, 0], q[:, min(dh - 1, 70)] = F32_MAX, -F32_MAX * rng.uniform(0.998, 1, rows).astype(np.float32)
    q = rnd(q, "f32")
    assert np.isfinite(q).all() and np.isinf(rnd(q, "bf16")).any()
    pages = i32(np.broadcast_to(np.arange(6, dtype=np.int32), (rows, 1, 6)).copy())
    for pg in (None, pages):
        got = attention(pool, dev(q, torch.float32), [rows], 1, "f32", pg).double().cpu().numpy()
        assert np.isfinite(got).all()
        assert attention_errors(pool, got, q, [rows], 1, "f32") <= 1
