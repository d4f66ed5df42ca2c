"""The paged key/value cache on the GPU at the ends of its types' ranges."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import DT, TORCH, Pool, attention, attention_errors, dev, i32, offsets, rnd

pytestmark = pytest.mark.gpu

F32_MAX = float(np.finfo(np.float32).max)
BF16_MAX = 255 * 2.0 ** 120


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


# ------------------------------------------------------------------ infinite keys and values

# lens, rows, group, dh, every row lists: None, or pages of the cache
INF_CASES = [
    ([200], [1], 1, 64, None), ([200], [40], 1, 80, None), ([90, 130], [3, 5], 3, 128, None),
    ([3000, 40], [1, 1], 2, 64, None),               # split
    ([200], [1], 1, 80, 5), ([300], [9], 2, 64, 5),  # a block of one row, of several
    ([2500], [1], 1, 128, 150), ([2500], [3], 1, 64, 150),
]


def _inf_pool(lens, dh):
    """A bf16 cache in which every seventh key is -inf in one channel."""
    pool = Pool("bf16", lens, 1, dh, 16, seed=41)
    off = []
    for b, n in enumerate(lens):
        bad = np.arange(2, n, 7)
        for j in bad:
            pool.dk[0, int(pool.table[b, j // 16]), 0, j % 16, (5 * j) % dh] = float("-inf")
        off.append(bad)
    return pool, off


def _lists(lens, rows, n_list, rng):
    if n_list is None:
        return None
    out = [np.sort(rng.permutation(-(-n // 16))[:n_list]) for n, r in zip(lens, rows) for _ in range(r)]
    return np.stack(out).astype(np.int32)[:, None]


def _looked_at(pages, lens, rows):
    if pages is None:
        return [np.ones((r, 1, n), bool) for n, r in zip(lens, rows)]
    off = offsets(rows)
    out = []
    for b, n in enumerate(lens):
        look = np.zeros((rows[b], 1, n), bool)
        for i in range(rows[b]):
            look[i, 0] = np.isin(np.arange(n) // 16, pages[off[b] + i, 0])
        out.append(look)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", INF_CASES, ids=lambda c: "n{}r{}g{}d{}k{}".format(max(c[0]), sum(c[1]), *c[2:]))
def test_keys_of_minus_infinity_count_nothing(case, dtype):
    """Logits of -inf beside finite ones have weight zero (queries positive, so
    that -inf keys give -inf; ones and halves, whose lower parts are zeros)."""
    lens, rows, group, dh, n_list = case
    say(f"paged attention, keys of -inf {case} {dtype}")
    pool, bad = _inf_pool(lens, dh)
    rng = np.random.default_rng(42)
    q = rnd(np.abs(rng.standard_normal((sum(rows), group * dh))) * 0.3 + 0.01, dtype)
    q[0] = 1.0
    q[-1, ::2] = 0.5
    pages = _lists(lens, rows, n_list, rng)
    look = _looked_at(pages, lens, rows)
    for b, j in enumerate(bad):
        look[b][:, :, j] = False
    got = attention(pool, dev(q, TORCH[dtype]), rows, group, dtype, None if pages is None else i32(pages))
    got = got.double().cpu().numpy()
    pool.dk[pool.dk == float("-inf")] = 0.0  # (of keys that are not looked at below)
    assert np.isfinite(got).all()
    assert attention_errors(pool, got, q, rows, group, dtype, look) <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_whose_logits_are_all_minus_infinity(dtype):
    """0 / 0, beside rows with a finite logit and rows without a key."""
    say(f"paged attention, all logits -inf {dtype}")
    pool = Pool("bf16", [1024, 64, 0], 1, 64, 64, seed=6)
    for b, n in ((0, 992), (1, 64)):
        for p in range(-(-n // 64)):
            pool.dk[0, int(pool.table[b, p]), 0, :min(64, n - 64 * p)] = float("-inf")
    q = np.ones((3, 64))
    got = attention(pool, dev(q, TORCH[dtype]), [1, 1, 1], 1, dtype).double().cpu().numpy()
    assert np.isnan(got[1]).all() and (got[2] == 0).all()
    pool.dk[pool.dk == float("-inf")] = 0.0
    look = [np.arange(1024)[None, None] >= 992, np.zeros((1, 1, 64), bool), np.zeros((1, 1, 0), bool)]
    got[1] = 0.0
    assert attention_errors(pool, got, q, [1, 1, 1], 1, dtype, look) <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", INF_CASES, ids=lambda c: "n{}r{}g{}d{}k{}".format(max(c[0]), sum(c[1]), *c[2:]))
def test_infinite_values_reach_their_channel(case, dtype):
    """An infinite value with a weight above zero makes its channel infinite
    for the rows that look at it, and changes nothing else."""
    lens, rows, group, dh, n_list = case
    say(f"paged attention, infinite values {case} {dtype}")
    pool = Pool("bf16", lens, 1, dh, 16, seed=43)
    rng = np.random.default_rng(44)
    places = [[(n // 2, 3, 1), (n - 1, dh - 1, -1), (1, 40, 1)] for n in lens]  # token, channel, sign
    for b, some in enumerate(places):
        for j, d, sign in some:
            pool.dv[0, int(pool.table[b, j // 16]), 0, j % 16, d] = sign * float("inf")
    q = rnd(0.5 * rng.standard_normal((sum(rows), group * dh)), dtype)
    q[0] = 0.0  # weights that are all the same
    pages = _lists(lens, rows, n_list, rng)
    look = _looked_at(pages, lens, rows)
    got = attention(pool, dev(q, TORCH[dtype]), rows, group, dtype, None if pages is None else i32(pages))
    got = got.double().cpu().numpy().reshape(sum(rows), group, dh)
    want = np.zeros_like(got)
    off = offsets(rows)
    for b, some in enumerate(places):
        for j, d, sign in some:
            for i in range(rows[b]):
                if look[b][i, 0, j]:
                    want[off[b] + i, :, d] = sign * np.inf
    np.testing.assert_array_equal(np.where(np.isinf(got), got, 0.0), want)
    # the other channels, whatever these hold
    for d in (3, 40, dh - 1):
        pool.dv[..., d] = 0.0
        got[..., d] = 0.0
    assert attention_errors(pool, got, q, rows, group, dtype, look) <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_queries_that_are_not_finite_stay_among_themselves(fmt, dtype):
    """NaN and infinite queries in blocks whose rows list pages of their own, one
    of which holds a value that is not finite."""
    say(f"paged attention, queries that are not finite {fmt} {dtype}")
    for lens, rows, group, k in (([300], [9], 2, 5), ([2500, 70], [3, 4], 1, 4), ([2500], [3], 1, 150)):
        pool = Pool(fmt, lens, 1, 64, 16, seed=61)
        rng = np.random.default_rng(62)
        pages = _lists(lens, rows, k, rng)
        look = _looked_at(pages, lens, rows)
        q = rnd(rng.standard_normal((sum(rows), group * 64)), dtype)
        q[0, 5], q[2, 64 * group - 1] = np.nan, np.inf
        bad = np.zeros((sum(rows), group), bool)
        bad[0, 0] = bad[2, group - 1] = True
        for poisoned in (False, True):
            if poisoned:  # token 1 of the first sequence: rows that list page 0 are NaN whole
                at = int(pool.table[0, 0])
                if fmt == "bf16":
                    pool.dv[0, at, 0, 1] = float("nan")
                else:
                    pool.dv[0, at, 0, 1] = 0x7F if fmt == "e4m3" else 0
                    pool.dve[0, at, 0, 1] = 255
                bad[:rows[0]] |= look[0][:, 0, 1][:, None]
            got = attention(pool, dev(q, TORCH[dtype]), rows, group, dtype, i32(pages)).double().cpu().numpy()
            got = got.reshape(sum(rows), group, 64)
            assert np.array_equal(np.isnan(got).all(-1), bad) and np.array_equal(np.isnan(got).any(-1), bad)
            if poisoned:  # (the oracle's own zero weights times NaN)
                pool.dv[0, at, 0, 1] = 0
                if fmt != "bf16":
                    pool.dve[0, at, 0, 1] = 127
            fine = np.where(bad.repeat(64, 1), 0.0, q)  # queries of zero in place of those that are not finite
            want = np.where(bad[..., None], 0.0, got)
            for b, off in enumerate(offsets(rows)[:-1]):
                for i in range(rows[b]):
                    for g in range(group):
                        if bad[off + i, g]:
                            o, _, _ = ref.attention(fine[off + i, 64 * g:64 * g + 64][None], pool.seq("k", b)[:, 0],
                                                    pool.seq("v", b)[:, 0], look[b][i])
                            want[off + i, g] = o[0]
            assert attention_errors(pool, want, fine, rows, group, dtype, look) <= 1


# ------------------------------------------------------------------ the largest finite rows

def _top_rows(dh):
    """Finite float32 rows whose values next to 2^128 must not be rounded to it."""
    rng = np.random.default_rng(51)
    top = [F32_MAX, BF16_MAX, 1.9375 * 2.0 ** 127, 1.984375 * 2.0 ** 127, 1.96875 * 2.0 ** 127, 1.875 * 2.0 ** 127,
           1.75 * 2.0 ** 127, 1.9921875 * 2.0 ** 127]
    x = rng.uniform(-1, 1, (2 * len(top), 1, dh)) * 2.0 ** 127
    for i, t in enumerate(top):
        x[i, 0, i], x[i + len(top), 0, -1 - i] = t, -t
    x[:len(top), 0, 20:30] = np.linspace(-1, 1, 10) * BF16_MAX
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_largest_finite_rows_stay_finite(fmt, dh, dtype):
    say(f"paged write and read, largest rows {fmt} {dh} {dtype}")
    x = rnd(np.clip(_top_rows(dh), -BF16_MAX, BF16_MAX) if dtype == "bf16" else _top_rows(dh), dtype)
    assert np.isfinite(x).all()
    n = len(x)
    pool = Pool(fmt, [n], 1, dh, 16, seed=1)
    d = dev(x.reshape(n, dh), TORCH[dtype])
    binding.paged_write(pool.cache, 0, pool.dtable, pool.width, 1, i32(np.arange(n)), None, n, d, -d, dh, DT[dtype])
    out = [torch.zeros(1, 1, n, dh, dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16) for _ in range(2)]
    for i, t in ((0, "f32"), (2, "bf16")):
        binding.paged_read(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 1, n, out[i], out[i + 1], DT[t])
    torch.cuda.synchronize()
    q, code = ref.quantise(x, fmt)
    want = ref.value(q, code)
    assert (np.abs(want) < 2.0 ** 128).all()
    for name, sign in (("k", 1), ("v", -1)):
        got = pool.layer_of(name)
        np.testing.assert_array_equal(pool.seq(name, 0), sign * want)
        assert np.array_equal(got[1][pool.table[0, 0], 0], code[:16, 0])
    for i, t in enumerate(out):
        np.testing.assert_array_equal(t[0, 0].double().cpu().numpy(), (-1) ** i * want[:, 0])


def test_largest_keys_and_queries_in_bounds_and_scores():
    """Bounds and the selection's queries are INT8 rows, the largest among them."""
    say("paged bounds and select, largest values")
    x = rnd(np.clip(_top_rows(64), -BF16_MAX, BF16_MAX), "bf16")
    pool = Pool("bf16", [16 * 9], 1, 64, 16, seed=2, with_bounds=True)
    for p in range(9):
        pool.dk[0, int(pool.table[0, p]), 0, 3] = dev(x[p, 0] * 2.0 ** -(p % 3), torch.bfloat16)
    binding.paged_bounds(pool.cache, 0, pool.dtable, pool.width, pool.dlens, None, pool.width, 1)
    torch.cuda.synchronize()
    k = pool.seq("k", 0)
    at = pool.table[0, :9]
    for p in range(9):
        want, code = ref.bounds(k[16 * p:16 * p + 16])
        np.testing.assert_array_equal(pool.db[0, int(at[p])].cpu().numpy(), want)
        np.testing.assert_array_equal(pool.dbe[0, int(at[p])].cpu().numpy(), code)
    assert pool.dbe.max() == 249
    # scores within float32: queries at the top over small bounds
    rng = np.random.default_rng(3)
    pool.db[:] = dev(rng.integers(-127, 128, pool.db.shape).astype(np.int8))
    pool.dbe[:] = 30
    bound, code = pool.db[0].cpu().numpy().astype(float), pool.dbe[0].cpu().numpy().astype(int)
    for dtype in ("bf16", "f32"):
        q = x[:, 0] if dtype == "bf16" else rnd(_top_rows(64)[:, 0], "f32")
        n = len(q)
        pages = torch.zeros(n, 1, 4, dtype=torch.int32, device="cuda")
        binding.paged_select(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 1, dev(q, TORCH[dtype]), 64, None, n, 1,
                             DT[dtype], 4, pages)
        want = [ref.select(ref.scores(q[r][None], bound[at, 0], code[at, 0]), 4) for r in range(n)]
        assert pages[:, 0].tolist() == want


def test_largest_query_beside_the_largest_of_the_exponent_below():
    """Rows that share a call are quantised each by itself: 127 * 2^121 is 127
    beside a row that reaches past it."""
    say("paged select, two largest queries")
    pool = Pool("int8", [32], 1, 64, 16, with_bounds=True)
    pool.dbe[:] = 30
    a, b = (int(p) for p in pool.table[0, :2])
    pool.db[0, a, 0, 0, 0], pool.db[0, b, 0, 0, 1] = 100, 125  # 100 * 127 against 125 * 101
    q = np.zeros((2, 64))
    q[0, 5] = BF16_MAX
    q[1, :2] = 127 * 2.0 ** 121, 101 * 2.0 ** 121
    for dtype in ("bf16", "f32"):
        pages = torch.full((2, 1, 1), -5, dtype=torch.int32, device="cuda")
        binding.paged_select(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 1, dev(q, TORCH[dtype]), 64, None, 2, 1,
                             DT[dtype], 1, pages)
        assert pages[1, 0].tolist() == [0]
