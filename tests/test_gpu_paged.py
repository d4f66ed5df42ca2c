"""The paged key/value cache on the GPU against the float64 oracle: writing and
reading back (exact), page bounds and selection (exact), attention over whole
caches and over selected pages, and the calls as a decoding loop makes them."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import DT, FMT, TORCH, Pool, attention, attention_errors, dev, i32, offsets, rnd

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]


# ------------------------------------------------------------------ write

def _edge_rows(n, H, dh, rng):
    """Rows whose quantisation is delicate: zeros, rows at the borders of an
    exponent, tiny and huge ones, single values, ties between two steps."""
    x = rng.standard_normal((n, H, dh)) * np.exp(rng.uniform(-3, 3, (n, H, 1)))
    flat = x.reshape(-1, dh)
    edge = [np.zeros(dh)]
    for m in (448.0, 127.0):
        for f in (1.0, 1.0 + 2.0 ** -7, 1.0 - 2.0 ** -8):
            edge.append(np.concatenate([[m * f * 2.0 ** rng.integers(-20, 20)], rng.standard_normal(dh - 1)]))
    edge += [np.full(dh, 1e-30), np.full(dh, 1e30), np.full(dh, -2.0 ** -130),
             np.concatenate([np.zeros(dh - 1), [3.0]]), np.concatenate([[127.0], np.arange(dh - 1) + 0.5]),
             np.concatenate([[448.0], 16.0 + np.arange(dh - 1)])]
    for i, e in enumerate(edge[:len(flat)]):
        flat[i] = e
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("fmt", FORMATS)
def test_write_is_exact(fmt, dh, dtype):
    say(f"paged write {fmt} {dh} {dtype}")
    rng = np.random.default_rng(dh)
    lens, rows, H, page = [40, 0, 17, 33, 5], [9, 0, 17, 1, 2], 3, 16
    pool = Pool(fmt, lens, H, dh, page, seed=1, layers=2, layer=1)
    total, extra = sum(rows), 3
    idx = np.concatenate([rng.permutation(n)[:r] for n, r in zip(lens, rows)]).astype(np.int32)
    new = [rnd(_edge_rows(total, H, dh, rng), dtype) for _ in range(2)]
    # parts of a fused projection's rows, behind other columns
    stride = 8 + 2 * H * dh
    buf = torch.full((total + extra, stride), float("nan"), dtype=TORCH[dtype], device="cuda")
    buf[:total, 8:8 + H * dh] = dev(new[0].reshape(total, -1), TORCH[dtype])
    buf[:total, 8 + H * dh:] = dev(new[1].reshape(total, -1), TORCH[dtype])
    want = [[t.copy() if t is not None else None for t in pool.layer_of(w)] for w in ("k", "v")]
    off = offsets(rows)
    for b in range(len(lens)):
        for r in range(off[b], off[b + 1]):
            at, slot = pool.table[b][idx[r] // page], idx[r] % page
            for w in range(2):
                if fmt == "bf16":
                    want[w][0][at, :, slot] = rnd(new[w][r], "bf16")
                else:
                    want[w][0][at, :, slot], want[w][1][at, :, slot] = ref.quantise(new[w][r], fmt)
    binding.paged_write(pool.cache, 1, pool.dtable, pool.width, len(lens), i32(list(idx) + [0] * extra), i32(off),
                        total + extra, buf[:, 8:], buf[:, 8 + H * dh:], stride, DT[dtype])
    torch.cuda.synchronize()
    for w, name in enumerate(("k", "v")):
        got = pool.layer_of(name)
        np.testing.assert_array_equal(got[0], want[w][0])
        if fmt != "bf16":
            np.testing.assert_array_equal(got[1], want[w][1])
    if fmt != "bf16":  # the other layer
        assert (pool.dk[0] == 0x7F).all() and (pool.dke[0] == 255).all()
    else:
        assert pool.dk[0].isnan().all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_write_of_rows_that_are_not_finite(fmt):
    say(f"paged write not finite {fmt}")
    pool = Pool(fmt, [16], 1, 64, 16)
    x = np.ones((4, 64))
    x[0, 3], x[1, 60], x[2, 0] = np.inf, np.nan, -np.inf
    d = dev(x, torch.bfloat16)
    binding.paged_write(pool.cache, 0, pool.dtable, pool.width, 1, i32([0, 1, 2, 3]), None, 4, d, d, 64, DT["bf16"])
    k = pool.seq("k", 0)
    assert np.isnan(k[:3]).all() and (k[3] == 1).all()
    assert pool.layer_of("k")[1][pool.table[0, 0], 0, :4].tolist()[:3] == [255] * 3


@pytest.mark.parametrize("fmt", FORMATS)
def test_write_drops_what_has_no_page(fmt):
    """Tokens past the page table and pages outside the pool are not written,
    negative tokens neither; equal numbers of rows need no offsets."""
    say(f"paged write drops {fmt}")
    pool = Pool(fmt, [32, 32], 2, 64, 16, width_extra=0)
    pool.table[1] = [pool.n_pages, -7]
    before = [pool.layer_of(w) for w in ("k", "v")]
    x = dev(np.ones((6, 128)), torch.bfloat16)
    tok = [32, -1, 2147483647, 0, 16, 31]
    binding.paged_write(pool.cache, 0, i32(pool.table), 2, 2, i32(tok), None, 6, x, x, 128, DT["bf16"])
    torch.cuda.synchronize()
    for w, b in zip(("k", "v"), before):
        np.testing.assert_array_equal(pool.layer_of(w)[0], b[0])


def test_write_finds_sequences_among_many():
    """Row r's sequence, with empty sequences between, for more sequences than
    one round of probes tells apart."""
    say("paged write many sequences")
    rng = np.random.default_rng(5)
    n = 700
    rows = rng.integers(0, 3, n)
    rows[100:300] = 0
    rows[-1] = 0
    pool = Pool("int8", [1] * n, 1, 64, 16, seed=3)
    total = int(rows.sum())
    x = rng.integers(-100, 100, (total, 64)) * 1.0
    x[:, 0] = 127
    idx = np.concatenate([np.arange(r) for r in rows]).astype(np.int32)
    binding.paged_write(pool.cache, 0, pool.dtable, pool.width, n, i32(idx), i32(offsets(rows)), total,
                        dev(x, torch.bfloat16), dev(-x, torch.bfloat16), 64, DT["bf16"])
    torch.cuda.synchronize()
    k, v = pool.layer_of("k")[0], pool.layer_of("v")[0]
    off = offsets(rows)
    for b in range(n):
        for r in range(off[b], off[b + 1]):
            np.testing.assert_array_equal(k[pool.table[b, 0], 0, idx[r]], x[r])
            np.testing.assert_array_equal(v[pool.table[b, 0], 0, idx[r]], -x[r])


# ------------------------------------------------------------------ read

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,page", [(64, 64), (80, 16), (128, 32)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_read_is_exact(fmt, dh, page, dtype):
    say(f"paged read {fmt} {dh} {dtype}")
    lens, n = [150, 0, 1, 129, 300], 140
    pool = Pool(fmt, lens, 2, dh, page, seed=2, layers=2, layer=1, width_extra=0)
    pool.table[3, 0] = pool.n_pages + 5  # a page outside the pool: left as it was
    out = [torch.full((5, 2, n, dh), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
    binding.paged_read(pool.cache, 1, i32(pool.table), pool.width, pool.dlens, 5, n, out[0], out[1], DT[dtype])
    torch.cuda.synchronize()
    for w, name in enumerate(("k", "v")):
        t, e = pool.layer_of(name)
        for b, length in enumerate(lens):
            m = min(length, n)
            x, ok = ref.tokens(t, e, pool.table[b], m, page)
            got = out[w][b].double().cpu().numpy()
            np.testing.assert_array_equal(got[:, :m][:, ok], x.transpose(1, 0, 2)[:, ok])
            assert (got[:, :m][:, ~ok] == 7).all() and (got[:, m:] == 7).all()


def test_read_of_lengths_past_the_table():
    say("paged read past the table")
    pool = Pool("e4m3", [32, 16], 1, 64, 16, width_extra=0)
    out = [torch.full((2, 1, 64, 64), 7.0, device="cuda") for _ in range(2)]
    binding.paged_read(pool.cache, 0, pool.dtable, 2, i32([1 << 30, -5]), 2, 64, out[0], out[1], DT["f32"])
    torch.cuda.synchronize()
    np.testing.assert_array_equal(out[1][0, 0, :32].double().cpu().numpy(), pool.seq("v", 0)[:, 0])
    assert (out[0][0, :, 32:] == 7).all() and (out[0][1] == 7).all()


# ------------------------------------------------------------------ bounds

@pytest.mark.parametrize("dh,page", [(64, 64), (80, 16), (128, 32), (64, 256)])
@pytest.mark.parametrize("fmt", FORMATS)
def test_bounds_are_exact(fmt, dh, page):
    say(f"paged bounds {fmt} {dh} {page}")
    lens = [3 * page, 0, 1, page + 7, page - 1]
    pool = Pool(fmt, lens, 3, dh, page, seed=4, layers=2, layer=1, with_bounds=True)
    pool.db[:] = 99
    pool.dbe[:] = 77
    want, code = pool.db[1].cpu().numpy().astype(float), pool.dbe[1].cpu().numpy().astype(int)

    def update(b, pages):
        k = pool.seq("k", b)
        for p in pages:
            want[pool.table[b, p]], code[pool.table[b, p]] = ref.bounds(k[p * page:(p + 1) * page])

    def check():
        torch.cuda.synchronize()
        np.testing.assert_array_equal(pool.dbe[1].cpu().numpy(), code)
        np.testing.assert_array_equal(pool.db[1].cpu().numpy(), want)
        assert (pool.db[0] == 99).all() and (pool.dbe[0] == 77).all()

    # the last page of each sequence, as after an appended token
    binding.paged_bounds(pool.cache, 1, pool.dtable, pool.width, pool.dlens, i32([max(n - 1, 0) for n in lens]), 1, 5)
    for b, n in enumerate(lens):
        update(b, [(n - 1) // page] if n else [])
    check()
    binding.paged_bounds(pool.cache, 1, pool.dtable, pool.width, pool.dlens, None, pool.width, 5)
    for b, n in enumerate(lens):
        update(b, range(-(-n // page)))
    check()


@pytest.mark.parametrize("fmt", FORMATS)
def test_bounds_of_keys_that_are_not_finite(fmt):
    say(f"paged bounds not finite {fmt}")
    pool = Pool(fmt, [48], 2, 64, 16, with_bounds=True)
    at = int(pool.table[0, 1])
    if fmt == "bf16":
        pool.dk[0, at, 1, 5, 7] = float("-inf")
        pool.dk[0, int(pool.table[0, 2]), 0, 15, 63] = float("nan")
    else:
        pool.dk[0, at, 1, 5] = 0x7F if fmt == "e4m3" else 0
        pool.dke[0, at, 1, 5] = 255
        pool.dk[0, int(pool.table[0, 2]), 0, 15] = 0x7F if fmt == "e4m3" else 0
        pool.dke[0, int(pool.table[0, 2]), 0, 15] = 255
    binding.paged_bounds(pool.cache, 0, pool.dtable, pool.width, pool.dlens, None, 3, 1)
    torch.cuda.synchronize()
    code = pool.dbe[0].cpu().numpy()[pool.table[0, :3]]
    assert (code == 255).tolist() == [[False, False], [False, True], [True, False]]


# ------------------------------------------------------------------ select

def _oracle_pages(pool, q, rows, group, n_select):
    """Pages of each row and head by the oracle, from the bounds on the device."""
    off = offsets(rows)
    bound, code = pool.db[pool.layer].cpu().numpy().astype(float), pool.dbe[pool.layer].cpu().numpy().astype(int)
    q = q.reshape(-1, pool.H, group, pool.dh)
    out = np.full((sum(rows), pool.H, n_select), -1, np.int32)
    for b, n in enumerate(pool.lens):
        at = pool.table[b][:-(-n // pool.page)]
        for r in range(off[b], off[b + 1]):
            for h in range(pool.H):
                out[r, h] = ref.select(ref.scores(q[r, h], bound[at, h], code[at, h]), n_select)
    return out


def _select(pool, q, rows, group, n_select, dtype, off="csr", tail=0):
    D = pool.H * group * pool.dh
    total = sum(rows)
    pages = torch.full((total + tail, pool.H, n_select), -5, dtype=torch.int32, device="cuda")
    binding.paged_select(pool.cache, pool.layer, pool.dtable, pool.width, pool.dlens, len(rows), q, D,
                         i32(offsets(rows)) if off == "csr" else None, total + tail, pool.H * group, DT[dtype],
                         n_select, pages)
    torch.cuda.synchronize()
    assert (pages[total:] == -5).all()
    return pages[:total]


SELECT_CASES = [
    # lens, rows, group, heads, dh, page, n_select
    ([700], [1], 4, 2, 128, 16, 7),
    ([330, 0, 17, 160, 16], [5, 2, 1, 0, 3], 1, 3, 64, 16, 4),
    ([100, 300, 250], [1, 1, 1], 7, 2, 80, 32, 3),
    ([2000, 900], [2, 3], 20, 1, 64, 16, 11),
    ([16 * 1500 + 1], [2], 2, 1, 64, 16, 300),
    ([16 * 4095], [1], 1, 1, 80, 16, 64),
    ([64, 64, 64], [6, 6, 6], 1, 1, 64, 16, 9),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SELECT_CASES, ids=lambda c: "n{}r{}g{}d{}k{}".format(max(c[0]), sum(c[1]), c[2], c[4], c[6]))
def test_selected_pages_are_exact(case, dtype):
    lens, rows, group, heads, dh, page, k = case
    say(f"paged select {case} {dtype}")
    rng = np.random.default_rng(7)
    pool = Pool("e4m3", lens, heads, dh, page, seed=8, with_bounds=True, layers=2, layer=1)
    binding.paged_bounds(pool.cache, 1, pool.dtable, pool.width, pool.dlens, None, pool.width, len(lens))
    q = rnd(rng.standard_normal((sum(rows), heads * group * dh)), dtype)
    got = _select(pool, dev(np.concatenate([q, q[:1] * 0]), TORCH[dtype]), rows, group, k, dtype, tail=1)
    np.testing.assert_array_equal(got.cpu().numpy(), _oracle_pages(pool, q, rows, group, k))


def test_select_ties_and_values_that_are_not_finite():
    """Zero queries tie everywhere, equal pages tie in pairs; NaN ranks last."""
    say("paged select ties")
    pool = Pool("int8", [16 * 8] * 3, 1, 64, 16, with_bounds=True, width_extra=0)
    pool.db[:] = 3
    pool.dbe[:] = 127
    pool.dbe[0, torch.from_numpy(pool.table[1, [0, 3]].astype(np.int64)).cuda()] = 255
    pool.db[0, torch.from_numpy(pool.table[2, [5, 6]].astype(np.int64)).cuda()] = 9
    q = np.zeros((3, 64))
    q[1:] = 1
    d = dev(q, torch.bfloat16)
    pages = _select(pool, d, [1, 1, 1], 1, 3, "bf16", off=None).cpu().numpy()[:, 0].tolist()
    assert pages == [[0, 1, 2], [1, 2, 4], [0, 5, 6]]
    d[1, 5] = float("nan")
    d[2, 9] = float("inf")
    pages = _select(pool, d, [1, 1, 1], 1, 3, "bf16", off=None).cpu().numpy()[:, 0].tolist()
    assert pages == [[0, 1, 2]] * 3


# ------------------------------------------------------------------ attention

ATTEND_CASES = [
    # lens, rows, group, heads, page
    ([1], [1], 1, 1, 16),
    ([0, 1, 15, 16, 17], [1, 1, 1, 1, 1], 1, 2, 16),
    ([31, 32, 33, 64, 65], [1, 2, 1, 3, 1], 4, 2, 32),
    ([1000], [1], 8, 1, 64),
    ([4097, 100], [1, 1], 4, 2, 64),
    ([320], [17], 1, 2, 64),
    ([200, 0, 333], [33, 4, 0], 1, 2, 128),
    ([77, 500], [16, 70], 1, 1, 16),
    ([256, 90], [5, 11], 7, 1, 256),
    ([130], [150], 1, 1, 32),
    ([20], [2], 71, 1, 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", ATTEND_CASES, ids=lambda c: "n{}r{}g{}p{}".format(max(c[0]), sum(c[1]), c[2], c[4]))
def test_attention_parity(case, fmt, dh, dtype):
    lens, rows, group, heads, page = case
    say(f"paged attention {case} {fmt} {dh} {dtype}")
    pool = Pool(fmt, lens, heads, dh, page, seed=11, layers=2, layer=1)
    rng = np.random.default_rng(12)
    q = rnd(2 * rng.standard_normal((sum(rows), heads * group * dh)), dtype)
    got = attention(pool, dev(q, TORCH[dtype]), rows, group, dtype).double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = attention_errors(pool, got, q, rows, group, dtype)
    say(f"  worst error / allowed {worst:.3f}")
    assert worst <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_layout_of_rows(dtype):
    """Rows behind other columns, rows of no sequence left as they were, equal
    numbers of rows without offsets."""
    say(f"paged attention layout {dtype}")
    pool = Pool("e4m3", [50, 40], 2, 64, 16, seed=1)
    rng = np.random.default_rng(2)
    q = rnd(rng.standard_normal((6, 128)), dtype)
    wide = torch.full((6, 3 * 128 + 8), float("nan"), dtype=TORCH[dtype], device="cuda")
    wide[:, 8:136] = dev(q, TORCH[dtype])
    a = attention(pool, wide[:, 8:], [3, 3], 1, dtype, off=None, q_stride=392)
    b = attention(pool, dev(q, TORCH[dtype]), [3, 3], 1, dtype)
    assert torch.equal(a, b)
    assert attention_errors(pool, a.double().cpu().numpy(), q, [3, 3], 1, dtype) <= 1
    o = torch.full((6, 128), 7.0, dtype=TORCH[dtype], device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    binding.paged_attention(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 50, 2, dev(q, TORCH[dtype]), 128,
                            i32([1, 2, 4]), 6, 2, 2, DT[dtype], o, None, 0, ws, 1 << 20)
    torch.cuda.synchronize()
    assert (o[0] == 7).all() and (o[4:] == 7).all() and not (o[1:4] == 7).any()


def test_attention_of_rows_between_sequences_on_a_split_cache():
    """The same where the parts of a long cache are joined."""
    say("paged attention layout, split")
    pool = Pool("int8", [3000, 2000], 1, 64, 64, seed=1)
    rng = np.random.default_rng(2)
    q = rnd(rng.standard_normal((4, 64)), "bf16")
    n = binding.paged_attention_workspace_bytes(pool.cache, 2, 4, 1, 1, 3000)
    assert n > 0
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    o = torch.full((4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    binding.paged_attention(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 3000, 2, dev(q, torch.bfloat16), 64,
                            i32([1, 2, 3]), 4, 1, 1, DT["bf16"], o, None, 0, ws, n)
    torch.cuda.synchronize()
    assert (o[0] == 7).all() and (o[3] == 7).all()
    assert attention_errors(pool, o[1:3].double().cpu().numpy(), q[1:3], [1, 1], 1, "bf16") <= 1


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_of_extreme_logits(fmt):
    """Logits far apart, growing along the cache (every tile raises the
    maximum), falling along it, and a row of zeros."""
    say(f"paged attention extreme logits {fmt}")
    pool = Pool(fmt, [600], 1, 64, 32, seed=3, scale=6.0)
    k = pool.seq("k", 0)[:, 0]
    q = rnd(np.stack([k[0] * 2, k[-1] * 2, -k[300] * 2, np.zeros(64)]), "bf16")
    got = attention(pool, dev(q, torch.bfloat16), [4], 1, "bf16").double().cpu().numpy()
    assert attention_errors(pool, got, q, [4], 1, "bf16") <= 1


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_shows_values_that_are_not_finite(fmt):
    """A key or value that is not finite reaches the rows of its sequence and
    head, and no other."""
    say(f"paged attention not finite {fmt}")
    pool = Pool(fmt, [100, 100, 100], 2, 64, 16, seed=5)
    at = [int(pool.table[b, 2]) for b in range(3)]
    if fmt == "bf16":
        pool.dk[0, at[0], 1, 3, 9] = float("nan")
        pool.dv[0, at[1], 0, 3] = float("nan")
    else:
        for t, e, b, h in ((pool.dk, pool.dke, 0, 1), (pool.dv, pool.dve, 1, 0)):
            t[0, at[b], h, 3] = 0x7F if fmt == "e4m3" else 0
            e[0, at[b], h, 3] = 255
    rng = np.random.default_rng(2)
    q = rnd(rng.standard_normal((3, 128)), "bf16")
    o = attention(pool, dev(q, torch.bfloat16), [1, 1, 1], 1, "bf16").view(3, 2, 64)
    assert torch.equal(o.isnan().all(-1).cpu(), torch.tensor([[False, True], [True, False], [False, False]]))
    assert torch.equal(o.isnan().any(-1), o.isnan().all(-1))


def test_attention_of_all_minus_infinite_logits():
    """A key group whose logits are all -inf counts nothing; a row with
    nothing else is 0 / 0, a row without keys zero."""
    say("paged attention -inf logits")
    pool = Pool("bf16", [1024, 64, 0], 1, 64, 64, seed=6)
    q = np.ones((3, 64))
    for b, n in ((0, 992), (1, 64)):
        for p in range(-(-n // 64)):
            pool.dk[0, int(pool.table[b, p]), 0, :min(64, n - 64 * p)] = float("-inf")
    got = attention(pool, dev(q, torch.bfloat16), [1, 1, 1], 1, "bf16").double().cpu().numpy()
    k, v = pool.seq("k", 0)[992:, 0], pool.seq("v", 0)[992:, 0]
    o, a, _ = ref.attention(q[:1], k, v)
    assert (np.abs(got[0] - o[0]) <= 2.0 ** -8 * (np.abs(o[0]) + 1.01 * a[0])).all()
    assert np.isnan(got[1]).all() and (got[2] == 0).all()


def test_attention_skips_pages_outside_the_pool():
    say("paged attention bad pages")
    pool = Pool("e4m3", [64, 16], 1, 64, 16, seed=7)
    bad = pool.table.copy()
    bad[0, 1], bad[0, 3], bad[1, 0] = pool.n_pages, -3, 1 << 30
    pool.dtable = i32(bad)
    rng = np.random.default_rng(2)
    q = rnd(rng.standard_normal((2, 64)), "bf16")
    got = attention(pool, dev(q, torch.bfloat16), [1, 1], 1, "bf16").double().cpu().numpy()
    look = np.repeat(np.array([1, 0, 1, 0], bool), 16)[None]
    o, a, _ = ref.attention(q[:1], pool.seq("k", 0)[:, 0], pool.seq("v", 0)[:, 0], look)
    assert (np.abs(got[0] - o[0]) <= 2.0 ** -8 * (np.abs(o[0]) + 1.01 * a[0])).all()
    assert (got[1] == 0).all()


# ------------------------------------------------------------------ attention over selected pages

def _look(pool, pages, rows):
    """Which tokens each row and head may look at, per sequence."""
    off, pages = offsets(rows), np.asarray(pages)
    out = []
    for b, n in enumerate(pool.lens):
        look = np.zeros((rows[b], pool.H, n), bool)
        for i in range(rows[b]):
            for h in range(pool.H):
                for p in pages[off[b] + i, h]:
                    if 0 <= p < -(-n // pool.page):
                        look[i, h, p * pool.page:(p + 1) * pool.page] = True
        out.append(look)
    return out


PAGES_CASES = [
    # lens, rows, group, heads, dh, page, n_select
    ([900], [1], 4, 2, 128, 16, 9),
    ([5000, 4000], [1, 1], 4, 1, 128, 64, 20),
    ([400, 0, 17, 50], [3, 2, 1, 2], 1, 2, 64, 16, 3),
    ([300], [40], 1, 1, 80, 32, 2),
    ([500, 120], [70, 20], 1, 1, 64, 16, 4),
    ([260], [9], 7, 1, 64, 64, 2),
    ([900], [30], 3, 1, 128, 16, 5),
    ([6000], [2], 2, 1, 80, 32, 40),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", PAGES_CASES, ids=lambda c: "n{}r{}g{}d{}k{}".format(max(c[0]), sum(c[1]), c[2], c[4], c[6]))
def test_attention_over_listed_pages(case, fmt, dtype):
    """Random lists: repeated pages, -1, pages behind the sequence, rows
    without a page."""
    lens, rows, group, heads, dh, page, k = case
    say(f"paged attention of pages {case} {fmt} {dtype}")
    pool = Pool(fmt, lens, heads, dh, page, seed=13, layers=2, layer=1)
    rng = np.random.default_rng(14)
    pages = rng.integers(-1, pool.width + 1, (sum(rows), heads, k)).astype(np.int32)
    pages[0, 0] = -1
    q = rnd(2 * rng.standard_normal((sum(rows), heads * group * dh)), dtype)
    got = attention(pool, dev(q, TORCH[dtype]), rows, group, dtype, i32(pages)).double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = attention_errors(pool, got, q, rows, group, dtype, _look(pool, pages, rows))
    say(f"  worst error / allowed {worst:.3f}")
    assert worst <= 1


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_that_are_not_looked_at_do_not_matter(fmt):
    """Infinities and NaN in keys and values of a page reach the rows that list
    it and no other row of the block."""
    say(f"paged attention of pages, not finite elsewhere {fmt}")
    pool = Pool(fmt, [96], 1, 64, 16, seed=15)
    at = int(pool.table[0, 2])
    if fmt == "bf16":
        pool.dk[0, at, 0, 4, 5] = float("nan")
        pool.dv[0, at, 0, 7] = float("inf")
    else:
        for t, e, j in ((pool.dk, pool.dke, 4), (pool.dv, pool.dve, 7)):
            t[0, at, 0, j] = 0x7F if fmt == "e4m3" else 0
            e[0, at, 0, j] = 255
    rng = np.random.default_rng(16)
    q = rnd(rng.standard_normal((5, 64)), "bf16")
    pages = np.array([[0, 1], [1, 2], [3, 4], [5, 0], [2, 2]], np.int32).reshape(5, 1, 2)
    got = attention(pool, dev(q, torch.bfloat16), [5], 1, "bf16", i32(pages)).double().cpu().numpy()
    assert np.isnan(got).all(1).tolist() == [False, True, False, False, True]
    fine = [0, 2, 3]
    assert np.isfinite(got[fine]).all()
    k, v = pool.seq("k", 0)[:, 0], pool.seq("v", 0)[:, 0]
    look = _look(pool, pages, [5])[0][:, 0]
    o, a, _ = ref.attention(q[fine], k, v, look[fine])
    assert (np.abs(got[fine] - o) <= 2.0 ** -8 * (np.abs(o) + 1.01 * a)).all()


# ------------------------------------------------------------------ together

class Loop:
    """A decoding loop on one cache: sequences of different lengths, one new
    token each per step, written, bounded, selected for and attended to."""

    def __init__(self, fmt, dtype="bf16", lens=(75, 16, 1, 40), steps=4, group=2, heads=2, dh=64, page=16,
                 n_select=3, seed=0):
        self.steps, self.group, self.dtype, self.k = steps, group, dtype, n_select
        self.n = len(lens)
        full = [n + steps for n in lens]
        self.pool = Pool(fmt, full, heads, dh, page, seed=seed, with_bounds=True, layers=2, layer=1)
        p = self.pool
        rng = np.random.default_rng(seed + 1)
        D = heads * dh
        self.qkv = [dev(rnd(rng.standard_normal((self.n, (group + 2) * D)), dtype), TORCH[dtype]) for _ in range(steps)]
        self.D = D
        self.lens = [i32([n + s + 1 for n in lens]) for s in range(steps)]
        self.host_lens = [[n + s + 1 for n in lens] for s in range(steps)]
        self.last = [i32([n + s for n in lens]) for s in range(steps)]
        self.len0 = i32(lens)
        self.len_max = max(full)
        self.pages = torch.empty(self.n, heads, n_select, dtype=torch.int32, device="cuda")
        self.o = torch.empty(2, self.n, group * D, dtype=TORCH[dtype], device="cuda")
        self.ws_bytes = max(binding.paged_attention_workspace_bytes(p.cache, self.n, self.n, 1, heads * group,
                                                                    self.len_max, x) for x in (0, n_select))
        self.ws = torch.empty(max(256, self.ws_bytes), dtype=torch.uint8, device="cuda")

    def start(self, stream=None):
        p = self.pool
        binding.paged_bounds(p.cache, 1, p.dtable, p.width, self.len0, None, p.width, self.n, stream=stream)

    def step(self, s, stream=None):
        p, D, W = self.pool, self.D, self.qkv[s].shape[1]
        new = self.qkv[s]
        q, k, v = new, new[:, self.group * D:], new[:, (self.group + 1) * D:]
        heads = p.H * self.group
        binding.paged_write(p.cache, 1, p.dtable, p.width, self.n, self.last[s], None, self.n, k, v, W, DT[self.dtype],
                            stream=stream)
        binding.paged_bounds(p.cache, 1, p.dtable, p.width, self.lens[s], self.last[s], 1, self.n, stream=stream)
        binding.paged_select(p.cache, 1, p.dtable, p.width, self.lens[s], self.n, q, W, None, self.n, heads,
                             DT[self.dtype], self.k, self.pages, stream=stream)
        for i, (pages, k_sel) in enumerate(((None, 0), (self.pages, self.k))):
            binding.paged_attention(p.cache, 1, p.dtable, p.width, self.lens[s], self.len_max, self.n, q, W, None,
                                    self.n, 1, heads, DT[self.dtype], self.o[i], pages, k_sel, self.ws, self.ws_bytes,
                                    stream=stream)


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("int8", "f32")])
def test_decoding_loop(fmt, dtype):
    say(f"paged decoding loop {fmt} {dtype}")
    run = Loop(fmt, dtype)
    p, D = run.pool, run.D
    run.start()
    for s in range(run.steps):
        run.step(s)
        torch.cuda.synchronize()
        new = run.qkv[s].double().cpu().numpy()
        p.lens = run.host_lens[s]
        for b in range(run.n):
            x = new[b, run.group * D:].reshape(2, p.H, p.dh)
            for w, name in enumerate(("k", "v")):
                want = x[w] if fmt == "bf16" else ref.value(*ref.quantise(x[w], fmt))
                np.testing.assert_array_equal(p.seq(name, b)[-1], rnd(want, "bf16") if fmt == "bf16" else want)
        q = new[:, :run.group * D]
        rows = [1] * run.n
        np.testing.assert_array_equal(run.pages.cpu().numpy(), _oracle_pages(p, q, rows, run.group, run.k))
        for b in range(run.n):  # the bounds that the step kept up to date
            k = p.seq("k", b)
            for pg in range(-(-p.lens[b] // p.page)):
                want, code = ref.bounds(k[pg * p.page:(pg + 1) * p.page])
                np.testing.assert_array_equal(p.db[1, int(p.table[b, pg])].cpu().numpy(), want)
        look = _look(p, run.pages.cpu().numpy(), rows)
        assert attention_errors(p, run.o[0].double().cpu().numpy(), q, rows, run.group, dtype) <= 1
        assert attention_errors(p, run.o[1].double().cpu().numpy(), q, rows, run.group, dtype, look) <= 1


def test_captured_steps_replay():
    """Two captured steps that share a workspace, replayed between eager work
    on the same pool, give the eager results every time."""
    say("paged captured steps")
    want = []
    eager = Loop("e4m3", lens=(3000, 1500, 7), n_select=12, page=32)
    eager.start()
    for s in range(eager.steps):
        eager.step(s)
        torch.cuda.synchronize()
        want.append((eager.o.clone(), eager.pages.clone()))
    run = Loop("e4m3", lens=(3000, 1500, 7), n_select=12, page=32)
    assert run.ws_bytes > 0
    side = torch.cuda.Stream()
    graphs = []
    run.start()
    run.step(0)
    torch.cuda.synchronize()
    for s in (1, 2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            run.step(s, stream=torch.cuda.current_stream())
        graphs.append((s, g))
    for _ in range(3):
        for s, g in graphs:
            run.o.fill_(float("nan"))
            run.pages.fill_(-9)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(run.o, want[s][0]) and torch.equal(run.pages, want[s][1])
        run.step(3)
        torch.cuda.synchronize()
        assert torch.equal(run.o, want[3][0])
        run.start()
        torch.cuda.synchronize()
        # step 3's token lies behind the lengths of the steps before it, but in
        # the pages that they bound
        run.step(1)
        torch.cuda.synchronize()
        assert torch.equal(run.o, want[1][0]) and torch.equal(run.pages, want[1][1])


def test_two_streams_with_workspaces_of_their_own():
    say("paged two streams")
    runs = [Loop(f, lens=(2000, 900), n_select=8, seed=i) for i, f in enumerate(("int8", "bf16"))]
    want = []
    for r in runs:
        r.start()
        r.step(0)
        torch.cuda.synchronize()
        want.append(r.o.clone())
        r.o.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(4):
        for r, st in zip(runs, streams):
            r.step(0, stream=st)
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        assert torch.equal(r.o, w)


def test_pool_past_32_bits():
    """Pages whose byte and element offsets pass 2^32."""
    say("paged pool past 32 bits")
    H, dh, page, n_pages = 8, 128, 64, 70000  # 70000 * 8 * 64 * 128 = 4.59e9 elements
    shape = (n_pages, H, page, dh)
    k = torch.empty(shape, dtype=torch.uint8, device="cuda")
    v = torch.empty(shape, dtype=torch.uint8, device="cuda")
    ke = torch.empty(shape[:3], dtype=torch.uint8, device="cuda")
    ve = torch.empty(shape[:3], dtype=torch.uint8, device="cuda")
    bd = torch.empty(n_pages, H, 2, dh, dtype=torch.int8, device="cuda")
    be = torch.empty(n_pages, H, dtype=torch.uint8, device="cuda")
    cache = binding.paged_cache(1, n_pages, H, page, dh, FMT["int8"], k, v, ke, ve, bd, be)
    table = np.array([[n_pages - 1, 3, n_pages - 2, 65536]], np.int32)
    n = 4 * page
    rng = np.random.default_rng(1)
    x = rnd(rng.standard_normal((n, 3, H, dh)), "bf16")
    d = dev(x.reshape(n, -1), torch.bfloat16)
    D = H * dh
    binding.paged_write(cache, 0, i32(table), 4, 1, i32(np.arange(n)), None, n, d[:, D:], d[:, 2 * D:], 3 * D, DT["bf16"])
    lens = i32([n])
    out = [torch.empty(1, H, n, dh, device="cuda") for _ in range(2)]
    binding.paged_read(cache, 0, i32(table), 4, lens, 1, n, out[0], out[1], DT["f32"])
    binding.paged_bounds(cache, 0, i32(table), 4, lens, None, 4, 1)
    pages = torch.empty(n, H, 4, dtype=torch.int32, device="cuda")
    binding.paged_select(cache, 0, i32(table), 4, lens, 1, d, 3 * D, None, n, H, DT["bf16"], 4, pages)
    o = [torch.empty(n, D, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    wb = max(binding.paged_attention_workspace_bytes(cache, 1, n, n, H, n, s) for s in (0, 4))
    ws = torch.empty(max(wb, 256), dtype=torch.uint8, device="cuda")
    for i, (pg, s) in enumerate(((None, 0), (pages, 4))):
        binding.paged_attention(cache, 0, i32(table), 4, lens, n, 1, d, 3 * D, None, n, n, H, DT["bf16"], o[i], pg, s,
                                ws, wb)
    torch.cuda.synchronize()
    kv = [ref.value(*ref.quantise(x[:, w], "int8")) for w in (1, 2)]
    for w in range(2):
        np.testing.assert_array_equal(out[w][0].double().cpu().numpy(), kv[w].transpose(1, 0, 2))
    assert (pages.cpu().numpy() == np.arange(4)).all()
    want, code = ref.bounds(kv[0][page:2 * page])
    np.testing.assert_array_equal(bd[3].cpu().numpy(), want)
    ref_o, a, dl = ref.attention(x[:, 0, 2], kv[0][:, 2], kv[1][:, 2])
    allow = 2.0 ** -8 * (np.abs(ref_o) + a) + a * (2 * (dh + 8) * dl[:, None] + n + 64) * 2.0 ** -24
    for t in o:
        assert (np.abs(t.double().cpu().numpy().reshape(n, H, dh)[:, 2] - ref_o) <= allow).all()


def test_cache_in_one_buffer():
    """marche_paged_cache_init's parts, used through a write and a read."""
    say("paged cache in one buffer")
    n = binding.paged_cache_bytes(2, 5, 3, 16, 80, FMT["int8"], True)
    buf = torch.zeros(n, dtype=torch.uint8, device="cuda")
    cache = binding.paged_cache_init(2, 5, 3, 16, 80, FMT["int8"], True, buf, n)
    rng = np.random.default_rng(3)
    x = rnd(rng.standard_normal((20, 240)), "bf16")
    d = dev(x, torch.bfloat16)
    table, lens = i32([[4, 1]]), i32([20])
    binding.paged_write(cache, 1, table, 2, 1, i32(np.arange(20)), None, 20, d, -d, 240, DT["bf16"])
    out = [torch.zeros(1, 3, 20, 80, device="cuda") for _ in range(2)]
    binding.paged_read(cache, 1, table, 2, lens, 1, 20, out[0], out[1], DT["f32"])
    torch.cuda.synchronize()
    want = ref.value(*ref.quantise(x.reshape(20, 3, 80), "int8")).transpose(1, 0, 2)
    np.testing.assert_array_equal(out[0][0].double().cpu().numpy(), want)
    np.testing.assert_array_equal(out[1][0].double().cpu().numpy(), -want)


def test_cached_tokens_meet_the_segment_attention():
    """What the cache reads back is the cached segment of the two-segment
    attention, which then agrees with the attention over the cache itself."""
    say("paged read into segment attention")
    B, H, dh, n_c, n_a = 2, 4, 64, 256, 32
    pool = Pool("e4m3", [n_c, n_c], H, dh, 64, seed=21, extra=4)
    rng = np.random.default_rng(22)
    bf = torch.bfloat16
    kc, vc = (torch.empty(B, H, n_c, dh, dtype=bf, device="cuda") for _ in range(2))
    binding.paged_read(pool.cache, 0, pool.dtable, pool.width, pool.dlens, B, n_c, kc, vc, DT["bf16"])
    q = rnd(rng.standard_normal((B * n_a, H * dh)), "bf16")
    o = torch.empty(B, n_a, H * dh, dtype=bf, device="cuda")
    binding.attention_segments(dev(q, bf), o, n_a, None, None, 0, kc, vc, n_c, B, H, dh, DT["bf16"],
                               binding.MARCHE_ATTN_TWO_SEGMENT)
    got = attention(pool, dev(q, bf), [n_a, n_a], 1, "bf16")
    assert attention_errors(pool, got.double().cpu().numpy(), q, [n_a, n_a], 1, "bf16") <= 1
    assert attention_errors(pool, o.view(B * n_a, -1).double().cpu().numpy(), q, [n_a, n_a], 1, "bf16") <= 1


# ------------------------------------------------------------------ large calls, many sequences

@pytest.mark.parametrize("fmt,dtype,H,dh", [("e4m3", "bf16", 16, 64), ("int8", "f32", 8, 80), ("bf16", "f32", 4, 128),
                                            ("int8", "bf16", 16, 64)])
def test_large_writes_and_reads_are_small_ones_together(fmt, dtype, H, dh):
    """Rows and outputs of more than 64 MB at once and in pieces: the same bytes."""
    say(f"paged large write and read {fmt} {dtype} {dh}")
    page, n_seqs = 64, 20
    elem = 2 if dtype == "bf16" else 4
    n = 1 + 64_000_000 // (2 * H * dh * elem * n_seqs)
    per = -(-n // page)
    n_pages = n_seqs * per
    es, new = (2, torch.bfloat16) if fmt == "bf16" else (1, torch.uint8)
    table = i32(np.random.default_rng(1).permutation(n_pages).reshape(n_seqs, per))
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(n_seqs * n, 2 * H * dh, device="cuda", generator=g).to(TORCH[dtype])
    idx = i32(np.tile(np.arange(n), n_seqs))
    off = offsets([n] * n_seqs)
    pools = []
    for pieces in (1, n_seqs):
        kv = [torch.zeros(n_pages, H, page, dh, dtype=new, device="cuda") for _ in range(2)]
        ex = [torch.zeros(n_pages, H, page, dtype=torch.uint8, device="cuda") for _ in range(2)] if es == 1 else [None] * 2
        cache = binding.paged_cache(1, n_pages, H, page, dh, FMT[fmt], *kv, *ex, None, None)
        if pieces == 1:
            binding.paged_write(cache, 0, table, per, n_seqs, idx, i32(off), n_seqs * n, x, x[:, H * dh:], 2 * H * dh, DT[dtype])
        else:
            for b in range(n_seqs):
                r = x[off[b]:off[b + 1]]
                binding.paged_write(cache, 0, table[b:], per, 1, idx, None, n, r, r[:, H * dh:], 2 * H * dh, DT[dtype])
        torch.cuda.synchronize()
        pools.append(kv + [e for e in ex if e is not None])
    for a, b in zip(*pools):
        assert torch.equal(a, b)
    lens = i32([n - (b % 3) for b in range(n_seqs)])
    whole = [torch.full((n_seqs, H, n, dh), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
    parts = [torch.full((n_seqs, H, n, dh), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
    binding.paged_read(cache, 0, table, per, lens, n_seqs, n, whole[0], whole[1], DT[dtype])
    for b in range(n_seqs):
        binding.paged_read(cache, 0, table[b:], per, lens[b:], 1, n, parts[0][b], parts[1][b], DT[dtype])
    torch.cuda.synchronize()
    for a, b in zip(whole, parts):
        assert torch.equal(a, b)
    some = slice(3 * n + 5, 3 * n + 45)  # and right: sequence 3's tokens 5 .. 44
    for w in range(2):
        rows = x[some, w * H * dh:(w + 1) * H * dh].double().cpu().numpy().reshape(40, H, dh)
        want = rows if fmt == "bf16" else ref.value(*ref.quantise(rows, fmt))
        np.testing.assert_array_equal(whole[w][3, :, 5:45].double().cpu().numpy().transpose(1, 0, 2),
                                      rnd(want, "bf16") if fmt == "bf16" else want)


@pytest.mark.parametrize("fmt,dh", [("e4m3", 64), ("int8", 80), ("bf16", 128)])
def test_large_bounds_are_small_ones_together(fmt, dh):
    """Bounds of more than 128 MB of keys at once and sequence by sequence."""
    say(f"paged large bounds {fmt} {dh}")
    H, page, n_seqs, es = 16, 64, 24, 2 if fmt == "bf16" else 1
    per = 1 + 128_000_000 // (H * page * dh * es * n_seqs)
    n_pages = n_seqs * per
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(n_pages, H, page, dh, device="cuda", generator=g)
    if fmt == "bf16":
        k, ke = x.bfloat16(), None
    else:
        k = x.to(torch.float8_e4m3fn).view(torch.uint8) if fmt == "e4m3" else (40 * x).clamp(-127, 127).to(torch.int8).view(torch.uint8)
        ke = torch.randint(120, 131, (n_pages, H, page), generator=g, device="cuda", dtype=torch.uint8)
    out = []
    table = i32(np.random.default_rng(1).permutation(n_pages).reshape(n_seqs, per))
    lens = i32([per * page - 7 * b for b in range(n_seqs)])
    for pieces in (1, n_seqs):
        bd = torch.zeros(n_pages, H, 2, dh, dtype=torch.int8, device="cuda")
        be = torch.zeros(n_pages, H, dtype=torch.uint8, device="cuda")
        cache = binding.paged_cache(1, n_pages, H, page, dh, FMT[fmt], k, k, ke, ke, bd, be)
        for b in range(pieces):
            binding.paged_bounds(cache, 0, table[b:], per, lens[b:], None, per, n_seqs // pieces)
        torch.cuda.synchronize()
        out.append((bd, be))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    p = int(table[2, 1])
    keys = k[p].double().cpu().numpy() if fmt == "bf16" else ref.value(
        k[p].view(torch.float8_e4m3fn if fmt == "e4m3" else torch.int8).float().cpu().numpy().astype(np.float64),
        ke[p].cpu().numpy().astype(np.int64))
    want, code = ref.bounds(keys.transpose(1, 0, 2))
    np.testing.assert_array_equal(out[0][0][p].cpu().numpy(), want)
    np.testing.assert_array_equal(out[0][1][p].cpu().numpy(), code)


MANY_CASES = [
    # sequences, rows of each, dtype: caches cut into ranges of one length (up to
    # 256 sequences) or each by itself
    (65, 1, "bf16"), (100, 1, "f32"), (128, 1, "bf16"), (200, 20, "bf16"), (256, 20, "bf16"), (257, 20, "bf16"), (70, 20, "f32"),
]


@pytest.mark.parametrize("n,rows,dtype", MANY_CASES)
def test_attention_of_many_uneven_sequences(n, rows, dtype):
    say(f"paged attention of {n} sequences, {rows} rows, {dtype}")
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 40, n)
    lens[rng.permutation(n)[:n // 8]] = 0
    lens[rng.permutation(n)[:5]] = rng.integers(300, 1500, 5)
    lens[-1] = 1700
    pool = Pool("e4m3", lens.tolist(), 1, 64, 32, seed=9)
    q = rnd(2 * rng.standard_normal((n * rows, 64)), dtype)
    for off in ("csr", None):
        got = attention(pool, dev(q, TORCH[dtype]), [rows] * n, 1, dtype, off=off).double().cpu().numpy()
        assert np.isfinite(got).all()
        assert attention_errors(pool, got, q, [rows] * n, 1, dtype) <= 1


def test_attention_of_nothing_cached():
    """Every sequence empty, len_max 0: zeros, whatever the pool holds."""
    say("paged attention, nothing cached")
    pool = Pool("bf16", [0, 0, 0], 2, 64, 16)
    q = dev(np.ones((5, 256)), torch.bfloat16)
    for pages in (None, i32(np.zeros((5, 2, 3)))):
        o = attention(pool, q, [3, 0, 2], 2, "bf16", pages, len_max=0)
        assert (o == 0).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_sequences_that_share_pages(fmt):
    """Two sequences with a common first part in the same pages, and one that is
    the common part alone."""
    say(f"paged shared pages {fmt}")
    pool = Pool(fmt, [90, 70, 32], 2, 64, 16, seed=4, with_bounds=True)
    pool.table[1, :2] = pool.table[2, :2] = pool.table[0, :2]
    pool.dtable = i32(pool.table)
    binding.paged_bounds(pool.cache, 0, pool.dtable, pool.width, pool.dlens, None, pool.width, 3)
    rng = np.random.default_rng(6)
    rows = [2, 1, 3]
    q = rnd(rng.standard_normal((6, 256)), "bf16")
    pages = _select(pool, dev(q, torch.bfloat16), rows, 2, 3, "bf16")
    np.testing.assert_array_equal(pages.cpu().numpy(), _oracle_pages(pool, q, rows, 2, 3))
    for pg in (None, pages):
        got = attention(pool, dev(q, torch.bfloat16), rows, 2, "bf16", pg).double().cpu().numpy()
        look = None if pg is None else _look(pool, pages.cpu().numpy(), rows)
        assert attention_errors(pool, got, q, rows, 2, "bf16", look) <= 1


@pytest.mark.parametrize("big,small", [(118, 40), (40, 118)])
def test_scores_of_far_exponents(big, small):
    """Scores within range whose factors, applied one by one, are not."""
    say(f"paged select, exponents {big} {small}")
    pool = Pool("int8", [16 * 8] * 2, 1, 64, 16, with_bounds=True)
    rng = np.random.default_rng(8)
    pool.db[:] = dev(rng.integers(-127, 128, pool.db.shape).astype(np.int8))
    pool.dbe[:] = 127 + big
    q = rnd(rng.standard_normal((2, 64)) * 2.0 ** -small, "bf16")
    if big < small:
        pool.dbe[:] = 127 - small
        q = rnd(rng.standard_normal((2, 64)) * 2.0 ** big, "bf16")
    pages = _select(pool, dev(q, torch.bfloat16), [1, 1], 1, 3, "bf16")
    np.testing.assert_array_equal(pages.cpu().numpy(), _oracle_pages(pool, q, [1, 1], 1, 3))


# ------------------------------------------------------------------ debug validation

@pytest.mark.parametrize("bad,word", [
    (dict(lens=[65, 40]), "length"), (dict(lens=[-1, 40]), "length"), (dict(page=99), "page outside"),
    (dict(off=[0, 3, 2]), "offsets"), (dict(off=[0, 1, 3]), "offsets"), (dict(pages=4), "selected page"),
    (dict(), None)])
def test_validated_attention(monkeypatch, bad, word):
    say(f"paged validate attention {bad}")
    monkeypatch.setenv("MARCHE_VALIDATE", "1")
    pool = Pool("bf16", [64, 40], 1, 64, 16, width_extra=0)
    table = pool.table.copy()
    if "page" in bad:
        table[1, 2] = bad["page"]
    pages = i32(np.full((2, 1, 1), bad.get("pages", 1)))
    q = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    o = torch.zeros_like(q)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def call():
        binding.paged_attention(pool.cache, 0, i32(table), 4, i32(bad.get("lens", [64, 40])), 64, 2, q, 64,
                                i32(bad.get("off", [0, 1, 2])), 2, 1, 1, DT["bf16"], o, pages, 1, ws, 1 << 20)

    if word is None:
        call()
        return
    with pytest.raises(binding.MarcheError, match=word) as e:
        call()
    assert e.value.status == binding.MARCHE_ERR_INVALID_ARG


@pytest.mark.parametrize("idx,word", [([0, 5, 5, 1], "twice"), ([0, 5, 64, 1], "token out"), ([0, -1, 6, 1], "token out"),
                                      ([0, 5, 6, 50], "page outside"), ([0, 5, 6, 1], None)])
def test_validated_write(monkeypatch, idx, word):
    say(f"paged validate write {idx}")
    monkeypatch.setenv("MARCHE_VALIDATE", "1")
    pool = Pool("int8", [64, 40], 1, 64, 16, width_extra=0)
    x = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")

    def call():
        binding.paged_write(pool.cache, 0, pool.dtable, 4, 2, i32(idx), i32([0, 3, 4]), 4, x, x, 64, DT["bf16"])

    if word is None:
        call()
        return
    with pytest.raises(binding.MarcheError, match=word):
        call()


def test_validation_takes_what_the_calls_take(monkeypatch):
    """Rows of no sequence before and behind the others, and the first token of
    an empty sequence."""
    say("paged validate padding")
    monkeypatch.setenv("MARCHE_VALIDATE", "1")
    pool = Pool("int8", [64, 0], 1, 64, 16, width_extra=0, with_bounds=True)
    x = torch.ones(6, 64, dtype=torch.bfloat16, device="cuda")
    o = torch.full_like(x, 7.0)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    off, bf = i32([1, 3, 4]), DT["bf16"]
    binding.paged_write(pool.cache, 0, pool.dtable, 4, 2, i32([-1, 3, 9, 5, 99, 99]), i32([1, 3, 3]), 6, x, x, 64, bf)
    binding.paged_bounds(pool.cache, 0, pool.dtable, 4, pool.dlens, i32([63, -1]), 1, 2)
    pages = torch.full((6, 1, 2), -5, dtype=torch.int32, device="cuda")
    binding.paged_select(pool.cache, 0, pool.dtable, 4, pool.dlens, 2, x, 64, off, 6, 1, bf, 2, pages)
    binding.paged_attention(pool.cache, 0, pool.dtable, 4, pool.dlens, 64, 2, x, 64, off, 6, 2, 1, bf, o, pages, 2, ws, 1 << 20)
    torch.cuda.synchronize()
    assert (o[[0, 4, 5]] == 7).all() and (o[3] == 0).all() and not (o[1:3] == 7).any()
    assert (pages[[0, 4, 5]] == -5).all() and (pages[3] == -1).all()
