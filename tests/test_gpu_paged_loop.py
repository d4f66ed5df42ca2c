"""Positions, windows and drafted trees on the paged cache on the GPU against the
float64 oracle, and the calls together as a loop that drafts makes them."""
import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2506_12035_amd import binding

from gpu_util import say
from paged_util import DT, TORCH, Pool, attention_errors, dev, i32, offsets, rnd

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "int8"]
LAYOUT = {"halves": binding.MARCHE_ROTARY_HALVES, "neighbours": binding.MARCHE_ROTARY_NEIGHBOURS}
BIG = 2 ** 31 - 1


# ------------------------------------------------------------------ append

def _table(rot):
    return np.array(rot.freq[:rot.n_pairs]), np.array(rot.axis[:rot.n_pairs])


def _turn_error(x, pos, freq, axis, layout):
    """What float32 may add to turned rows: sine and cosine off by 2^-22 (their argument,
    at most pi/4, rounded twice, their sums of terms, the last one rounded) and by the 64-bit
    angle's own error (its factors and itself rounded: 3 * 2^-53 of it); a product and
    the fused sum rounded, half a step (2^-24) of |x| + |y| each."""
    allow = np.zeros(np.shape(x))
    n = len(freq)
    for i in range(n):
        one, two = (i, i + n) if layout == "halves" else (2 * i, 2 * i + 1)
        t = np.abs(np.asarray(pos, np.float64)[axis[i]] * freq[i])[:, None]
        size = np.abs(x[..., one]) + np.abs(x[..., two])
        allow[..., one] = allow[..., two] = size * (2.0 ** -22 + 3 * 2.0 ** -53 * t + 2 * 2.0 ** -24)
    return allow


def _half_step(x, code, fmt):
    """Half a step of the format at values x of rows with these exponent codes."""
    if fmt == "bf16":
        return np.maximum(np.abs(x) * 2.0 ** -8, 2.0 ** -134)
    e = np.exp2(np.asarray(code, np.float64) - 127)[..., None]
    return 0.5 * e + 0 * x if fmt == "int8" else np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * e)


class Append:
    """Rows [queries | keys | values] behind other columns, of sequences in a pool."""

    def __init__(self, pool, rows, group, dtype, seed=0, extra=0, scale=1.0, before=0):
        rng = np.random.default_rng(seed)
        self.pool, self.rows, self.group, self.dtype = pool, rows, group, dtype
        H, dh, n = pool.H, pool.dh, sum(rows) + extra + before
        self.off = offsets(rows) + before
        self.heads = H * (group + 2)
        self.x = rnd(rng.standard_normal((n, self.heads, dh)) * scale, dtype)
        self.stride = 8 + self.heads * dh
        self.buf = torch.full((n, self.stride), float("nan"), dtype=TORCH[dtype], device="cuda")
        self.buf[:, 8:] = dev(self.x.reshape(n, -1), TORCH[dtype])
        self.D, self.n = H * group * dh, n
        self.q_out = torch.full((n, self.D + 16), 7.0, dtype=TORCH[dtype], device="cuda")

    def cut(self):
        D, E = self.D, self.pool.H * self.pool.dh
        b = self.buf[:, 8:]
        return b, b[:, D:], b[:, D + E:]

    def call(self, idx, rot, pos, q_out=None, off="csr", stream=None):
        p = self.pool
        q, k, v = self.cut()
        out = self.q_out if q_out is None else q_out
        binding.paged_append(p.cache, p.layer, p.dtable, p.width, len(self.rows), idx,
                             i32(self.off) if off == "csr" else None, self.n, rot, pos, q if self.group else None,
                             p.H * self.group, k, v, self.stride, DT[self.dtype], out if self.group else None,
                             out.stride(0), stream=stream)


APPEND_CASES = [
    # layout, pairs of each axis, per axis, group
    ("halves", [1.0], False, 2), ("halves", [0.25, 0.375, 0.375], False, 1), ("halves", [0.5], False, 4),
    ("neighbours", [1.0], False, 1), ("neighbours", [0.3, 0.3, 0.05], True, 3), ("neighbours", [0.2, 0.2, 0.2, 0.2], True, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,page", [(64, 64), (80, 16), (128, 32)])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", APPEND_CASES, ids=lambda c: f"{c[0]}{len(c[1])}g{c[3]}")
def test_append(case, fmt, dh, page, dtype):
    say(f"paged append {case} {fmt} {dh} {dtype}")
    layout, share, per_axis, group = case
    pairs = [int(s * dh // 2) for s in share]
    if layout == "halves":
        pairs[0] -= sum(pairs) % 4
    rot = binding.rotary(dh, LAYOUT[layout], pairs, per_axis, 10000.0)
    freq, axis = _table(rot)
    rng = np.random.default_rng(dh)
    lens, rows, H = [70, 0, 33, 5, 200], [9, 0, 17, 1, 40], 3
    pool = Pool(fmt, lens, H, dh, page, seed=1, layers=2, layer=1)
    a = Append(pool, rows, group, dtype, seed=2, extra=3)
    idx = np.concatenate([rng.permutation(n)[:r] for n, r in zip(lens, rows)] + [[0] * 3]).astype(np.int32)
    pos = rng.integers(-3000, 3000, (rot.n_axes, a.n)).astype(np.int32)
    pos[:, :4] = [0, 1 << 20, 123456789, -(1 << 30)]
    a.call(i32(idx), rot, i32(pos))
    torch.cuda.synchronize()
    n, off = sum(rows), a.off
    turned = ref.rotate(a.x[:n, :H * (group + 1)], pos[:, :n], freq, axis, layout)
    allow = _turn_error(a.x[:n, :H * (group + 1)], pos[:, :n], freq, axis, layout)
    got = a.q_out.double().cpu().numpy()
    assert (got[n:] == 7).all() and (got[:, a.D:] == 7).all()
    q = got[:n, :a.D].reshape(n, H * group, dh)
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    want, room = turned[:, :H * group], allow[:, :H * group]
    assert (np.abs(q - want) <= room + step * (np.abs(want) + room)).all()
    # the slots: keys within their roundings, values exact, everything else as it was
    before = {w: Pool(fmt, lens, H, dh, page, seed=1, layers=2, layer=1).layer_of(w) for w in ("k", "v")}
    for w in ("k", "v"):
        num, code = pool.layer_of(w)
        old, old_code = before[w]
        for b in range(len(lens)):
            for r in range(off[b], off[b + 1]):
                at, slot = pool.table[b][idx[r] // page], idx[r] % page
                x = a.x[r, H * (group + 1):] if w == "v" else turned[r, H * group:]
                if w == "v":
                    if fmt == "bf16":
                        np.testing.assert_array_equal(num[at, :, slot], rnd(x, "bf16"))
                    else:
                        y, c = ref.quantise(x, fmt)
                        np.testing.assert_array_equal(num[at, :, slot], y)
                        np.testing.assert_array_equal(code[at, :, slot], c)
                else:
                    room = allow[r, H * group:]
                    y = num[at, :, slot]
                    c = None
                    if fmt != "bf16":
                        c = code[at, :, slot]
                        most = np.abs(x).max(-1)
                        slack = room.max(-1)
                        lo, hi = (ref.quantise((most + s)[:, None], fmt)[1] for s in (-slack, slack))
                        assert ((lo <= c) & (c <= hi)).all()
                        y = ref.value(y, c)
                    assert (np.abs(y - x) <= room + _half_step(np.abs(x) + room, c, fmt)).all()
                old[at, :, slot] = num[at, :, slot]
                if fmt != "bf16":
                    old_code[at, :, slot] = code[at, :, slot]
        np.testing.assert_array_equal(num, old)
        if fmt != "bf16":
            np.testing.assert_array_equal(code, old_code)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_append_without_a_turn_is_a_write(fmt, dtype):
    """No pairs, or every position 0: queries come back and the cache holds what
    marche_paged_write puts there, bit for bit; enough rows for several heads a lane group."""
    say(f"paged append as write {fmt} {dtype}")
    lens = [300, 260, 129]
    for layout, pairs, pos in (("halves", [0], None), ("neighbours", [0, 0], None), ("halves", [32], "zero"), ("neighbours", [30], "zero")):
        rot = binding.rotary(64, LAYOUT[layout], pairs)
        one, two = (Pool(fmt, lens, 2, 64, 16, seed=3) for _ in range(2))
        a = Append(one, lens, 3, dtype, seed=5, scale=10.0)
        idx = i32(np.concatenate([np.arange(n)[::-1] for n in lens]))
        p = torch.zeros(rot.n_axes, a.n, dtype=torch.int32, device="cuda") if pos else None
        a.call(idx, rot, p)
        _, k, v = a.cut()
        binding.paged_write(two.cache, 0, two.dtable, two.width, 3, idx, i32(a.off), a.n, k, v, a.stride, DT[dtype])
        torch.cuda.synchronize()
        assert torch.equal(a.q_out[:, :a.D], a.cut()[0][:, :a.D])
        for x, y in ((one.dk, two.dk), (one.dv, two.dv), (one.dke, two.dke), (one.dve, two.dve)):
            assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_in_place_and_without_positions(fmt):
    """q_out is q; pos NULL means a_idx on every axis; equal numbers of rows need no
    offsets; the result does not depend on how many rows share the call."""
    say(f"paged append in place {fmt}")
    rot = binding.rotary(128, LAYOUT["halves"], [24, 40], True)
    lens, rows = [900] * 2, [700] * 2
    pool, small = (Pool(fmt, lens, 2, 128, 64, seed=3) for _ in range(2))
    a, b = (Append(pool, rows, 2, "bf16", seed=9) for _ in range(2))
    idx = np.concatenate([100 + np.arange(700), np.arange(700)]).astype(np.int32)
    a.call(i32(idx), rot, i32(np.stack([idx, idx])))
    k0, v0 = (t.clone() for t in (pool.dk, pool.dv))
    q = b.cut()[0]
    b.call(i32(idx), rot, None, q_out=q, off=None)
    torch.cuda.synchronize()
    assert torch.equal(q[:, :b.D], a.q_out[:, :a.D])
    assert torch.equal(k0.view(torch.uint8), pool.dk.view(torch.uint8)) and torch.equal(v0.view(torch.uint8), pool.dv.view(torch.uint8))
    # row by row
    d = Append(small, rows, 2, "bf16", seed=9)
    for r in (0, 699, 700, 1399):
        one = Append(small, [1], 2, "bf16")
        one.buf.copy_(d.buf[r:r + 1])
        seq = r // 700
        qq, k, v = one.cut()
        binding.paged_append(small.cache, 0, small.dtable[seq:seq + 1].contiguous(), small.width, 1, i32(idx[r:r + 1]), None, 1, rot,
                             None, qq, 4, k, v, one.stride, DT["bf16"], one.q_out, one.q_out.stride(0))
        torch.cuda.synchronize()
        assert torch.equal(one.q_out[0, :one.D], a.q_out[r, :a.D])
        page, slot = small.table[seq][idx[r] // 64], idx[r] % 64
        assert torch.equal(small.dk[0, page, :, slot].view(torch.uint8), pool.dk[0, page, :, slot].view(torch.uint8))


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_drops_what_has_no_page(fmt):
    """Tokens past the page table, negative ones and pages outside the pool are not
    written; their rows' queries are turned all the same.  Rows of no sequence are left."""
    say(f"paged append drops {fmt}")
    pool = Pool(fmt, [32, 32], 2, 64, 16, width_extra=0)
    pool.table[1] = [pool.n_pages, -7]
    pool.dtable = i32(pool.table)
    before = [pool.layer_of(w) for w in ("k", "v")]
    a = Append(pool, [3, 3], 1, "bf16", before=2, extra=2)
    a.buf[:2] = float("nan")
    rot = binding.rotary(64, LAYOUT["halves"], [32])
    a.call(i32([5, 6, 32, -1, BIG, 0, 16, 31, 7, 8]), rot, i32(np.arange(10)[None]))
    torch.cuda.synchronize()
    for w, b in zip(("k", "v"), before):
        np.testing.assert_array_equal(pool.layer_of(w)[0], b[0])
    got = a.q_out.double().cpu().numpy()
    assert (got[[0, 1, 8, 9]] == 7).all()
    want = ref.rotate(a.x[:, :2], np.arange(10)[None], *_table(rot), "halves").reshape(10, -1)[2:8]
    assert (np.abs(got[2:8, :a.D] - want) <= 2.0 ** -7 * np.abs(a.x[2:8, :2]).max()).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_of_rows_that_are_not_finite(fmt):
    """A row that is not finite, or whose turned values pass float32's range, reads back as
    NaN and leaves the rows beside it alone; what is not turned meets no sine."""
    say(f"paged append not finite {fmt}")
    pool = Pool(fmt, [16], 1, 64, 16)
    a = Append(pool, [6], 1, "f32")
    a.x[:] = 1.0
    a.x[0, 1, 3], a.x[1, 2, 60], a.x[2, 1, 40] = np.inf, np.nan, -np.inf
    a.x[3, 1, [0, 32]] = 3e38
    a.x[4, 0, 50] = np.inf
    a.buf[:, 8:] = dev(a.x.reshape(6, -1), torch.float32)
    rot = binding.rotary(64, LAYOUT["halves"], [32])
    rot.freq[0] = np.pi / 4
    a.call(i32(range(6)), rot, i32([[0, 1, 2, 1, 0, 3]]))
    k, v = pool.seq("k", 0), pool.seq("v", 0)
    assert np.isnan(k[[0, 2, 3]]).all() and np.isfinite(k[[1, 4, 5]]).all()
    assert np.isnan(v[1]).all() and (v[[0, 2, 3, 4, 5]] == 1).all()
    q = a.q_out[:, :64].cpu()
    assert q[4, 50].isinf() and q[4, 18].isnan() and q[4].isfinite().sum() == 62
    # channels of no pair
    b = Append(Pool(fmt, [16], 1, 64, 16), [1], 1, "f32")
    b.buf[0, 8 + 40] = float("inf")
    b.call(i32([3]), binding.rotary(64, LAYOUT["neighbours"], [18]), None)
    torch.cuda.synchronize()
    assert b.q_out[0, 40].isinf() and b.q_out[0, :64].isfinite().sum() == 63


def test_append_finds_sequences_among_many():
    """Row r's sequence, with empty sequences between."""
    say("paged append many sequences")
    rng = np.random.default_rng(5)
    n = 700
    rows = rng.integers(0, 3, n)
    rows[100:300] = 0
    rows[-1] = 0
    pool = Pool("int8", [1] * n, 1, 64, 16, seed=3)
    a = Append(pool, rows.tolist(), 1, "bf16")
    a.x[:] = rng.integers(-100, 100, a.x.shape)
    a.x[..., 0] = 127
    a.buf[:, 8:] = dev(a.x.reshape(a.n, -1), torch.bfloat16)
    idx = np.concatenate([np.arange(r) for r in rows]).astype(np.int32)
    a.call(i32(idx), binding.rotary(64, LAYOUT["halves"], [0]), None)
    torch.cuda.synchronize()
    k, v = pool.layer_of("k")[0], pool.layer_of("v")[0]
    for b in range(n):
        for r in range(a.off[b], a.off[b + 1]):
            np.testing.assert_array_equal(k[pool.table[b, 0], 0, idx[r]], a.x[r, 1])
            np.testing.assert_array_equal(v[pool.table[b, 0], 0, idx[r]], a.x[r, 2])


# ------------------------------------------------------------------ windows and trees

def _workspace(n):
    return torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device="cuda")


def window(pool, q, rows, group, dtype, t, size, sinks, o=None, off="csr", q_stride=None, stream=None, len_max=None, ws=None,
           lens=None):
    total, D, heads = len(t), pool.H * group * pool.dh, pool.H * group
    if o is None:
        o = torch.full((total, D), float("nan"), dtype=TORCH[dtype], device="cuda")
    len_max = max(pool.lens) if len_max is None else len_max
    n = binding.paged_attention_window_workspace_bytes(pool.cache, len(rows), total, max(rows), heads, len_max, size, sinks)
    ws = _workspace(n) if ws is None else ws
    off = i32(offsets(rows)) if isinstance(off, str) else off
    binding.paged_attention_window(pool.cache, pool.layer, pool.dtable, pool.width, pool.dlens if lens is None else lens, len_max,
                                   len(rows), q, q_stride or D, i32(t), off, total, max(rows), heads, DT[dtype], size, sinks, o, ws, n,
                                   stream=stream)
    torch.cuda.synchronize()
    return o


def tree(pool, q, rows, group, dtype, ctx, mask, o=None, off="csr", q_stride=None, stream=None, len_max=None):
    total, D, heads = len(mask), pool.H * group * pool.dh, pool.H * group
    if o is None:
        o = torch.full((total, D), float("nan"), dtype=TORCH[dtype], device="cuda")
    len_max = max(pool.lens) if len_max is None else len_max
    n = binding.paged_attention_tree_workspace_bytes(pool.cache, len(rows), total, max(rows), heads, len_max)
    off = i32(offsets(rows)) if isinstance(off, str) else off
    m = i32(np.asarray(mask).view(np.int32))
    binding.paged_attention_tree(pool.cache, pool.layer, pool.dtable, pool.width, pool.dlens, len_max, len(rows), q, q_stride or D, off,
                                 total, max(rows), heads, DT[dtype], i32(ctx), m, m.shape[1], o, _workspace(n), n, stream=stream)
    torch.cuda.synchronize()
    return o


def _window_look(pool, rows, t, size, sinks):
    off = offsets(rows)
    return [np.repeat(ref.window(t[off[b]:off[b + 1]], pool.lens[b], size, sinks)[:, None], pool.H, 1) for b in range(len(rows))]


def _tree_look(pool, rows, ctx, mask):
    off = offsets(rows)
    return [np.repeat(ref.tree(mask[off[b]:off[b + 1]], pool.lens[b], ctx[b])[:, None], pool.H, 1) for b in range(len(rows))]


WINDOW_CASES = [
    # lens, rows, group, page, window, sinks, tokens: each sequence's newest ("new"), or any
    ([150, 0, 1, 33, 700], [5, 3, 1, 0, 40], 1, 16, 7, 3, "any"),
    ([150, 0, 1, 33, 700], [5, 3, 1, 0, 40], 2, 32, 1, 0, "any"),
    ([150, 64, 1, 33, 700], [5, 64, 1, 33, 140], 4, 64, 100, 19, "new"),
    ([2500, 31], [1, 1], 4, 128, 1000, 4, "new"),
    ([9000], [1], 1, 64, 8500, 40, "new"),
    ([9000], [3], 7, 256, 40, 7000, "any"),
    ([513, 290], [300, 290], 1, 16, BIG, 0, "new"),
    ([513, 290], [90, 29], 2, 16, BIG, BIG, "any"),
    ([513, 290], [90, 29], 1, 64, 1, BIG, "any"),
    ([400] * 9, [17] * 9, 1, 32, 64, 0, "new"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", WINDOW_CASES, ids=lambda c: f"n{max(c[0])}r{sum(c[1])}g{c[2]}w{c[4]}s{c[5]}{c[6]}")
def test_window(case, fmt, dh, dtype):
    say(f"paged window {case} {fmt} {dh} {dtype}")
    lens, rows, group, page, size, sinks, where = case
    rng = np.random.default_rng(len(rows) + dh)
    pool = Pool(fmt, lens, 2, dh, page, seed=1, layers=2, layer=1)
    total = sum(rows)
    if where == "new":
        t = np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)])
    else:
        t = np.concatenate([rng.integers(-3, n + 10, r) for n, r in zip(lens, rows)])
        t[:2] = [BIG, -BIG - 1]
    q = rnd(2 * rng.standard_normal((total, 2 * group * dh)), dtype)
    got = window(pool, dev(q, TORCH[dtype]), rows, group, dtype, t, size, sinks).double().cpu().numpy()
    assert attention_errors(pool, got, q, rows, group, dtype, _window_look(pool, rows, t, size, sinks)) <= 1


TREE_CASES = [
    # lens, rows, group, page, words
    ([150, 20, 1, 33, 700], [5, 20, 1, 0, 40], 1, 16, 2),
    ([150, 20, 1, 33, 700], [8, 3, 1, 2, 64], 4, 64, 2),
    ([2500, 31], [1, 1], 4, 128, 1),
    ([9000], [7], 1, 64, 1),
    ([1100, 1000], [12, 25], 2, 256, 33),
    ([400] * 9, [17] * 9, 1, 32, 1),
]


def _tree_case(lens, rows, words, rng):
    """Masks of every kind, contexts at any token: drafted behind the mask's last word, none
    drafted, no context, rows without any bit."""
    ctx = np.array([max(0, n - r) for n, r in zip(lens, rows)])
    some = rng.random(len(lens)) < 0.4
    ctx = np.where(some, [rng.integers(0, n + 1) for n in lens], ctx)
    mask = rng.integers(0, 2 ** 32, (sum(rows), words), dtype=np.uint32)
    mask &= rng.integers(0, 2 ** 32, mask.shape, dtype=np.uint32)
    if len(mask):
        mask[0] = 0
        mask[-1] = 0xFFFFFFFF
    return ctx, mask


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 80, 128])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("case", TREE_CASES, ids=lambda c: f"n{max(c[0])}r{sum(c[1])}g{c[2]}w{c[4]}")
def test_tree(case, fmt, dh, dtype):
    say(f"paged tree {case} {fmt} {dh} {dtype}")
    lens, rows, group, page, words = case
    rng = np.random.default_rng(len(rows) + dh)
    pool = Pool(fmt, lens, 2, dh, page, seed=1, layers=2, layer=1)
    q = rnd(2 * rng.standard_normal((sum(rows), 2 * group * dh)), dtype)
    for ctx, mask in (_tree_case(lens, rows, words, rng), (np.full(len(lens), -7), _tree_case(lens, rows, words, rng)[1])):
        got = tree(pool, dev(q, TORCH[dtype]), rows, group, dtype, ctx, mask).double().cpu().numpy()
        assert attention_errors(pool, got, q, rows, group, dtype, _tree_look(pool, rows, ctx, mask)) <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing_get_zeros(dtype):
    """Empty masks, windows before the first token, whole blocks and single rows of them,
    on caches that are split and on others."""
    say(f"paged masks that leave nothing {dtype}")
    lens, rows = [6000, 40, 0], [33, 1, 2]
    pool = Pool("e4m3", lens, 1, 64, 16, seed=2)
    q = dev(np.ones((36, 64)), TORCH[dtype])
    t = np.full(36, -1)
    t[5] = 7000
    o = window(pool, q, rows, 1, dtype, t, 900, 0)
    assert (o == 0).all()
    o = window(pool, q, rows, 1, dtype, t, 900, 3).cpu()
    assert (o[5] != 0).any() and (o[[i for i in range(36) if i != 5]] == 0).all()
    mask = np.zeros((36, 3), np.uint32)
    o = tree(pool, q, rows, 1, dtype, [0, 0, 0], mask)
    assert (o == 0).all()
    mask[20, 2] = 1
    o = tree(pool, q, rows, 1, dtype, [0, 0, 0], mask).cpu()
    assert (o[20] != 0).any() and (o[[i for i in range(36) if i != 20]] == 0).all()
    # one drafted row of one short sequence
    pool = Pool("bf16", [5], 1, 64, 16, seed=2)
    assert (tree(pool, q[:1], [1], 1, dtype, [0], mask[:1] * 0) == 0).all()
    assert (window(pool, q[:1], [1], 1, dtype, [-1], 5, 5) == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows", [1, 3, 40, 150])
def test_masked_places_count_nothing(rows, fmt, dtype):
    """Infinities and NaN in masked keys and values, in tiles that rows see a part of."""
    say(f"paged masked infinities {fmt} {dtype} {rows}")
    rng = np.random.default_rng(3)
    n, dh, group = 400, 64, 2
    pool = Pool(fmt, [n], 2, dh, 16, seed=4)
    bad = [3, 150, 151, 249, n - 1]
    for j, x in zip(bad, (np.nan, np.inf, -np.inf, np.nan, np.inf)):
        page, slot = pool.table[0][j // 16], j % 16
        for d, e in ((pool.dk, pool.dke), (pool.dv, pool.dve)):
            if fmt == "bf16":
                d[0, page, :, slot, 5:9] = x
            else:
                d[0, page, :, slot] = 0x7F if fmt == "e4m3" else 0
                e[0, page, :, slot] = 255
    q = rnd(rng.standard_normal((rows, 2 * group * dh)), dtype)
    # every row sees the token before its own, up to 20 of them, and the first three
    t = np.array([250 + 20 + 119 * i // rows for i in range(rows)])
    t = np.where(t == n - 1, n - 2, t)
    got = window(pool, dev(q, TORCH[dtype]), [rows], group, dtype, t, 20, 3).double().cpu().numpy()
    assert np.isfinite(got).all()
    assert attention_errors(pool, got, q, [rows], group, dtype, _window_look(pool, [rows], t, 20, 3)) <= 1
    # a tree behind 3 tokens: bits of the bad tokens are clear
    words = 13
    mask = rng.integers(0, 2 ** 32, (rows, words), dtype=np.uint32)
    for j in bad:
        mask[:, (j - 3) // 32] &= ~np.uint32(1 << ((j - 3) % 32))
    got = tree(pool, dev(q, TORCH[dtype]), [rows], group, dtype, [3], mask).double().cpu().numpy()
    assert np.isfinite(got).all()
    assert attention_errors(pool, got, q, [rows], group, dtype, _tree_look(pool, [rows], [3], mask)) <= 1


def _inf_output(o, want):
    assert np.array_equal(np.isnan(o), np.isnan(want)) and np.array_equal(np.isinf(o), np.isinf(want))


@pytest.mark.parametrize("rows", [2, 100])
def test_seen_values_that_are_not_finite_stay_in_their_rows(rows):
    """An infinite value reaches its channel in the rows that see it, and no other."""
    say(f"paged seen infinities {rows}")
    n, dh = 200, 64
    pool = Pool("bf16", [n], 1, dh, 16, seed=4)
    page, slot = pool.table[0][100 // 16], 100 % 16
    pool.dv[0, page, 0, slot, 9] = float("inf")
    q = np.ones((rows, dh))
    t = np.array([100 + (i % 2) * 60 for i in range(rows)])
    o = window(pool, dev(q, torch.bfloat16), [rows], 1, "bf16", t, 30, 0).double().cpu().numpy()
    want = np.zeros((rows, dh))
    want[::2, 9] = np.inf
    _inf_output(o, want)
    mask = np.zeros((rows, 7), np.uint32)
    mask[:, 0] = 1
    mask[::2, 100 // 32] = 1 << (100 % 32)
    o = tree(pool, dev(q, torch.bfloat16), [rows], 1, "bf16", [0], mask).double().cpu().numpy()
    _inf_output(o, want)


@pytest.mark.parametrize("rows", [1, 40, 130])
def test_pages_that_no_row_sees_may_be_gone(monkeypatch, rows):
    """Pages before every window given back (their entries -1), with and without checks."""
    say(f"paged window, pages gone, {rows} rows")
    n, page = 1000, 16
    pool = Pool("int8", [n, n], 2, 64, page, seed=6)
    rng = np.random.default_rng(1)
    q = rnd(rng.standard_normal((2 * rows, 2 * 64)), "bf16")
    t = np.concatenate([np.arange(n - rows, n)] * 2)
    look = _window_look(pool, [rows] * 2, t, 50, 20)
    pool.table[:, 2:(n - rows - 50) // page] = -1
    pool.dtable = i32(pool.table)
    for validate in ("0", "1"):
        monkeypatch.setenv("MARCHE_VALIDATE", validate)
        got = window(pool, dev(q, torch.bfloat16), [rows] * 2, 1, "bf16", t, 50, 20).double().cpu().numpy()
        saved, pool.table = pool.table, np.where(pool.table < 0, 0, pool.table)  # (what no row sees)
        assert attention_errors(pool, got, q, [rows] * 2, 1, "bf16", look) <= 1
        pool.table = saved


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[3, 0, 2], [70, 1, 140]])
def test_layout_of_rows(dtype, rows):
    """Rows before the first sequence's and behind the last one's are left alone, strides
    and outputs of any place."""
    say(f"paged masks, layout of rows {dtype} {rows}")
    rng = np.random.default_rng(2)
    lens, before, extra, total = [300, 20, 600], 2, 3, sum(rows)
    pool = Pool("bf16", lens, 2, 64, 32, seed=7)
    q = rnd(rng.standard_normal((total, 128)), dtype)
    buf = torch.full((before + total + extra, 152), float("nan"), dtype=TORCH[dtype], device="cuda")
    buf[before:before + total, 8:136] = dev(q, TORCH[dtype])
    off = i32(offsets(rows) + before)
    t = np.concatenate([[BIG] * before] + [n - 1 - np.arange(r) for n, r in zip(lens, rows)] + [[5] * extra])
    mask = rng.integers(0, 2 ** 32, (before + total + extra, 2), dtype=np.uint32)
    ctx = [max(0, n - r) for n, r in zip(lens, rows)]
    for kind in ("window", "tree"):
        o = torch.full((before + total + extra, 128), 7.0, dtype=TORCH[dtype], device="cuda")
        if kind == "window":
            window(pool, buf[:, 8:], rows, 1, dtype, t, 77, 5, o=o, off=off, q_stride=152)
            look = _window_look(pool, rows, t[before:before + total], 77, 5)
        else:
            tree(pool, buf[:, 8:], rows, 1, dtype, ctx, mask, o=o, off=off, q_stride=152)
            look = _tree_look(pool, rows, ctx, mask[before:before + total])
        assert (o[:before] == 7).all() and (o[before + total:] == 7).all()
        got = o[before:before + total].double().cpu().numpy()
        assert attention_errors(pool, got, q, rows, 1, dtype, look) <= 1


def test_windows_past_every_token_are_the_whole_attention():
    """A window that ends at the last token and begins before the first: what
    marche_paged_attention gives, within roundings; lens cut by len_max."""
    say("paged window as whole attention")
    from paged_util import attention
    rng = np.random.default_rng(2)
    pool = Pool("e4m3", [700, 1300], 2, 128, 64, seed=8)
    rows = [4, 9]
    q = dev(rnd(rng.standard_normal((13, 2 * 4 * 128)), "f32"), torch.float32)
    t = [BIG - 1] * 13  # (a row at BIG does not see token 0 in a window of BIG)
    one = attention(pool, q, rows, 4, "f32", len_max=1100)
    for size, sinks in ((BIG, 0), (1, BIG)):
        two = window(pool, q, rows, 4, "f32", t, size, sinks, len_max=1100)
        assert (one - two).abs().max() <= 2.0 ** -18 * 6  # some 64 + 1300 fp32 steps of values below 6
    three = tree(pool, q, rows, 4, "f32", [BIG, BIG], np.zeros((13, 1), np.uint32), len_max=1100)
    assert (one - three).abs().max() <= 2.0 ** -18 * 6


# ------------------------------------------------------------------ together

class Drafts:
    """A model's layer that decodes on a cache: rows appended with their positions, then attention."""

    def __init__(self, fmt, dtype, lens, H=2, group=2, dh=64, page=16, seed=0):
        self.pool = Pool(fmt, lens, H, dh, page, seed=seed)
        self.H, self.group, self.dh, self.dtype = H, group, dh, dtype
        self.rot = binding.rotary(dh, LAYOUT["halves"], [8, 12, 12])
        self.rng = np.random.default_rng(seed + 1)
        self.q = None

    def append(self, rows, idx, pos):
        a = Append(self.pool, rows, self.group, self.dtype, seed=int(self.rng.integers(1 << 30)))
        a.call(i32(idx), self.rot, i32(pos))
        torch.cuda.synchronize()
        return a


@pytest.mark.parametrize("fmt,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("int8", "f32")])
def test_a_loop_that_drafts(fmt, dtype):
    """Prompts appended and attended to (windows), a tree of drafted tokens, one of its
    branches kept (moved up in the cache by appending it again) and one more token."""
    say(f"paged drafting loop {fmt} {dtype}")
    prompt, nodes = [37, 90], 6
    lens = [n + nodes for n in prompt]
    d = Drafts(fmt, dtype, lens)
    pool = d.pool

    def check(got, a, rows, look, n):
        """against the oracle on what the cache now holds and the turned queries that were returned"""
        saved, pool.lens = pool.lens, n
        q = a.q_out[:, :a.D].double().cpu().numpy()
        assert attention_errors(pool, got.double().cpu().numpy(), q, rows, d.group, dtype, look) <= 1
        pool.lens = saved

    # prompts: image tokens of 4 columns behind 5 places of text
    idx = np.concatenate([np.arange(n) for n in prompt])
    pos = np.stack([5 + idx // 64, idx // 4, idx % 4])
    a = d.append(prompt, idx, pos)
    pool.lens = prompt
    o = window(pool, a.q_out, prompt, d.group, dtype, idx, 24, 2, q_stride=a.q_out.stride(0), lens=i32(prompt))
    check(o, a, prompt, _window_look(pool, prompt, idx, 24, 2), prompt)
    want = ref.rotate(a.x[:, :4], pos, *_table(d.rot), "halves").reshape(len(idx), -1)
    assert np.abs(a.q_out[:, :a.D].double().cpu().numpy() - want).max() <= 2.0 ** -7 * np.abs(a.x).max()

    # drafts: two branches from the root, 0 - 1 - 3 and 0 - 2 - 4 - 5
    parent = [-1, 0, 0, 1, 2, 4]
    sees = []
    for i, p in enumerate(parent):
        sees.append((1 << i) | (sees[p] if p >= 0 else 0))
    mask = np.array(sees * 2, np.uint32)[:, None]
    depth = np.array([bin(s).count("1") - 1 for s in sees])
    idx = np.concatenate([n + np.arange(nodes) for n in prompt])
    at = np.concatenate([n + depth for n in prompt])
    pos = np.stack([5 + at // 64, at // 4, at % 4])
    pool.lens, pool.dlens = lens, i32(lens)
    a = d.append([nodes] * 2, idx, pos)
    o = tree(pool, a.q_out, [nodes] * 2, d.group, dtype, prompt, mask, q_stride=a.q_out.stride(0))
    check(o, a, [nodes] * 2, _tree_look(pool, [nodes] * 2, prompt, mask), lens)

    # the second branch is kept: its rows once more, side by side
    keep = [0, 2, 4, 5]
    rows = [4, 4]
    b = Append(pool, rows, d.group, dtype)
    pick = keep + [nodes + i for i in keep]
    b.buf.copy_(a.buf[pick])
    b.call(i32(np.concatenate([n + np.arange(4) for n in prompt])), d.rot, i32(np.ascontiguousarray(pos[:, pick])))
    after = [n + 4 for n in prompt]
    pool.lens, pool.dlens = after, i32(after)
    t = np.concatenate([n + np.arange(4) for n in prompt])
    o2 = window(pool, b.q_out, rows, d.group, dtype, t, BIG, 0, q_stride=b.q_out.stride(0))
    check(o2, b, rows, _window_look(pool, rows, t, BIG, 0), after)
    # the same rows over the same keys, in other tiles
    assert torch.equal(b.q_out[:, :b.D], a.q_out[pick][:, :a.D])
    np.testing.assert_allclose(o2.double().cpu().numpy(), o[pick].double().cpu().numpy(), rtol=0,
                               atol=0.05 if dtype == "bf16" else 1e-4)


def test_captured_loop_replays():
    """Append, window and tree attention captured in one graph, replayed after the inputs
    changed, with eager work between, against eager calls."""
    say("paged loop captured")
    lens, rows, group = [900, 5000, 64], [4, 4, 4], 2
    pools = [Pool("e4m3", lens, 2, 64, 16, seed=3) for _ in range(2)]
    a, b = (Append(p, rows, group, "bf16", seed=4) for p in pools)
    rot = binding.rotary(64, LAYOUT["neighbours"], [32])
    idx = i32(np.concatenate([np.arange(n - 4, n) for n in lens]))
    ctx, mask = i32([n - 4 for n in lens]), i32(np.array([[1], [3], [5], [9]] * 3))
    off, bf = i32(offsets(rows)), DT["bf16"]
    heads = 2 * group

    def make(p, x):
        n1 = binding.paged_attention_window_workspace_bytes(p.cache, 3, 12, 4, heads, 5000, 3000, 4)
        n2 = binding.paged_attention_tree_workspace_bytes(p.cache, 3, 12, 4, heads, 5000)
        w1, w2 = _workspace(n1), _workspace(n2)
        o1, o2 = (torch.zeros(12, heads * 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        qs, (q, k, v) = x.q_out.stride(0), x.cut()

        def run(stream):
            binding.paged_append(p.cache, 0, p.dtable, p.width, 3, idx, off, 12, rot, None, q, heads, k, v, x.stride, bf, x.q_out, qs,
                                 stream=stream)
            binding.paged_attention_window(p.cache, 0, p.dtable, p.width, p.dlens, 5000, 3, x.q_out, qs, idx, off, 12, 4, heads, bf,
                                           3000, 4, o1, w1, n1, stream=stream)
            binding.paged_attention_tree(p.cache, 0, p.dtable, p.width, p.dlens, 5000, 3, x.q_out, qs, off, 12, 4, heads, bf, ctx,
                                         mask, 1, o2, w2, n2, stream=stream)
        return run, o1, o2

    eager, e1, e2 = make(pools[0], a)
    run, o1, o2 = make(pools[1], b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        run(side)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            run(torch.cuda.current_stream())
    for i in range(4):
        new = dev(rnd(np.random.default_rng(i).standard_normal(a.buf.shape), "bf16"), torch.bfloat16)
        a.buf.copy_(new)
        b.buf.copy_(new)
        b.q_out.fill_(3)
        o1.fill_(float("nan"))
        o2.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(a.q_out[:, :a.D], b.q_out[:, :b.D]) and torch.equal(e1, o1) and torch.equal(e2, o2)
        assert e1.isfinite().all() and torch.equal(pools[0].dk, pools[1].dk) and torch.equal(pools[0].dve, pools[1].dve)


def test_two_streams():
    """Calls in flight on two streams, each with a workspace of its own, give what they give alone."""
    say("paged masks on two streams")
    rng = np.random.default_rng(1)
    pool = Pool("int8", [8000, 3], 2, 128, 64, seed=5)
    q = [dev(rnd(rng.standard_normal((4, 2 * 2 * 128)), "bf16"), torch.bfloat16) for _ in range(2)]
    t, mask = [7999, 7000, 2, 1], np.array([[1], [3], [1], [3]], np.uint32)
    alone = [window(pool, q[0], [2, 2], 2, "bf16", t, 5000, 4), tree(pool, q[1], [2, 2], 2, "bf16", [7990, 1], mask)]
    n = [binding.paged_attention_window_workspace_bytes(pool.cache, 2, 4, 2, 4, 8000, 5000, 4),
         binding.paged_attention_tree_workspace_bytes(pool.cache, 2, 4, 2, 4, 8000)]
    ws, streams = [_workspace(x) for x in n], [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros(4, 512, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    args = i32(t), i32(offsets([2, 2])), i32([7990, 1]), i32(mask.view(np.int32))
    torch.cuda.synchronize()
    for _ in range(10):
        binding.paged_attention_window(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 8000, 2, q[0], 512, args[0], args[1], 4, 2,
                                       4, DT["bf16"], 5000, 4, outs[0], ws[0], n[0], stream=streams[0])
        binding.paged_attention_tree(pool.cache, 0, pool.dtable, pool.width, pool.dlens, 8000, 2, q[1], 512, args[1], 4, 2, 4,
                                     DT["bf16"], args[2], args[3], 1, outs[1], ws[1], n[1], stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1])


# ------------------------------------------------------------------ debug validation

def test_validated_calls(monkeypatch):
    say("paged loop validated")
    monkeypatch.setenv("MARCHE_VALIDATE", "1")
    pool = Pool("bf16", [64, 40], 1, 64, 16, width_extra=0)
    q = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    mask = np.ones((2, 1), np.uint32)
    tree(pool, q, [1, 1], 1, "bf16", [64, 0], mask)
    window(pool, q, [1, 1], 1, "bf16", [-5, BIG], 3, 0)
    for ctx in ([65, 0], [3, -1]):
        with pytest.raises(binding.MarcheError, match="context out of range"):
            tree(pool, q, [1, 1], 1, "bf16", ctx, mask)
    with pytest.raises(binding.MarcheError, match="length"):
        window(pool, q, [1, 1], 1, "bf16", [0, 0], 3, 0, lens=i32([65, 3]))
    with pytest.raises(binding.MarcheError, match="offsets"):
        window(pool, q, [1, 1], 1, "bf16", [0, 0], 3, 0, off=i32([0, 2, 1]))
    pool.dtable = i32([[0, 1, 2, 99], [3, 4, 5, -1]])
    with pytest.raises(binding.MarcheError, match="page outside"):
        tree(pool, q, [1, 1], 1, "bf16", [1, 1], mask)
    a = Append(pool, [1, 1], 1, "bf16")
    rot = binding.rotary(64, LAYOUT["halves"], [32])
    for idx, word in (([0, 64], "token out"), ([-1, 0], "token out"), ([50, 3], "page outside")):
        with pytest.raises(binding.MarcheError, match=word):
            a.call(i32(idx), rot, None)
    a.call(i32([3, 4]), rot, None)
    torch.cuda.synchronize()
