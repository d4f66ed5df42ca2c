"""Operators of a paged key/value cache, whose time on the GPU is measured.

The cache is a pool of pages, ``[n_pages][heads][page][head_dim]`` for K and
for V, that sequences reach through a page table.  It holds bf16, or 8 bits
(e4m3 or int8) with one power-of-two exponent per token and head, so that
quantising and reading back are exact operations.  Five kinds of passes:

* ``write``: rows of new keys and values, quantised into their tokens' slots;
* ``read``: the cached tokens back in the resident layout;
* ``bounds``: per page and head the largest and smallest key channel, in 8
  bits (what the selection scores pages with);
* ``attend``: attention of one or more new rows per sequence over its cache;
* ``select``: the pages whose bounds promise each row the highest logits, and
  the attention over those pages alone.

With ``own`` unset a pass is plain torch in 32 bits, otherwise the framework's
calls (``binding.paged_*``).  ``exact`` is the definition in 64 bits, sequence
by sequence.
"""
import math

import torch

DEV = "cuda"
own = False

LIMIT = {"e4m3": 448.0, "int8": 127.0}
LEAST_EXP = -111  # the exponent of a row of zeros and of rows too small for a smaller one


def listed():
    return [
        # One new token for each of eight sequences, as every decoding step of
        # an interactive service writes it: latency is everything.
        dict(name="write-token-8", op="write", fmt="e4m3", dtype="bf16", seqs=8, heads=16, group=1,
             head_dim=64, page=64, len_lo=300, len_hi=2000, rows_lo=1, rows_hi=1),
        # The full step of the headline batch: every token of 128 images.
        dict(name="write-full-128", op="write", fmt="int8", dtype="bf16", seqs=128, heads=16, group=1,
             head_dim=64, page=64, len_lo=320, len_hi=320, rows_lo=320, rows_hi=320),
        # A few short sequences of odd lengths (one of them empty) read back in
        # fp32, heads of width 80.
        dict(name="read-odd-5", op="read", fmt="int8", dtype="f32", seqs=5, heads=16, group=1,
             head_dim=80, page=32, len_lo=0, len_hi=229, rows_lo=1, rows_hi=1),
        # The cached segment of 64 high-resolution images for the attention
        # over two resident segments.
        dict(name="read-hires-64", op="read", fmt="e4m3", dtype="bf16", seqs=64, heads=16, group=1,
             head_dim=64, page=64, len_lo=1088, len_hi=1088, rows_lo=1, rows_hi=1),
        # Bounds of the last page after a new token, shared key heads.
        dict(name="bounds-tail-32", op="bounds", fmt="bf16", dtype="bf16", seqs=32, heads=8, group=4,
             head_dim=128, page=64, len_lo=100, len_hi=4000, rows_lo=1, rows_hi=1, tail=True),
        # Bounds of whole caches after a full step.
        dict(name="bounds-hires-64", op="bounds", fmt="e4m3", dtype="bf16", seqs=64, heads=16, group=1,
             head_dim=64, page=32, len_lo=1024, len_hi=1088, rows_lo=1, rows_hi=1, tail=False),
        # The smallest call: one row over one image's 320 tokens.
        dict(name="attend-token-1", op="attend", fmt="bf16", dtype="bf16", seqs=1, heads=16, group=1,
             head_dim=64, page=64, len_lo=320, len_hi=320, rows_lo=1, rows_hi=1),
        # The active rows of the headline batch's cache-aware step (images at
        # different points of their schedules) over an 8-bit cache.
        dict(name="attend-step-128", op="attend", fmt="e4m3", dtype="bf16", seqs=128, heads=16, group=1,
             head_dim=64, page=64, len_lo=320, len_hi=320, rows_lo=9, rows_hi=71),
        # One new token over long ragged caches, four query heads to a key head.
        dict(name="attend-long-16", op="attend", fmt="int8", dtype="bf16", seqs=16, heads=8, group=4,
             head_dim=128, page=64, len_lo=4000, len_hi=32768, rows_lo=1, rows_hi=1),
        # fp32 rows, from one to a few hundred, over caches of odd lengths (one
        # of them empty), heads of width 80.
        dict(name="attend-odd-f32-6", op="attend", fmt="int8", dtype="f32", seqs=6, heads=16, group=1,
             head_dim=80, page=16, len_lo=0, len_hi=1503, rows_lo=1, rows_hi=333),
        # One new token that looks at 32 pages of a long cache.
        dict(name="select-token-8", op="select", fmt="e4m3", dtype="bf16", seqs=8, heads=8, group=4,
             head_dim=128, page=64, len_lo=30000, len_hi=32768, rows_lo=1, rows_hi=1, n_select=32),
        # Active rows of high-resolution images, each over 8 pages of its own.
        dict(name="select-hires-32", op="select", fmt="bf16", dtype="bf16", seqs=32, heads=16, group=1,
             head_dim=64, page=32, len_lo=1088, len_hi=1088, rows_lo=36, rows_hi=100, n_select=8),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _draw(rng):
    op = rng.choice(["write", "read", "bounds", "attend", "attend", "select"])
    heads, group, dh = rng.choice([(12, 1, 64), (16, 1, 64), (16, 1, 80), (8, 4, 128), (2, 7, 64), (1, 8, 80)])
    c = dict(op=op, fmt=rng.choice(["bf16", "e4m3", "int8"]), dtype="f32" if rng.random() < 0.25 else "bf16",
             seqs=_log(rng, 1, 128), heads=heads, group=group, head_dim=dh, page=rng.choice([16, 32, 64, 128, 256]))
    top = 16384 if c["page"] == 16 else 32768
    a, b = _log(rng, 1, top), _log(rng, 1, top)
    c["len_lo"], c["len_hi"] = min(a, b) - (rng.random() < 0.2), max(a, b)
    c["rows_lo"] = c["rows_hi"] = 1
    if op == "write" or (op in ("attend", "select") and rng.random() < 0.5):
        a, b = _log(rng, 1, 400), _log(rng, 1, 400)
        c["rows_lo"], c["rows_hi"] = min(a, b), max(a, b)
    if op == "write":
        c["rows_hi"] = min(c["rows_hi"], c["len_hi"])
        c["rows_lo"] = min(c["rows_lo"], c["rows_hi"])
    if op == "bounds":
        c["tail"] = rng.random() < 0.3
    if op == "select":
        c["n_select"] = _log(rng, 1, 64)
    return c


def _plain_bytes(c):
    """Memory of a plain pass's largest intermediates and of the state."""
    pages = sum(_pages(c))
    tokens = max(pages * c["page"], c["seqs"] * max(_pages(c)) * c["page"])
    n = tokens * c["heads"] * c["head_dim"] * 20
    if c["op"] in ("attend", "select"):
        n += c["seqs"] * c["heads"] * c["group"] * c["rows_hi"] * max(_pages(c)) * c["page"] * 16
    return n


def _cost(c):
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / 0.7e15


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most and _plain_bytes(c) <= 40e9:
            return c


# ------------------------------------------------------------------ sizes

def _spread(lo, hi, n):
    """n sizes from hi down to lo (hi alone for one)."""
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _lens(c):
    lens = _spread(c["len_lo"], c["len_hi"], c["seqs"])
    return lens[::2] + lens[1::2][::-1]


def _rows(c):
    """New rows of each sequence; written rows are tokens of it."""
    rows = _spread(c["rows_lo"], c["rows_hi"], c["seqs"])[::-1]
    return [min(r, n) for r, n in zip(rows, _lens(c))] if c["op"] == "write" else rows


def _pages(c):
    return [-(-n // c["page"]) for n in _lens(c)]


def work(case):
    """Each input read once and each output written once: rows, the cached
    tokens that the rows see, page bounds, and what the call returns."""
    c = case
    es, io = {"bf16": 2, "e4m3": 1, "int8": 1}[c["fmt"]], {"bf16": 2, "f32": 4}[c["dtype"]]
    H, dh = c["heads"], c["head_dim"]
    row = H * (dh * es + (c["fmt"] != "bf16"))  # one token's K or V
    lens, rows, pages = _lens(c), _rows(c), _pages(c)
    n = sum(rows)
    if c["op"] == "write":
        return {"bytes": 2.0 * n * (row + H * dh * io) + 8.0 * n, "flops": 0.0}
    if c["op"] == "read":
        return {"bytes": 2.0 * sum(lens) * (row + H * dh * io) + 4.0 * sum(pages), "flops": 0.0}
    bound = H * (2 * dh + 1)
    if c["op"] == "bounds":
        seen = [min(x, (x - 1) % c["page"] + 1) if c["tail"] else x for x in lens]
        some = [min(p, 1) if c["tail"] else p for p in pages]
        return {"bytes": float(sum(seen)) * row + float(sum(some)) * (bound + 4), "flops": 0.0}
    D = H * c["group"] * dh
    if c["op"] == "attend":
        return {"bytes": 2.0 * sum(lens) * row + 2.0 * n * D * io + 4.0 * sum(pages),
                "flops": 4.0 * D * sum(r * x for r, x in zip(rows, lens))}
    k = c["n_select"]
    seen = [min(x, r * k * c["page"]) for r, x in zip(rows, lens)]
    each = [min(x, k * c["page"]) for x in lens]
    return {"bytes": 2.0 * sum(seen) * row + float(sum(pages)) * (bound + 4) + 2.0 * n * D * io + 4.0 * n * H * k,
            "flops": 4.0 * D * sum(r * x for r, x in zip(rows, each)) +
            2.0 * D * sum(r * p for r, p in zip(rows, pages))}


# ------------------------------------------------------------------ inputs

def _exp_of(amax, limit):
    """The least exponent e >= LEAST_EXP with amax <= limit * 2^e."""
    e = torch.frexp(amax / limit).exponent  # amax/limit in [2^(e-1), 2^e)
    e = torch.where(torch.ldexp(torch.full_like(amax, limit), e - 1) >= amax, e - 1, e)
    return torch.where(amax > 0, e, LEAST_EXP).clamp(min=LEAST_EXP)


def _quantise(x, fmt):
    """Rows (last axis) in 8 bits: values of the format and exponent codes."""
    x = x.float()
    e = _exp_of(x.abs().amax(-1), LIMIT[fmt])
    y = torch.ldexp(x, -e[..., None])
    q = y.to(torch.float8_e4m3fn) if fmt == "e4m3" else torch.round(y).to(torch.int8)
    return q, (e + 127).to(torch.uint8)


def _value(q, code):
    """What quantised rows stand for, in 32 bits."""
    return torch.ldexp(q.float(), code.int()[..., None] - 127)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    H, dh, page = c["heads"], c["head_dim"], c["page"]
    lens, rows, pages = _lens(c), _rows(c), _pages(c)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    # pages of the sequences in any order, among others that belong to nobody here
    total, width = sum(pages) + 3, max(1, max(pages))
    perm = torch.randperm(total, generator=g, device=DEV).int()
    table = torch.full((c["seqs"], width), -1, dtype=torch.int32, device=DEV)
    have = torch.arange(width, device=DEV) < torch.tensor(pages, device=DEV)[:, None]
    table[have] = perm[:sum(pages)]
    # keys of a page resemble each other, and some channels are large
    channel = 1.0 + 3.0 * (torch.rand(H, 1, dh, generator=g, device=DEV) < 0.06)
    k = (0.6 * rnd(total, H, 1, dh) + 0.8 * rnd(total, H, page, dh)) * channel
    v = rnd(total, H, page, dh)
    s = {"case": c, "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device=DEV)}
    if c["fmt"] == "bf16":
        s["k"], s["v"], s["k_exp"], s["v_exp"] = k.bfloat16(), v.bfloat16(), None, None
    else:
        (s["k"], s["k_exp"]), (s["v"], s["v_exp"]) = _quantise(k, c["fmt"]), _quantise(v, c["fmt"])
    del k, v
    off = torch.tensor([0] + rows, device=DEV).cumsum(0)
    s["off"], s["total"], s["most"], s["len_max"] = off.int(), sum(rows), max(rows), max(lens)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    s["dtype"] = dt
    n = s["total"]
    if c["op"] == "write":
        # distinct tokens of each sequence, the newest for a single row; K and V
        # rows are parts of a projection's [queries | keys | values]
        pick = [torch.tensor([x - 1]) if r == 1 else torch.randperm(x, generator=torch.Generator().manual_seed(
            int(seed) % (1 << 31) + 31 * b))[:r] for b, (r, x) in enumerate(zip(rows, lens))]
        s["idx"] = torch.cat(pick).int().to(DEV)[:n] if n else torch.zeros(0, dtype=torch.int32, device=DEV)
        s["qkv"] = rnd(n, 3 * H * dh).to(dt)
    if c["op"] == "read":
        s["k_out"] = torch.zeros(c["seqs"], H, max(1, max(lens)), dh, dtype=dt, device=DEV)
        s["v_out"] = torch.zeros_like(s["k_out"])
    if c["op"] in ("bounds", "select"):
        s["bounds"] = torch.zeros(total, H, 2, dh, dtype=torch.int8, device=DEV)
        s["bounds_exp"] = torch.zeros(total, H, dtype=torch.uint8, device=DEV)
        s["first"] = (s["lens"] - 1).clamp(min=0) if c.get("tail") else None
    if c["op"] in ("attend", "select"):
        s["q"] = rnd(n, H * c["group"] * dh).to(dt)
        s["o"] = torch.zeros(n, H * c["group"] * dh, dtype=dt, device=DEV)
    if c["op"] == "select":
        s["pages"] = torch.empty(n, H, c["n_select"], dtype=torch.int32, device=DEV)
        _plain_bounds(s, None)
    return s


# ------------------------------------------------------------------ a pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


def _handle(s):
    """The cache's handle, which a program makes once."""
    from paper_2506_12035_amd import binding
    if "handle" not in s:
        c = s["case"]
        fmt = {"bf16": binding.MARCHE_CACHE_BF16, "e4m3": binding.MARCHE_CACHE_E4M3,
               "int8": binding.MARCHE_CACHE_INT8}[c["fmt"]]
        s["handle"] = binding.paged_cache(1, s["k"].shape[0], c["heads"], c["page"], c["head_dim"], fmt, s["k"],
                                          s["v"], s["k_exp"], s["v_exp"], s.get("bounds"), s.get("bounds_exp"))
        s["dt"] = binding.MARCHE_F32 if c["dtype"] == "f32" else binding.MARCHE_BF16
        if c["op"] in ("attend", "select"):
            s["ws_bytes"] = binding.paged_attention_workspace_bytes(
                s["handle"], c["seqs"], s["total"], s["most"], c["heads"] * c["group"], s["len_max"],
                c.get("n_select", 0))
            s["ws"] = torch.empty(max(s["ws_bytes"], 256), dtype=torch.uint8, device=DEV)
        if c["op"] == "write":
            D = c["heads"] * c["head_dim"]
            s["new"] = s["qkv"][:, D:2 * D], s["qkv"][:, 2 * D:]
    return binding, s["handle"], torch.cuda.current_stream()


def _stored(s):
    return [t for t in (s["k"], s["v"], s["k_exp"], s["v_exp"]) if t is not None]


def _own_write(s):
    b, cache, stream = _handle(s)
    b.paged_write(cache, 0, s["table"], s["table"].shape[1], s["case"]["seqs"], s["idx"], s["off"], s["total"],
                  s["new"][0], s["new"][1], s["qkv"].shape[1], s["dt"], stream=stream)
    return _stored(s)


def _own_read(s):
    b, cache, stream = _handle(s)
    b.paged_read(cache, 0, s["table"], s["table"].shape[1], s["lens"], s["case"]["seqs"], s["k_out"].shape[2],
                 s["k_out"], s["v_out"], s["dt"], stream=stream)
    return s["k_out"], s["v_out"]


def _own_bounds(s):
    b, cache, stream = _handle(s)
    width = s["table"].shape[1]
    b.paged_bounds(cache, 0, s["table"], width, s["lens"], s["first"], 1 if s["case"]["tail"] else width,
                   s["case"]["seqs"], stream=stream)
    return s["bounds"], s["bounds_exp"]


def _own_attention(s, b, cache, stream, pages, n_select):
    c = s["case"]
    b.paged_attention(cache, 0, s["table"], s["table"].shape[1], s["lens"], s["len_max"], c["seqs"], s["q"],
                      s["q"].shape[1], s["off"], s["total"], s["most"], c["heads"] * c["group"], s["dt"], s["o"],
                      pages, n_select, s["ws"], s["ws_bytes"], stream=stream)


def _own_attend(s):
    _own_attention(s, *_handle(s), None, 0)
    return s["o"]


def _own_select(s):
    b, cache, stream = _handle(s)
    c = s["case"]
    b.paged_select(cache, 0, s["table"], s["table"].shape[1], s["lens"], c["seqs"], s["q"], s["q"].shape[1],
                   s["off"], s["total"], c["heads"] * c["group"], s["dt"], c["n_select"], s["pages"], stream=stream)
    _own_attention(s, b, cache, stream, s["pages"], c["n_select"])
    return s["pages"], s["o"]


_OWN = {"write": _own_write, "read": _own_read, "bounds": _own_bounds, "attend": _own_attend, "select": _own_select}


# ------------------------------------------------------------------ plain forms

def _row_seq(s):
    """Sequence of each row."""
    return torch.searchsorted(s["off"][1:].contiguous(), torch.arange(s["total"], device=DEV), right=True)


def _plain_write(s):
    c = s["case"]
    H, dh = c["heads"], c["head_dim"]
    tok = s["idx"].long()
    at, slot = s["table"][_row_seq(s), tok // c["page"]].long(), tok % c["page"]
    new = s["qkv"].view(-1, 3, H, dh)
    if c["fmt"] == "bf16":
        s["k"][at, :, slot], s["v"][at, :, slot] = new[:, 1].bfloat16(), new[:, 2].bfloat16()
    else:
        kq, ke = _quantise(new[:, 1], c["fmt"])
        vq, ve = _quantise(new[:, 2], c["fmt"])
        s["k"].view(torch.int8)[at, :, slot], s["k_exp"][at, :, slot] = kq.view(torch.int8), ke
        s["v"].view(torch.int8)[at, :, slot], s["v_exp"][at, :, slot] = vq.view(torch.int8), ve
    return _stored(s)


def _values(s, which, at):
    """K or V of pages in 32 bits."""
    t, e = s[which], s[which + "_exp"]
    return t[at].float() if e is None else _value(t.view(torch.int8)[at].view(t.dtype), e[at])


def _resident(s, which):
    """K or V of every sequence in 32 bits, [seqs][heads][tokens][head_dim],
    zero past its length."""
    x = _values(s, which, s["table"].clamp(min=0).long())
    B, P, H, page, dh = x.shape
    x = x.permute(0, 2, 1, 3, 4).reshape(B, H, P * page, dh)
    seen = torch.arange(P * page, device=DEV) < s["lens"][:, None]
    return x.masked_fill_(~seen[:, None, :, None], 0.0), seen


def _plain_read(s):
    n = s["k_out"].shape[2]
    return tuple(_resident(s, w)[0][:, :, :n].to(s["dtype"]) for w in ("k", "v"))


def _plain_bounds(s, first):
    """Bounds of the pages from those of the tokens `first` on, in place."""
    c = s["case"]
    start = torch.arange(s["table"].shape[1], device=DEV) * c["page"]
    todo = start < s["lens"][:, None]
    if first is not None:
        todo &= start + c["page"] > first[:, None]
    at = s["table"][todo].long()
    seen = (s["lens"][:, None] - start)[todo][:, None] > torch.arange(c["page"], device=DEV)
    k = _values(s, "k", at)
    hi = k.masked_fill(~seen[:, None, :, None], -math.inf).amax(2)
    lo = k.masked_fill(~seen[:, None, :, None], math.inf).amin(2)
    both = torch.stack((hi, lo), 2)
    e = _exp_of(both.abs().amax((2, 3)), 127.0)
    s["bounds"][at] = torch.round(torch.ldexp(both, -e[..., None, None])).to(torch.int8)
    s["bounds_exp"][at] = (e + 127).to(torch.uint8)
    return s["bounds"], s["bounds_exp"]


def _padded(s):
    """Rows of each sequence side by side: indexes and which of them exist."""
    i = torch.arange(s["most"], device=DEV)
    at = s["off"][:-1, None] + i
    return at.clamp(max=s["total"] - 1).long(), at < s["off"][1:, None]


def _attention(s, allowed):
    """`allowed`: None, or which pages each row may look at, per key head."""
    c = s["case"]
    H, G, dh, page = c["heads"], c["group"], c["head_dim"], c["page"]
    at, real = _padded(s)
    B, R = at.shape
    q = s["q"][at].float().view(B, R, H, G, dh).permute(0, 2, 1, 3, 4).reshape(B, H, R * G, dh)
    k, seen = _resident(s, "k")
    x = torch.matmul(q, k.transpose(2, 3)).view(B, H, R, G, -1) / math.sqrt(dh)
    del k
    off = ~seen[:, None, None, None, :]
    if allowed is not None:
        off = off | ~allowed[at].permute(0, 2, 1, 3).repeat_interleave(page, 3)[:, :, :, None, :]
    x.masked_fill_(off, -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(m.masked_fill(m == -math.inf, 0.0)).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, H, R * G, -1), _resident(s, "v")[0]).view(B, H, R, G, dh)
    o = (o / z.masked_fill(z == 0, 1.0)).permute(0, 2, 1, 3, 4).reshape(B, R, H * G * dh)
    out = torch.zeros_like(s["o"])
    out[at[real]] = o[real].to(s["dtype"])
    return out


def _plain_select(s):
    c = s["case"]
    H, G, dh, k = c["heads"], c["group"], c["head_dim"], c["n_select"]
    seq = _row_seq(s)
    q, e = _quantise(s["q"].view(-1, H, G, dh), "int8")
    q = q.float()
    at, real = _padded(s)
    B, R = at.shape
    P = s["table"].shape[1]
    both = s["bounds"][s["table"].clamp(min=0).long()].float().permute(0, 2, 1, 3, 4)  # [B][H][P][2][dh]
    signs = torch.stack((q.clamp(min=0), q.clamp(max=0)), 3)[at]                        # [B][R][H][G][2][dh]
    signs = signs.permute(0, 2, 1, 3, 4, 5).reshape(B, H, R * G, 2 * dh)
    whole = torch.matmul(signs, both.reshape(B, H, P, 2 * dh).transpose(2, 3)).view(B, H, R, G, P)
    be = s["bounds_exp"][s["table"].clamp(min=0).long()].int().transpose(1, 2) - 127    # [B][H][P]
    qe = e.int()[at].permute(0, 2, 1, 3) - 127                                          # [B][H][R][G]
    score = torch.ldexp(torch.ldexp(whole, be[:, :, None, None, :]), qe[..., None]).amax(3)  # [B][H][R][P]
    score = score.permute(0, 2, 1, 3)[real]                                             # [rows][H][P]
    have = torch.arange(P, device=DEV) * c["page"] < s["lens"][seq][:, None]
    score = score.masked_fill(~have[:, None], -math.inf)
    best, order = score.sort(dim=-1, descending=True, stable=True)
    order = order.masked_fill(best == -math.inf, P)[..., :k]
    order = torch.nn.functional.pad(order, (0, k - order.shape[-1]), value=P).sort(-1).values
    pages = order.masked_fill(order == P, -1).int()
    allowed = torch.zeros(*score.shape[:2], P + 1, dtype=torch.bool, device=DEV).scatter_(2, order, True)[..., :P]
    return pages, _attention(s, allowed)


_PLAIN = {"write": _plain_write, "read": _plain_read, "bounds": lambda s: _plain_bounds(s, s["first"]),
          "attend": lambda s: _attention(s, None), "select": _plain_select}


# ------------------------------------------------------------------ 64 bits

def _exact_rows(x, fmt):
    """Rows of 64-bit values in the 8-bit format: the values, and codes."""
    amax = x.abs().amax(-1)
    e = torch.full_like(amax, LEAST_EXP)
    while bool((amax > LIMIT[fmt] * torch.exp2(e)).any()):
        e = torch.where(amax > LIMIT[fmt] * torch.exp2(e), e + 1, e)
    y = x / torch.exp2(e)[..., None]
    if fmt == "int8":
        return torch.round(y), e + 127
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)  # 3 bits behind the first
    return torch.round(y / step) * step, e + 127


def _exact_kv(s, which, b):
    """Sequence b's cached K or V in 64 bits, [tokens][heads][head_dim]."""
    c, n = s["case"], int(s["lens"][b])
    j = torch.arange(n, device=DEV)
    at, slot = s["table"][b].long()[j // c["page"]], j % c["page"]
    if s[which + "_exp"] is None:
        return s[which][at, :, slot].double()
    raw = s[which].view(torch.int8)[at, :, slot].view(s[which].dtype)
    raw = raw.float().double() if c["fmt"] == "e4m3" else raw.double()
    return raw * torch.exp2(s[which + "_exp"][at, :, slot].double() - 127)[..., None]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    H, G, dh, page = c["heads"], c["group"], c["head_dim"], c["page"]
    off = s["off"].tolist()
    if c["op"] == "write":
        tokens = [(b, i) for b in range(c["seqs"]) for i in range(off[b], off[b + 1])]
        seq = torch.tensor([b for b, _ in tokens], dtype=torch.long, device=DEV)
        tok = s["idx"].long()
        at, slot = s["table"][seq, tok // page].long(), tok % page
        out, codes = [], []
        for w, lo in (("k", H * dh), ("v", 2 * H * dh)):
            x = s["qkv"][:, lo:lo + H * dh].double().view(-1, H, dh)
            if c["fmt"] == "bf16":
                t = s[w].double()
                t[at, :, slot] = x
                out.append(t)
                continue
            q, e = _exact_rows(x, c["fmt"])
            t, u = s[w].float().double(), s[w + "_exp"].clone()
            t[at, :, slot], u[at, :, slot] = q, e.to(torch.uint8)
            out.append(t.to(torch.int8) if c["fmt"] == "int8" else t)
            codes.append(u)
        return out + codes
    if c["op"] == "read":
        out = [torch.zeros(s["k_out"].shape, dtype=torch.float64, device=DEV) for _ in range(2)]
        for b, n in enumerate(_lens(c)):
            for t, w in zip(out, ("k", "v")):
                t[b, :, :n] = _exact_kv(s, w, b).transpose(0, 1)
        return tuple(out)
    if c["op"] == "bounds":
        for b, n in enumerate(_lens(c)):
            k = _exact_kv(s, "k", b)
            for p in range((n - 1) // page if c["tail"] and n else 0, -(-n // page)):
                x = k[p * page:(p + 1) * page]
                q, e = _exact_rows(torch.cat((x.amax(0), x.amin(0)), -1), "int8")
                at = int(s["table"][b, p])
                s["bounds"][at], s["bounds_exp"][at] = q.view(H, 2, dh).to(torch.int8), e.to(torch.uint8)
        return s["bounds"], s["bounds_exp"]
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV)
    pages = torch.full((s["total"], H, c.get("n_select", 1)), -1, dtype=torch.int32, device=DEV)
    lens = _lens(c)
    for b, n in enumerate(lens):
        lo, hi = off[b], off[b + 1]
        if n == 0 or hi == lo:
            continue
        k, v = _exact_kv(s, "k", b), _exact_kv(s, "v", b)
        q = s["q"][lo:hi].double().view(hi - lo, H, G, dh)
        for h in range(H):
            x = (q[:, h].reshape(-1, dh) @ k[:, h].t().contiguous()).view(hi - lo, G, n) / math.sqrt(dh)
            if c["op"] == "select":
                q8, qe = _exact_rows(q[:, h], "int8")
                at = s["table"][b, :-(-n // page)].long()
                top, bot = s["bounds"][at, h, 0].double(), s["bounds"][at, h, 1].double()
                best = (q8.clamp(min=0).reshape(-1, dh) @ top.t().contiguous() +
                        q8.clamp(max=0).reshape(-1, dh) @ bot.t().contiguous()).view(hi - lo, G, -1)
                best = best * torch.exp2(qe - 127)[..., None] * torch.exp2(s["bounds_exp"][at, h].double() - 127)
                order = best.amax(1).argsort(dim=-1, descending=True, stable=True)[:, :c["n_select"]].sort(-1).values
                pages[lo:hi, h, :order.shape[1]] = order.int()
                look = torch.zeros(hi - lo, at.numel(), dtype=torch.bool, device=DEV).scatter_(1, order, True)
                x = x.masked_fill(~look[:, torch.arange(n, device=DEV) // page][:, None], -math.inf)
            p = torch.softmax(x, -1)
            o[lo:hi].view(hi - lo, H, G, dh)[:, h] = (p.view(-1, n) @ v[:, h].contiguous()).view(hi - lo, G, dh)
    return o if c["op"] == "attend" else (pages, o)
